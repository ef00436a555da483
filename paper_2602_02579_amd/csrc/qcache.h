// The 4-bit format of a cache (pkv_qcache): 16 neighbouring elements of a head share a scale
// 2^(byte - 127), an element is a code of one sign, two exponent and one mantissa bit
// (0, 0.5, 1, 1.5, 2, 3, 4, 6).  Two significant bits times a power of two: every value is exact in
// bf16, and gfx950 converts in both directions with the scale as an operand.
#pragma once

#include "pkv_common.h"

namespace pkv {

constexpr int kQBlock = 16;                    // elements that share a scale
constexpr int kQScaleMin = 32, kQScaleMax = 252;
constexpr int kQScaleNan = 255;

// offsets in bytes; head-major, so that a head's keys are consecutive for the attention
struct QLayout {
    int64_t rows;
    int D;
    __device__ __forceinline__ int64_t code(int h, int64_t t) const {
        return (h * rows + t) * (D / 2);
    }
    __device__ __forceinline__ int64_t k_scale(int h, int64_t t, int b) const {
        return (h * rows + t) * (D / kQBlock) + b;
    }
    __device__ __forceinline__ int64_t v_scale(int h, int64_t t, int b) const {
        return ((h * (rows / 8) + t / 8) * (D / kQBlock) + b) * 8 + t % 8;
    }
};

__device__ __forceinline__ float q_scale(uint32_t byte) {
    return __uint_as_float(byte == kQScaleNan ? 0x7fc00000u : byte << 23);
}

}  // namespace pkv
