// Exchanges between the lanes of a wave that stay in the vector unit (an LDS permutation takes some 100
// clocks, and the setting up of a small attention is a chain of them).
#pragma once

#include "pkv_common.h"

namespace pkv {

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// v of another lane: CTRL 0x120 + n: of the 16, rotated by n; 0x110 + n: n lanes in front (`old` where
// there is none); 0x142, 0x143: the last of the 16, of the 32 in front.  ROWS: which rows of 16 receive.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int dpp(int old, int v) {
    return __builtin_amdgcn_update_dpp(old, v, CTRL, ROWS, 0xf, false);
}
// over 16 lanes, for all of them; over the first 32 lanes of the wave, uniform
__device__ __forceinline__ int min16(int v) {
    v = min(v, dpp<0x128>(v, v));
    v = min(v, dpp<0x124>(v, v));
    v = min(v, dpp<0x122>(v, v));
    return min(v, dpp<0x121>(v, v));
}
__device__ __forceinline__ int max16(int v) { return ~min16(~v); }
__device__ __forceinline__ int min32(int v) {
    v = min16(v);
    return min(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16));
}
__device__ __forceinline__ int max32(int v) { return ~min32(~v); }

// Bits a .. b - 1 of 32, whatever a and b are; x, or -infinity where a bit is not set.  (Comparisons of
// every element with both ends go through scalar registers: 16 of them took some 800 clocks.)
__device__ __forceinline__ uint32_t bits_between(int a, int b) {
    const uint32_t below_b = b >= 32 ? ~0u : (1u << max(b, 0)) - 1u;
    const uint32_t below_a = a >= 32 ? ~0u : (1u << max(a, 0)) - 1u;
    return below_b & ~below_a;
}
__device__ __forceinline__ float where_bit(uint32_t bits, int at, float x) {
    const uint32_t on = (uint32_t)__builtin_amdgcn_sbfe((int)bits, at, 1);   // all bits, or none
    return __uint_as_float((on & __float_as_uint(x)) | (~on & 0xff800000u));
}

__device__ __forceinline__ int wave_scan(int v) {   // inclusive
    v += dpp<0x111>(0, v);
    v += dpp<0x112>(0, v);
    v += dpp<0x114>(0, v);
    v += dpp<0x118>(0, v);
    v += dpp<0x142, 0xa>(0, v);
    return v + dpp<0x143, 0xc>(0, v);
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }

}  // namespace pkv
