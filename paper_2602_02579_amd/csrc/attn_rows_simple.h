// Attention of one (row, head) by one wave, for any head_dim: 64 keys at a time, a key per lane for
// the scores, an element of the head per lane for the products with the values.
#pragma once

#include "pkv_common.h"

namespace pkv {

// keys lo <= t < hi; src.key(t, d), src.value(t, d): elements as fp32
template <typename T, typename Src>
__device__ __forceinline__ void attend_simple(const T* __restrict__ q, const Src& src, int64_t lo,
                                              int64_t hi, int D, float scale, T* out, float* lse) {
    __shared__ float s_q[256], s_p[64];
    const int lane = threadIdx.x;
    for (int d = lane; d < D; d += 64) s_q[d] = Elem<T>::load(q + d) * scale;
    __syncthreads();
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, mx = -INFINITY, sum = 0.f;
    for (int64_t t0 = lo; t0 < hi; t0 += 64) {
        const int64_t t = t0 + lane;
        float s = -INFINITY;
        if (t < hi) {
            s = 0.f;
            for (int d = 0; d < D; ++d) s += s_q[d] * src.key(t, d);
        }
        float m = s;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        m = fmaxf(m, mx);
        const float ref = m == -INFINITY ? 0.f : m;
        const float corr = expf(mx - ref), p = expf(s - ref);
        float ps = p;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) ps += __shfl_xor(ps, o);
        sum = sum * corr + ps;
        mx = m;
        s_p[lane] = p;
        __syncthreads();
        const int n = (int)(hi - t0 < 64 ? hi - t0 : 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = lane + 64 * i;
            if (d >= D) continue;
            float a = acc[i] * corr;
            for (int j = 0; j < n; ++j) a += s_p[j] * src.value(t0 + j, d);
            acc[i] = a;
        }
        __syncthreads();
    }
    const float inv = lo < hi ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < D) out[lane + 64 * i] = Elem<T>::from_f32(acc[i] * inv);
    if (lane == 0 && lse) *lse = lo < hi ? mx + logf(sum) : -INFINITY;
}

}  // namespace pkv
