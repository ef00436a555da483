// Keys and values into a cache in 4 bits, and back with their positions (qcache.h: the format).
#include <algorithm>

#include "qcache.h"

namespace pkv {

namespace {

// The scale byte of 16 elements of which `top` holds the largest magnitude's bits (as integers, so
// that a NaN is the largest of all).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return kQScaleNan;
    const int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) >= 0x600000u ? 1 : 0);
    return (uint32_t)min(max(e, kQScaleMin), kQScaleMax);
}

// 8 fp32 values to 8 codes
__device__ __forceinline__ uint32_t encode8(const float* x, float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    return c;
}

__device__ __forceinline__ void decode8(uint32_t c, float scale, float* x) {
    f32x2 p;
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0);
    x[0] = p[0]; x[1] = p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
    x[2] = p[0]; x[3] = p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2);
    x[4] = p[0]; x[5] = p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
    x[6] = p[0]; x[7] = p[1];
}

// A thread owns 16 elements of a head; blockIdx.y: keys or values.
template <typename T>
__global__ __launch_bounds__(256) void qcache_store_kernel(const T* __restrict__ k,
                                                           const T* __restrict__ v,
                                                           const int32_t* __restrict__ dst_row,
                                                           pkv_qcache cache, int64_t total,
                                                           int heads, QLayout lay) {
    typedef typename Vec16<T>::type vec_t;
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w >= total) return;
    const int blocks = lay.D / kQBlock;
    const int b = (int)(w % blocks);
    const int64_t rh = w / blocks;
    const int h = (int)(rh % heads);
    const int64_t i = rh / heads, row = dst_row ? dst_row[i] : i;
    if (row < 0 || row >= lay.rows) return;
    const vec_t* src = reinterpret_cast<const vec_t*>((blockIdx.y ? v : k) + w * kQBlock);
    float x[kQBlock];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < kQBlock / Vec16<T>::N; ++p) {
        const vec_t a = src[p];
#pragma unroll
        for (int e = 0; e < Vec16<T>::N; ++e) {
            const float f = Elem<T>::to_f32(a[e]);
            x[p * Vec16<T>::N + e] = f;
            top = max(top, __float_as_uint(f) & 0x7fffffffu);
        }
    }
    const uint32_t byte = scale_byte(top);
    uint2 codes = make_uint2(0, 0);
    if (byte != kQScaleNan) {
        const float s = q_scale(byte);
        codes = make_uint2(encode8(x, s), encode8(x + 8, s));
    }
    unsigned char* cd = static_cast<unsigned char*>(blockIdx.y ? cache.v_codes : cache.k_codes);
    *reinterpret_cast<uint2*>(cd + lay.code(h, row) + b * 8) = codes;
    if (blockIdx.y)
        static_cast<unsigned char*>(cache.v_scales)[lay.v_scale(h, row, b)] = (unsigned char)byte;
    else
        static_cast<unsigned char*>(cache.k_scales)[lay.k_scale(h, row, b)] = (unsigned char)byte;
}

// A thread owns, for one token, 8 pairs of elements (i, i + D / 2) and walks over the heads: sines and
// cosines are worked out once.  blockIdx.y: keys or values.
template <typename T>
__global__ __launch_bounds__(256) void qcache_restore_kernel(
    pkv_qcache cache, const int32_t* __restrict__ row_idx, const int32_t* __restrict__ pos,
    int64_t pos_base, bool rotate, T* __restrict__ k_out, T* __restrict__ v_out, int64_t total,
    int heads, QLayout lay, RopeTable tab) {
    typedef typename Vec16<T>::type vec_t;
    const int half = lay.D / 2, chunks = half / 8;
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w >= total) return;
    const int64_t i = w / chunks, row = row_idx ? row_idx[i] : i;
    const int d0 = (int)(w - i * chunks) * 8;
    if (row < 0 || row >= lay.rows) return;
    const bool keys = blockIdx.y == 0, turn = keys && rotate;
    const unsigned char* codes = static_cast<const unsigned char*>(keys ? cache.k_codes : cache.v_codes);
    const unsigned char* scales =
        static_cast<const unsigned char*>(keys ? cache.k_scales : cache.v_scales);
    T* out = (keys ? k_out : v_out) + i * heads * lay.D;
    float sn[8], cs[8];
    if (turn) {
        const double p = pos ? (double)pos[i] : (double)(pos_base + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) rope_sincos(p, tab.inv_freq[d0 + j], &sn[j], &cs[j]);
    }
    for (int h = 0; h < heads; ++h) {
        float x[2][8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int d = d0 + s * half, b = d / kQBlock;
            const uint32_t c =
                *reinterpret_cast<const uint32_t*>(codes + lay.code(h, row) + d / 2);
            decode8(c, q_scale(scales[keys ? lay.k_scale(h, row, b) : lay.v_scale(h, row, b)]), x[s]);
        }
        if (turn) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float a = x[0][j], b = x[1][j];
                x[0][j] = a * cs[j] - b * sn[j];
                x[1][j] = b * cs[j] + a * sn[j];
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int p = 0; p < 8 / Vec16<T>::N; ++p) {
                vec_t o;
#pragma unroll
                for (int e = 0; e < Vec16<T>::N; ++e)
                    o[e] = Elem<T>::from_f32(x[s][p * Vec16<T>::N + e]);
                reinterpret_cast<vec_t*>(out + h * lay.D + d0 + s * half)[p] = o;
            }
    }
}

}  // namespace

pkv_status launch_qcache_store(const pkv_layer_cfg& cfg, const void* k, const void* v,
                               const int32_t* dst_row, const pkv_qcache& cache, int64_t m,
                               hipStream_t st) {
    const int64_t total = m * cfg.n_kv_heads * (cfg.head_dim / kQBlock);
    const int64_t blocks = ceil_div(total, 256);
    if (blocks > INT32_MAX) return PKV_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, 2);
    const QLayout lay = {cache.rows, cfg.head_dim};
    if (cfg.dtype == PKV_BF16)
        hipLaunchKernelGGL((qcache_store_kernel<bf16_t>), grid, dim3(256), 0, st, (const bf16_t*)k,
                           (const bf16_t*)v, dst_row, cache, total, cfg.n_kv_heads, lay);
    else
        hipLaunchKernelGGL((qcache_store_kernel<float>), grid, dim3(256), 0, st, (const float*)k,
                           (const float*)v, dst_row, cache, total, cfg.n_kv_heads, lay);
    return launch_status();
}

pkv_status launch_qcache_restore(const pkv_layer_cfg& cfg, const pkv_qcache& cache,
                                 const int32_t* row_idx, const int32_t* pos, int64_t pos_base,
                                 bool rotate, void* k_out, void* v_out, int64_t m,
                                 hipStream_t st) {
    RopeTable tab;
    fill_rope_table(&tab, cfg.head_dim, (double)cfg.rope_theta);
    const int64_t total = m * (cfg.head_dim / 16);
    const int64_t blocks = ceil_div(total, 256);
    if (blocks > INT32_MAX) return PKV_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, 2);
    const QLayout lay = {cache.rows, cfg.head_dim};
    if (cfg.dtype == PKV_BF16)
        hipLaunchKernelGGL((qcache_restore_kernel<bf16_t>), grid, dim3(256), 0, st, cache, row_idx,
                           pos, pos_base, rotate, (bf16_t*)k_out, (bf16_t*)v_out, total,
                           cfg.n_kv_heads, lay, tab);
    else
        hipLaunchKernelGGL((qcache_restore_kernel<float>), grid, dim3(256), 0, st, cache, row_idx,
                           pos, pos_base, rotate, (float*)k_out, (float*)v_out, total,
                           cfg.n_kv_heads, lay, tab);
    return launch_status();
}

}  // namespace pkv
