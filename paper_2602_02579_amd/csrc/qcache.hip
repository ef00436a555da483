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

// A thread owns 16 elements of a head, a workgroup all of them for 256 / (D / 16) tokens and one head:
// rows that follow each other in the cache are then written in runs of hundreds of bytes, codes and
// scales (a workgroup for all heads of few tokens wrote value scales byte by byte into 64 lines:
// 32k tokens of 8 heads of 128 43 us).  blockIdx.z: keys or values.  Bound by the bytes: 32k tokens of 8
// heads of 128 in bf16, 134 MB in and 38 MB out, 32.4 us, 5.3 TB/s (a large copy: 5.1; with two, four and
// eight tokens a thread 32.4, 33.2 and 34.3).
template <typename T>
__global__ __launch_bounds__(256) void qcache_store_kernel(const T* __restrict__ k,
                                                           const T* __restrict__ v,
                                                           const int32_t* __restrict__ dst_row,
                                                           pkv_qcache cache, int64_t m, int heads,
                                                           int blocks, QLayout lay) {
    typedef typename Vec16<T>::type vec_t;
    constexpr int N = Vec16<T>::N;
    const int in_tile = threadIdx.x / blocks, b = threadIdx.x - in_tile * blocks;
    const int tile_rows = 256 / blocks, h = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * tile_rows + in_tile;
    if (in_tile >= tile_rows || i >= m) return;
    const vec_t* src = reinterpret_cast<const vec_t*>((blockIdx.z ? v : k) +
                                                      (i * heads + h) * lay.D + b * kQBlock);
    vec_t x[kQBlock / N];
#pragma unroll
    for (int p = 0; p < kQBlock / N; ++p) x[p] = __builtin_nontemporal_load(src + p);
    const int64_t row = dst_row ? dst_row[i] : i;
    if (row < 0 || row >= lay.rows) return;
    float f[kQBlock];
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < kQBlock; ++e) {
        f[e] = Elem<T>::to_f32(x[e / N][e % N]);
        top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
    }
    const uint32_t byte = scale_byte(top);
    uint2 codes = make_uint2(0, 0);
    if (byte != kQScaleNan) {
        const float s = q_scale(byte);
        codes = make_uint2(encode8(f, s), encode8(f + 8, s));
    }
    unsigned char* cd = static_cast<unsigned char*>(blockIdx.z ? cache.v_codes : cache.k_codes);
    *reinterpret_cast<uint2*>(cd + lay.code(h, row) + b * 8) = codes;
    if (blockIdx.z)
        static_cast<unsigned char*>(cache.v_scales)[lay.v_scale(h, row, b)] = (unsigned char)byte;
    else
        static_cast<unsigned char*>(cache.k_scales)[lay.k_scale(h, row, b)] = (unsigned char)byte;
}

// A thread owns, for one token, 8 pairs of elements (i, i + D / 2) and walks over heads_each heads:
// sines and cosines are worked out once, under the latency of the first heads' bytes.  blockIdx.y: which
// heads, blockIdx.z: keys or values.  Bound by the bytes written: 32k tokens of 8 heads of 128 to bf16, 38 MB in
// and 134 MB out, 28 us out of a warm cache, 38 out of a cold one, however the heads and the stores are laid
// out; 7 chunks of 512 out of a store 6.9 us, of which the bytes are 3.7.
template <typename T>
__global__ __launch_bounds__(256) void qcache_restore_kernel(
    pkv_qcache cache, const int32_t* __restrict__ row_idx, const int32_t* __restrict__ pos,
    int64_t pos_base, bool rotate, T* __restrict__ k_out, T* __restrict__ v_out, int64_t total,
    int heads, int heads_each, QLayout lay, RopeTable tab) {
    typedef typename Vec16<T>::type vec_t;
    constexpr int HB = 4;                 // heads whose bytes are requested together
    const int half = lay.D / 2, chunks = half / 8;
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w >= total) return;
    const int64_t i = w / chunks, row = row_idx ? row_idx[i] : i;
    const int d0 = (int)(w - i * chunks) * 8;
    if (row < 0 || row >= lay.rows) return;
    const bool keys = blockIdx.z == 0, turn = keys && rotate;
    const unsigned char* codes = static_cast<const unsigned char*>(keys ? cache.k_codes : cache.v_codes);
    const unsigned char* scales =
        static_cast<const unsigned char*>(keys ? cache.k_scales : cache.v_scales);
    T* out = (keys ? k_out : v_out) + i * heads * lay.D + d0;
    const int head0 = blockIdx.y * heads_each, head_end = min(heads, head0 + heads_each);
    uint32_t c[HB][2];
    unsigned char b[HB][2];
    auto load = [&](int h0) {
#pragma unroll
        for (int u = 0; u < HB; ++u)
            if (h0 + u < head_end)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int h = h0 + u, d = d0 + s * half, blk = d / kQBlock;
                    c[u][s] = *reinterpret_cast<const uint32_t*>(codes + lay.code(h, row) + d / 2);
                    b[u][s] = scales[keys ? lay.k_scale(h, row, blk) : lay.v_scale(h, row, blk)];
                }
    };
    load(head0);
    float sn[8], cs[8];
    if (turn) {
        const double p = pos ? (double)pos[i] : (double)(pos_base + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) rope_sincos(p, tab.inv_freq[d0 + j], &sn[j], &cs[j]);
    }
    for (int h0 = head0; h0 < head_end; h0 += HB) {
        if (h0 > head0) load(h0);
#pragma unroll
        for (int u = 0; u < HB; ++u) {
            if (h0 + u >= head_end) break;
            float x[2][8];
#pragma unroll
            for (int s = 0; s < 2; ++s) decode8(c[u][s], q_scale(b[u][s]), x[s]);
            if (turn) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float p = x[0][j], q = x[1][j];
                    x[0][j] = p * cs[j] - q * sn[j];
                    x[1][j] = q * cs[j] + p * sn[j];
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
                    __builtin_nontemporal_store(
                        o, reinterpret_cast<vec_t*>(out + (h0 + u) * lay.D + s * half) + p);
                }
        }
    }
}

}  // namespace

pkv_status launch_qcache_store(const pkv_layer_cfg& cfg, const void* k, const void* v,
                               const int32_t* dst_row, const pkv_qcache& cache, int64_t m,
                               hipStream_t st) {
    const int blocks = cfg.head_dim / kQBlock;
    const int64_t tiles = ceil_div(m, 256 / blocks);
    if (tiles >= 1 << 24) return PKV_ERR_UNSUPPORTED;   // a launch holds less than 2^32 threads a side
    const dim3 grid((unsigned)tiles, (unsigned)cfg.n_kv_heads, 2);
    const QLayout lay = {cache.rows, cfg.head_dim};
    if (cfg.dtype == PKV_BF16)
        hipLaunchKernelGGL((qcache_store_kernel<bf16_t>), grid, dim3(256), 0, st, (const bf16_t*)k,
                           (const bf16_t*)v, dst_row, cache, m, cfg.n_kv_heads, blocks, lay);
    else
        hipLaunchKernelGGL((qcache_store_kernel<float>), grid, dim3(256), 0, st, (const float*)k,
                           (const float*)v, dst_row, cache, m, cfg.n_kv_heads, blocks, lay);
    return launch_status();
}

pkv_status launch_qcache_restore(const pkv_layer_cfg& cfg, const pkv_qcache& cache,
                                 const int32_t* row_idx, const int32_t* pos, int64_t pos_base,
                                 bool rotate, void* k_out, void* v_out, int64_t m,
                                 hipStream_t st) {
    // the table of a configuration, which a program hardly changes: its 64 powers take 3 us
    static thread_local struct { int head_dim; float theta; RopeTable tab; } last = {};
    if (rotate && (last.head_dim != cfg.head_dim || last.theta != cfg.rope_theta)) {
        fill_rope_table(&last.tab, cfg.head_dim, (double)cfg.rope_theta);
        last.head_dim = cfg.head_dim;
        last.theta = cfg.rope_theta;
    }
    const RopeTable& tab = last.tab;
    const int64_t total = m * (cfg.head_dim / 16);
    const int64_t blocks = ceil_div(total, 256);
    if (blocks >= 1 << 24) return PKV_ERR_UNSUPPORTED;
    // heads in as many parts as bring the launch to two workgroups per CU; more would only make sines anew
    const int64_t parts = std::min<int64_t>(cfg.n_kv_heads, std::max<int64_t>(1, 256 / blocks));
    const int each = (int)ceil_div(cfg.n_kv_heads, parts);
    const dim3 grid((unsigned)blocks, (unsigned)ceil_div(cfg.n_kv_heads, each), 2);
    const QLayout lay = {cache.rows, cfg.head_dim};
    if (cfg.dtype == PKV_BF16)
        hipLaunchKernelGGL((qcache_restore_kernel<bf16_t>), grid, dim3(256), 0, st, cache, row_idx,
                           pos, pos_base, rotate, (bf16_t*)k_out, (bf16_t*)v_out, total,
                           cfg.n_kv_heads, each, lay, tab);
    else
        hipLaunchKernelGGL((qcache_restore_kernel<float>), grid, dim3(256), 0, st, cache, row_idx,
                           pos, pos_base, rotate, (float*)k_out, (float*)v_out, total,
                           cfg.n_kv_heads, each, lay, tab);
    return launch_status();
}

}  // namespace pkv
