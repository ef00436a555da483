// Attention of a decoding step's rows over a cache held in 4 bits (qcache.h: the format).
#include "attn_rows_simple.h"
#include "qcache.h"

namespace pkv {

namespace {

struct RowsOfCache {
    const unsigned char *k, *ks, *v, *vs;
    QLayout lay;
    int h;
    __device__ static float at(const unsigned char* codes, int d, uint32_t scale) {
        const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[d / 2], q_scale(scale), 0);
        return d & 1 ? p[1] : p[0];
    }
    __device__ float key(int64_t t, int d) const {
        return at(k + lay.code(h, t), d, ks[lay.k_scale(h, t, d / kQBlock)]);
    }
    __device__ float value(int64_t t, int d) const {
        return at(v + lay.code(h, t), d, vs[lay.v_scale(h, t, d / kQBlock)]);
    }
};

template <typename T>
__global__ __launch_bounds__(64) void qcache_attn_simple_kernel(
    const T* q, pkv_qcache cache, const int32_t* row_pos, const int32_t* seq_start, T* out,
    float* lse, int rows_each, int hq, int hkv, QLayout lay, float scale) {
    const int64_t row = blockIdx.x / hq;
    const int h = blockIdx.x % hq;
    int64_t start = seq_start ? seq_start[row / rows_each] : 0;
    start = start < 0 ? 0 : start > lay.rows ? lay.rows : start;
    const int64_t end = start + row_pos[row] + 1;
    const RowsOfCache src = {
        (const unsigned char*)cache.k_codes, (const unsigned char*)cache.k_scales,
        (const unsigned char*)cache.v_codes, (const unsigned char*)cache.v_scales, lay,
        h / (hq / hkv)};
    const int64_t o = row * hq + h;
    attend_simple<T>(q + o * lay.D, src, start, end < lay.rows ? end : lay.rows, lay.D, scale,
                     out + o * lay.D, lse ? lse + o : nullptr);
}

}  // namespace

size_t qcache_attn_ws_bytes(const pkv_layer_cfg&, int64_t, int64_t, int64_t) { return 0; }

pkv_status launch_qcache_attn(const pkv_layer_cfg& cfg, const void* q, const pkv_qcache& cache,
                              const int32_t* row_pos, const int32_t* seq_start, void* out,
                              float* lse_out, int64_t m, int64_t n_seq, float scale, void*,
                              hipStream_t st) {
    const dim3 grid((unsigned)(m * cfg.n_q_heads));
    const QLayout lay = {cache.rows, cfg.head_dim};
    const int each = (int)(m / n_seq);
    if (cfg.dtype == PKV_BF16)
        hipLaunchKernelGGL((qcache_attn_simple_kernel<bf16_t>), grid, dim3(64), 0, st,
                           (const bf16_t*)q, cache, row_pos, seq_start, (bf16_t*)out, lse_out, each,
                           cfg.n_q_heads, cfg.n_kv_heads, lay, scale);
    else
        hipLaunchKernelGGL((qcache_attn_simple_kernel<float>), grid, dim3(64), 0, st,
                           (const float*)q, cache, row_pos, seq_start, (float*)out, lse_out, each,
                           cfg.n_q_heads, cfg.n_kv_heads, lay, scale);
    return launch_status();
}

}  // namespace pkv
