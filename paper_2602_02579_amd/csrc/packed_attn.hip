// Causal attention over a packed prompt: row i attends the row_pos[i] + 1 rows that end with itself.
// (Paper: Sec. 2 - the method's input are chunks that were prefilled one by one.)
#include "attn_rows_simple.h"

namespace pkv {

namespace {

template <typename T>
struct RowsOfPrompt {
    const T *k, *v;   // of the kv head
    int64_t stride;
    __device__ float key(int64_t t, int d) const { return Elem<T>::load(k + t * stride + d); }
    __device__ float value(int64_t t, int d) const { return Elem<T>::load(v + t * stride + d); }
};

template <typename T>
__global__ __launch_bounds__(64) void packed_simple_kernel(const T* q, const T* k, const T* v,
                                                           const int32_t* row_pos, T* out,
                                                           float* lse, int hq, int hkv, int D,
                                                           float scale) {
    const int64_t row = blockIdx.x / hq;
    const int h = blockIdx.x % hq, g = h / (hq / hkv);
    const int64_t pos = row_pos[row] < row ? row_pos[row] : row;
    const RowsOfPrompt<T> src = {k + g * D, v + g * D, (int64_t)hkv * D};
    const int64_t o = row * hq + h;
    attend_simple<T>(q + o * D, src, pos < 0 ? row + 1 : row - pos, row + 1, D, scale, out + o * D,
                     lse ? lse + o : nullptr);
}

}  // namespace

size_t packed_attn_ws_bytes(const pkv_layer_cfg&, int64_t) { return 0; }

pkv_status launch_packed_attn(const pkv_layer_cfg& cfg, const void* q, const void* k,
                              const void* v, const int32_t* row_pos, void* out, float* lse_out,
                              int64_t m, float scale, void*, hipStream_t st) {
    const dim3 grid((unsigned)(m * cfg.n_q_heads));
    if (cfg.dtype == PKV_BF16)
        hipLaunchKernelGGL((packed_simple_kernel<bf16_t>), grid, dim3(64), 0, st, (const bf16_t*)q,
                           (const bf16_t*)k, (const bf16_t*)v, row_pos, (bf16_t*)out, lse_out,
                           cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, scale);
    else
        hipLaunchKernelGGL((packed_simple_kernel<float>), grid, dim3(64), 0, st, (const float*)q,
                           (const float*)k, (const float*)v, row_pos, (float*)out, lse_out,
                           cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, scale);
    return launch_status();
}

}  // namespace pkv
