// Attention of a decoding step's rows over a cache held in 4 bits (qcache.h: the format).
//
//     S^T = K Q^T,   O^T += V^T P^T     (v_mfma_f32_16x16x32_bf16)
//
// 16 columns (row, head of the group) share the keys of a kv head.  A wave takes 32 keys at a time,
// straight from global memory into registers and from there, converted, into the matrix
// instructions: both layouts are such that no lane needs what another one loaded.
//   Keys: lane (g4, l16) holds 32 consecutive elements of key 8 (l16 / 4) + l16 % 4 (+ 4 for the
//     second half), 16 bytes; contraction index 8 g4 + e of step f is element 32 g4 + 8 f + e, on
//     both sides.  Row 4 a + i of half kt being key 8 a + 4 kt + i, a lane ends with the scores of keys
//     8 g4 .. 8 g4 + 7 of its column: the B operand of the second product as they are.
//   Values: lane (g4, l16) holds elements 8 l16 .. + 7 of keys 8 g4 .. + 7; row i of output block f
//     is element 8 i + f.  A conversion gives two elements of one key, the operand wants two keys of
//     one element: a byte permutation per pair.  The scales of a lane's 8 keys are 8 adjacent bytes.
// Every value of the format is exact in bf16.  fp32: queries and weights go in as three bf16 parts
// (24 bits), so the products are as exact as fp32 ones.
//
// What bounds it: reading the cache, 4.5 bits an element.
//
// The reference of a column's exponentials follows the running maximum only when that is 2^8 or more
// above it: few steps rescale, and the lanes of a column need not meet every step.
//
// Split.  The keys of all sequences, in groups of NW * 32, are one line that the workgroups of a kv head
// share evenly, whatever the lengths; a workgroup's piece may begin and end inside sequences.
// Pieces of a sequence that several workgroups hold go to the workspace, and a second launch joins them.
#include <algorithm>

#include "qcache.h"

namespace pkv {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kGroup = kWaves * 32;   // keys of a workgroup's step

struct QAttnParams {
    const void* q;                // [m, hq, D]
    const unsigned char *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t* row_pos;       // [m]
    const int32_t* seq_start;     // [n_seq] or nullptr
    void* out;                    // [m, hq, D]
    float* lse;                   // [m, hq] or nullptr
    float* part_o;                // [n_wg + n_seq, hkv, cols, D], not normalised, and
    float2* part_ml;              // their (reference * c2, sum)
    int rows, each, n_seq, hq, hkv, group, cols, D;   // cols = each * group
    int n_wg;                     // workgroups of a kv head and column tile
    float c2;                     // softmax scale * log2(e)
};

__device__ __forceinline__ int wave_sum_i32(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Cache rows start .. end - 1 are what the rows of a sequence see, together; groups: of keys, counted
// from `start` rounded down to 32
struct Seq {
    int start, end;
    __device__ __forceinline__ int base() const { return start & ~31; }
    __device__ __forceinline__ int groups() const {
        return end > start ? (end - base() + kGroup - 1) / kGroup : 0;
    }
};
__device__ __forceinline__ int row_end(const QAttnParams& p, int start, int row) {
    const int64_t e = (int64_t)start + p.row_pos[row] + 1;
    return (int)min(e, (int64_t)p.rows);
}
__device__ __forceinline__ Seq seq_of(const QAttnParams& p, int s) {
    Seq q;
    q.start = p.seq_start ? min(max(p.seq_start[s], 0), p.rows) : 0;
    q.end = q.start;
    for (int r = 0; r < p.each; ++r) q.end = max(q.end, row_end(p, q.start, s * p.each + r));
    return q;
}

// The line of groups: how many there are, and where a group or a sequence lies.
struct Line {
    int64_t total;
    int n_wg;   // workgroups that have a piece
    __device__ __forceinline__ int64_t begin(int j) const { return j * total / n_wg; }
    __device__ __forceinline__ int wg_of(int64_t group) const {
        return (int)(((group + 1) * n_wg - 1) / total);
    }
};
__device__ __forceinline__ Line line_of(const QAttnParams& p) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += 64)
        total += wave_sum_i32(s0 + lane < p.n_seq ? seq_of(p, s0 + lane).groups() : 0);
    return {total, (int)min((int64_t)p.n_wg, total)};
}
// sum of the groups in front of sequence s; or, with find >= 0, the sequence that holds that group
__device__ __forceinline__ int64_t groups_before(const QAttnParams& p, int64_t find, int* s) {
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        const int mine = s0 + lane < p.n_seq ? seq_of(p, s0 + lane).groups() : 0;
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        const bool hit = find >= 0 ? before + incl > find : s0 + lane >= *s;
        const uint64_t hits = __ballot(hit);
        if (hits) {
            const int at = __builtin_ctzll(hits);
            *s = s0 + at;
            return before + __shfl(incl - mine, at);
        }
        before += __shfl(incl, 63);
    }
    return before;
}

__device__ __forceinline__ uint32_t cvt2(uint32_t codes, float scale, int byte) {
    switch (byte) {
        case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
        case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
        case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
        default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    }
}
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// x as the sum of PARTS bf16 numbers, the leading one first
template <int PARTS>
__device__ __forceinline__ void split(float x, bf16_t* part) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        part[i] = (bf16_t)x;
        x -= (float)part[i];
    }
}

// What a lane holds of 32 keys.  WIDE: head_dim is NB * 128, and a lane's piece of a key is contiguous;
// otherwise step f takes elements 32 f + 8 g4 .. of a key, nothing beyond head_dim.
template <int NB>
struct Tile {
    uint32_t kc[2][NB * 4];   // codes of a key's steps
    uint32_t ks[2][NB * 2];   // their scale bytes: of steps 2 i and 2 i + 1 (WIDE: one each half word)
    uint32_t vc[NB][8];       // codes of 8 elements of 8 keys
    u32x2 vs[NB];             // the 8 keys' scale bytes
};

template <typename T, int NB, int NC, bool WIDE>
__global__ __launch_bounds__(kWaves * 64) void qcache_attn_kernel(QAttnParams p) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int F = NB * 4;                      // contraction steps of a score
    __shared__ f32x4 s_o[kWaves / 2][NC * NB * 8][64];
    __shared__ float s_m[kWaves][NC * 16], s_l[kWaves][NC * 16];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g4 = lane >> 4, l16 = lane & 15;
    const int h = blockIdx.y, tile0 = blockIdx.z * (NC * 16);

    const Line line = line_of(p);
    if ((int)blockIdx.x >= line.n_wg) return;
    int64_t at = line.begin(blockIdx.x);
    const int64_t piece_end = line.begin(blockIdx.x + 1);
    int s = 0;
    int64_t before = groups_before(p, at, &s);

    const int code_row = p.D / 2, scale_row = p.D / kQBlock;
    const int krow = 8 * (l16 >> 2) + (l16 & 3);
    uint32_t k_off[2], ks_off[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        k_off[kt] = (uint32_t)((krow + 4 * kt) * code_row + g4 * (WIDE ? 16 : 4));
        ks_off[kt] = (uint32_t)((krow + 4 * kt) * scale_row + (WIDE ? 2 * g4 : g4 >> 1));
    }
    const uint32_t v_off = (uint32_t)(8 * g4 * code_row + 4 * l16);
    const uint32_t vs_off = (uint32_t)((g4 * scale_row + (l16 >> 1)) * 8);

    auto load = [&](int r0, Tile<NB>& t) {          // r0: a multiple of 32, r0 + 32 <= rows
        const int64_t row = (int64_t)h * p.rows + r0;
        const unsigned char* kc = p.k_codes + row * code_row;
        const unsigned char* ks = p.k_scales + row * scale_row;
        const unsigned char* vc = p.v_codes + row * code_row;
        const unsigned char* vs = p.v_scales + row * scale_row;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            if (WIDE) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const u32x4 c = *reinterpret_cast<const u32x4*>(kc + k_off[kt] + nb * 64);
#pragma unroll
                    for (int f = 0; f < 4; ++f) t.kc[kt][nb * 4 + f] = c[f];
                    t.ks[kt][nb * 2] = *reinterpret_cast<const uint16_t*>(ks + ks_off[kt] + nb * 8);
                }
            } else {
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const bool in = 32 * f + 8 * g4 < p.D;
                    t.kc[kt][f] =
                        in ? *reinterpret_cast<const uint32_t*>(kc + k_off[kt] + 16 * f) : 0u;
                    const uint32_t b = in ? ks[ks_off[kt] + 2 * f] : 127u;
                    if (f & 1) t.ks[kt][f >> 1] |= b << 8;
                    else t.ks[kt][f >> 1] = b;
                }
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const bool in = WIDE || 128 * nb + 8 * l16 < p.D;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                t.vc[nb][j] = in ? *reinterpret_cast<const uint32_t*>(vc + v_off + j * code_row +
                                                                      nb * 64)
                                 : 0u;
            t.vs[nb] = in ? *reinterpret_cast<const u32x2*>(vs + vs_off + nb * 64)
                          : u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
        }
    };

    while (at < piece_end) {
        const Seq seq = seq_of(p, s);
        const int groups = seq.groups();
        const int g0 = (int)(at - before);
        const int g1 = (int)min((int64_t)groups, piece_end - before);
        const bool whole = g0 == 0 && g1 == groups;

        // ---- this lane's columns -----------------------------------------------------------
        int end[NC], end_min = 0x7fffffff;   // first cache row that the column does not see
        bf16x8 qf[NC][PARTS][F];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = tile0 + c * 16 + l16;
            const bool valid = col < p.cols;
            const int row = s * p.each + (valid ? col / p.group : 0);
            const int head = h * p.group + (valid ? col % p.group : 0);
            end[c] = valid ? max(row_end(p, seq.start, row), seq.start) : seq.start;
            if (valid) end_min = min(end_min, end[c]);
            const T* q = static_cast<const T*>(p.q) + ((int64_t)row * p.hq + head) * p.D;
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int d = WIDE ? (f >> 2) * 128 + 32 * g4 + 8 * (f & 3) : 32 * f + 8 * g4;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; e += Vec16<T>::N) {
                    typename Vec16<T>::type v = {};
                    if (valid && (WIDE || d < p.D))
                        v = *reinterpret_cast<const typename Vec16<T>::type*>(q + d + e);
#pragma unroll
                    for (int i = 0; i < Vec16<T>::N; ++i) x[e + i] = Elem<T>::to_f32(v[i]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bf16_t part[PARTS];
                    split<PARTS>(x[e], part);
#pragma unroll
                    for (int i = 0; i < PARTS; ++i) qf[c][i][f][e] = part[i];
                }
            }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) end_min = min(end_min, __shfl_xor(end_min, o));
        end_min = __builtin_amdgcn_readfirstlane(end_min);

        float m2[NC], l[NC];
        f32x4 o[NC][NB][8];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            m2[c] = -INFINITY;
            l[c] = 0.f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int f = 0; f < 8; ++f) o[c][nb][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        auto use = [&](int r0, Tile<NB>& t) {
            // keys in front of the sequence or behind what some column sees
            const bool edge = r0 < seq.start || r0 + 32 > end_min;
            const int key0 = r0 + 8 * g4;      // of this lane's 8 scores and values
            f32x4 sc[NC][2];
#pragma unroll
            for (int c = 0; c < NC; ++c) sc[c][0] = sc[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const uint32_t two = t.ks[kt][WIDE ? (f >> 2) * 2 : f >> 1];
                    const uint32_t byte = (WIDE ? (f & 3) >> 1 : f & 1) ? two >> 8 : two & 255u;
                    const float scale = q_scale(byte);
                    u32x4 w;
#pragma unroll
                    for (int b = 0; b < 4; ++b) w[b] = cvt2(t.kc[kt][f], scale, b);
                    const bf16x8 a = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int i = PARTS - 1; i >= 0; --i) sc[c][kt] = mfma16(a, qf[c][i][f], sc[c][kt]);
                }
            bf16x8 pb[NC][PARTS];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                float x[8], top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = sc[c][j >> 2][j & 3] * p.c2;
                    if (edge && (key0 + j < seq.start || key0 + j >= end[c])) x[j] = -INFINITY;
                    top = fmaxf(top, x[j]);
                }
                if (__any(top > m2[c] + 8.f)) {
                    float m = fmaxf(top, m2[c]);
                    m = fmaxf(m, __shfl_xor(m, 16));
                    m = fmaxf(m, __shfl_xor(m, 32));
                    const float corr = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m2[c] - m);
                    m2[c] = m;
                    l[c] *= corr;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int f = 0; f < 8; ++f) o[c][nb][f] *= corr;
                }
                const float ref = m2[c] == -INFINITY ? 0.f : m2[c];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float e = __builtin_amdgcn_exp2f(x[j] - ref);
                    bf16_t part[PARTS];
                    split<PARTS>(e, part);
                    l[c] += e;
#pragma unroll
                    for (int i = 0; i < PARTS; ++i) pb[c][i][j] = part[i];
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                u32x2 vs = t.vs[nb];
                if (edge) {        // what nobody sees may be anything; its weight is 0
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (key0 + j < seq.start || key0 + j >= seq.end)
                            vs[j >> 2] = (vs[j >> 2] & ~(255u << (j & 3) * 8)) | 127u << (j & 3) * 8;
                }
                // scale bytes that stand for NaN: their keys count as 0, and go into the columns that
                // see them by a product of their own (weights of 0 keep them out of the others)
                const uint32_t nan = (((vs[0] & 0x7f7f7f7fu) + 0x01010101u) & vs[0] & 0x80808080u) |
                                     (((vs[1] & 0x7f7f7f7fu) + 0x01010101u) & vs[1] & 0x80808080u);
                if (__any(nan != 0)) {
                    bf16x8 is_nan;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const bool n = ((vs[j >> 2] >> (j & 3) * 8) & 255u) == kQScaleNan;
                        is_nan[j] = (bf16_t)(n ? 1.f : 0.f);
                        if (n) vs[j >> 2] ^= 128u << (j & 3) * 8;
                    }
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        bf16x8 seen;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            seen[j] = (bf16_t)(key0 + j >= seq.start && key0 + j < end[c] ? 1.f : 0.f);
                        const f32x4 n = mfma16(is_nan, seen, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (n[r] > 0.f)
#pragma unroll
                                for (int f = 0; f < 8; ++f) o[c][nb][f][r] = __builtin_nanf("");
                    }
                }
                float scale[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    scale[j] = __uint_as_float(((vs[j >> 2] >> (j & 3) * 8) & 255u) << 23);
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    u32x4 lo, hi;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t x0 = cvt2(t.vc[nb][2 * j], scale[2 * j], b);
                        const uint32_t x1 = cvt2(t.vc[nb][2 * j + 1], scale[2 * j + 1], b);
                        lo[j] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
                        hi[j] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
                    }
                    const bf16x8 a0 = __builtin_bit_cast(bf16x8, lo), a1 = __builtin_bit_cast(bf16x8, hi);
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int i = PARTS - 1; i >= 0; --i) {
                            o[c][nb][2 * b] = mfma16(a0, pb[c][i], o[c][nb][2 * b]);
                            o[c][nb][2 * b + 1] = mfma16(a1, pb[c][i], o[c][nb][2 * b + 1]);
                        }
                }
            }
        };

        // ---- the wave's steps, the next one's bytes on their way -----------------------------
        {
            const int base = seq.base() + wave * 32;
            int g = g0;
            Tile<NB> cur, next;
            bool more = g < g1 && base + g * kGroup < seq.end;
            if (more) load(base + g * kGroup, cur);
            while (more) {
                const int r0 = base + g * kGroup;
                ++g;
                more = g < g1 && r0 + kGroup < seq.end;
                if (more) load(r0 + kGroup, next);
                use(r0, cur);
                cur = next;
            }
        }

        // ---- the waves meet, always in the same order -----------------------------------------
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            l[c] += __shfl_xor(l[c], 16);
            l[c] += __shfl_xor(l[c], 32);
        }
        __syncthreads();     // the previous sequence's exchange has been read
        if (g4 == 0)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                s_m[wave][c * 16 + l16] = m2[c];
                s_l[wave][c * 16 + l16] = l[c];
            }
        __syncthreads();
        float m_all[NC], l_all[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_m[w][c * 16 + l16]);
            m_all[c] = m;
            l_all[c] = 0.f;
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                l_all[c] += s_l[w][c * 16 + l16] * __builtin_amdgcn_exp2f(s_m[w][c * 16 + l16] - ref);
            const float mine = __builtin_amdgcn_exp2f(m2[c] - ref);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int f = 0; f < 8; ++f) o[c][nb][f] *= mine;
        }
#pragma unroll
        for (int half = kWaves / 2; half > 0; half >>= 1) {
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int f = 0; f < 8; ++f)
                            s_o[wave - half][(c * NB + nb) * 8 + f][lane] = o[c][nb][f];
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int f = 0; f < 8; ++f)
                            o[c][nb][f] += s_o[wave][(c * NB + nb) * 8 + f][lane];
            if (half > 1) __syncthreads();
        }
        if (wave == 0) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = tile0 + c * 16 + l16;
                if (col >= p.cols) continue;
                const int64_t row = (int64_t)s * p.each + col / p.group;
                const int64_t oc = row * p.hq + h * p.group + col % p.group;
                const int64_t part =
                    ((int64_t)(blockIdx.x + s) * p.hkv + h) * p.cols + col;
                const float inv = l_all[c] > 0.f ? 1.f / l_all[c] : l_all[c] == 0.f ? 0.f : l_all[c];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int d = nb * 128 + 8 * (4 * g4 + r);
                        if (!WIDE && d >= p.D) continue;
                        if (whole) {
                            T* op = static_cast<T*>(p.out) + oc * p.D + d;
#pragma unroll
                            for (int e = 0; e < 8; e += Vec16<T>::N) {
                                typename Vec16<T>::type v;
#pragma unroll
                                for (int i = 0; i < Vec16<T>::N; ++i)
                                    v[i] = Elem<T>::from_f32(o[c][nb][e + i][r] * inv);
                                *reinterpret_cast<typename Vec16<T>::type*>(op + e) = v;
                            }
                        } else {
                            float* op = p.part_o + part * p.D + d;
#pragma unroll
                            for (int e = 0; e < 8; e += 4)
                                *reinterpret_cast<f32x4*>(op + e) =
                                    f32x4{o[c][nb][e][r], o[c][nb][e + 1][r], o[c][nb][e + 2][r],
                                          o[c][nb][e + 3][r]};
                        }
                    }
                if (g4 == 0) {
                    if (!whole) p.part_ml[part] = make_float2(m_all[c], l_all[c]);
                    else if (p.lse)
                        p.lse[oc] = l_all[c] == 0.f ? -INFINITY
                                                    : (m_all[c] + __builtin_amdgcn_logf(l_all[c])) *
                                                          0.69314718055994531f;
                }
            }
        }
        at = before + g1;
        before += groups;
        ++s;
        while (at < piece_end && seq_of(p, s).groups() == 0) ++s;   // a group is left: it ends
    }
}

// A row and head whose sequence several workgroups hold: their parts, joined by four waves; rows of
// sequences without keys are written here too.
template <typename T>
__global__ __launch_bounds__(256) void qcache_attn_join_kernel(QAttnParams p) {
    __shared__ float s_o[4][256], s_l[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t oc = blockIdx.x;
    const int row = (int)(oc / p.hq), head = (int)(oc % p.hq);
    int s = row / p.each;
    T* out = static_cast<T*>(p.out) + oc * p.D;
    const int groups = seq_of(p, s).groups();
    if (groups == 0) {
        if ((int)threadIdx.x < p.D) out[threadIdx.x] = Elem<T>::from_f32(0.f);
        if (threadIdx.x == 0 && p.lse) p.lse[oc] = -INFINITY;
        return;
    }
    const Line line = line_of(p);
    const int64_t before = groups_before(p, -1, &s);
    const int j0 = line.wg_of(before), j1 = line.wg_of(before + groups - 1);
    if (j0 == j1) return;                 // written by the workgroup that held it all
    const int h = head / p.group, col = (row - s * p.each) * p.group + head % p.group;
    auto part = [&](int j) { return ((int64_t)(j + s) * p.hkv + h) * p.cols + col; };
    float m = -INFINITY;
    for (int j = j0 + lane; j <= j1; j += 64) m = fmaxf(m, p.part_ml[part(j)].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float ref = m == -INFINITY ? 0.f : m;
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
#pragma unroll 4
    for (int j = j0 + wave; j <= j1; j += 4) {
        const float2 ml = p.part_ml[part(j)];
        const float w = __builtin_amdgcn_exp2f(ml.x - ref);
        l += ml.y * w;
        const float* po = p.part_o + part(j) * p.D;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < p.D) acc[i] += po[lane + 64 * i] * w;
    }
    if (lane == 0) s_l[wave] = l;
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[wave][lane + 64 * i] = acc[i];
    __syncthreads();
    l = (s_l[0] + s_l[1]) + (s_l[2] + s_l[3]);
    const int d = threadIdx.x;
    if (d < p.D) {
        const float a = (s_o[0][d] + s_o[1][d]) + (s_o[2][d] + s_o[3][d]);
        out[d] = Elem<T>::from_f32(l == 0.f ? 0.f : a / l);
    }
    if (d == 0 && p.lse)
        p.lse[oc] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

template <typename T, int NB, int NC>
void launch_main(const QAttnParams& p, bool wide, dim3 grid, hipStream_t st) {
    if (wide)
        hipLaunchKernelGGL((qcache_attn_kernel<T, NB, NC, true>), grid, dim3(kWaves * 64), 0, st, p);
    else
        hipLaunchKernelGGL((qcache_attn_kernel<T, NB, NC, false>), grid, dim3(kWaves * 64), 0, st, p);
}

struct QPlan {
    int nb, nc, tiles, n_wg;
    size_t parts;
};

QPlan plan(const pkv_layer_cfg& cfg, int64_t rows, int64_t m, int64_t n_seq) {
    QPlan pl;
    const int64_t cols = m / n_seq * (cfg.n_q_heads / cfg.n_kv_heads);
    pl.nb = cfg.head_dim > 128 ? 2 : 1;
    // columns of a workgroup: as many as there are, up to what the registers hold
    const int most = (cfg.dtype == PKV_F32 ? 2 : 4) / pl.nb;
    pl.nc = cols <= 16 || most == 1 ? 1 : cols <= 32 || most == 2 ? 2 : 4;
    pl.tiles = (int)ceil_div(cols, 16 * pl.nc);
    // two workgroups per CU
    const int64_t want = ceil_div(512, (int64_t)cfg.n_kv_heads * pl.tiles);
    const int64_t groups = ceil_div(rows, kGroup) * n_seq;   // no more than that
    pl.n_wg = (int)std::max<int64_t>(1, std::min(want, groups));
    pl.parts = (size_t)(pl.n_wg + n_seq) * cfg.n_kv_heads * cols;
    return pl;
}

}  // namespace

size_t qcache_attn_ws_bytes(const pkv_layer_cfg& cfg, int64_t rows, int64_t m, int64_t n_seq) {
    return plan(cfg, rows, m, n_seq).parts * (cfg.head_dim + 2) * sizeof(float);
}

pkv_status launch_qcache_attn(const pkv_layer_cfg& cfg, const void* q, const pkv_qcache& cache,
                              const int32_t* row_pos, const int32_t* seq_start, void* out,
                              float* lse_out, int64_t m, int64_t n_seq, float scale, void* ws,
                              hipStream_t st) {
    const QPlan pl = plan(cfg, cache.rows, m, n_seq);
    // a workgroup per row and head joins: a launch holds less than 2^32 threads
    if (m * cfg.n_q_heads >= 1 << 24 || pl.tiles > 65535) return PKV_ERR_UNSUPPORTED;
    QAttnParams p = {};
    p.q = q;
    p.k_codes = static_cast<const unsigned char*>(cache.k_codes);
    p.k_scales = static_cast<const unsigned char*>(cache.k_scales);
    p.v_codes = static_cast<const unsigned char*>(cache.v_codes);
    p.v_scales = static_cast<const unsigned char*>(cache.v_scales);
    p.row_pos = row_pos;
    p.seq_start = seq_start;
    p.out = out;
    p.lse = lse_out;
    p.part_o = static_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float2*>(p.part_o + pl.parts * cfg.head_dim);
    p.rows = (int)cache.rows;
    p.each = (int)(m / n_seq);
    p.n_seq = (int)n_seq;
    p.hq = cfg.n_q_heads;
    p.hkv = cfg.n_kv_heads;
    p.group = p.hq / p.hkv;
    p.cols = p.each * p.group;
    p.D = cfg.head_dim;
    p.n_wg = pl.n_wg;
    p.c2 = scale * 1.4426950408889634f;
    const bool bf16 = cfg.dtype == PKV_BF16, wide = cfg.head_dim == 128 * pl.nb;
    const dim3 grid((unsigned)pl.n_wg, (unsigned)cfg.n_kv_heads, (unsigned)pl.tiles);
    if (bf16 && pl.nb == 1) {
        if (pl.nc == 1) launch_main<bf16_t, 1, 1>(p, wide, grid, st);
        else if (pl.nc == 2) launch_main<bf16_t, 1, 2>(p, wide, grid, st);
        else launch_main<bf16_t, 1, 4>(p, wide, grid, st);
    } else if (bf16) {
        if (pl.nc == 1) launch_main<bf16_t, 2, 1>(p, wide, grid, st);
        else launch_main<bf16_t, 2, 2>(p, wide, grid, st);
    } else if (pl.nb == 1) {
        if (pl.nc == 1) launch_main<float, 1, 1>(p, wide, grid, st);
        else launch_main<float, 1, 2>(p, wide, grid, st);
    } else {
        launch_main<float, 2, 1>(p, wide, grid, st);
    }
    if (launch_status() != PKV_OK) return PKV_ERR_LAUNCH;
    const dim3 rows_heads((unsigned)(m * cfg.n_q_heads));
    if (bf16)
        hipLaunchKernelGGL((qcache_attn_join_kernel<bf16_t>), rows_heads, dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((qcache_attn_join_kernel<float>), rows_heads, dim3(256), 0, st, p);
    return launch_status();
}

}  // namespace pkv
