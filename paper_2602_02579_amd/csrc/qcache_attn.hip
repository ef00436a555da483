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
// Split.  The keys of a sequence come in groups of kGroup, a step of a workgroup.  One sequence: workgroup j
// of a kv head takes groups j, j + n_wg, ..: the first one's bytes are on their way before the
// sequence's length is known.  Several: their groups make one line that the workgroups share evenly,
// whatever the lengths; a workgroup's piece may begin and end inside sequences.  What several
// workgroups hold parts of goes to the workspace, and a second launch joins it.
#include <algorithm>

#include "qcache.h"

namespace pkv {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kGroup = kWaves * 32;   // keys of a workgroup's step
constexpr int kJoinWaves = 8;

struct QAttnParams {
    const void* q;                // [m, hq, D]
    const unsigned char *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t* row_pos;       // [m]
    const int32_t* seq_start;     // [n_seq] or nullptr
    void* out;                    // [m, hq, D]
    float* lse;                   // [m, hq] or nullptr
    float* part_o;                // [n_wg (+ n_seq), hkv, cols, D], not normalised, and
    float2* part_ml;              // their (reference * c2, sum)
    int2* held_by;                // [n_seq] first and last workgroup of a sequence; several only
    int rows, each, n_seq, hq, hkv, group, cols, D;   // cols = each * group
    int n_wg, log2_wg;            // workgroups of a kv head and column tile, a power of two
    float c2;                     // softmax scale * log2(e)
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The cache rows of a sequence from `start` on; row_end: the first one that a row does not see
__device__ __forceinline__ int seq_start(const QAttnParams& p, int s) {
    return p.seq_start ? min(max(p.seq_start[s], 0), p.rows) : 0;
}
__device__ __forceinline__ int row_end(const QAttnParams& p, int start, int row) {
    const int64_t e = (int64_t)start + p.row_pos[row] + 1;
    return max(start, (int)min(e, (int64_t)p.rows));
}
__device__ __forceinline__ int seq_end(const QAttnParams& p, int start, int s) {
    int end = start;
    for (int r = 0; r < p.each; ++r) end = max(end, row_end(p, start, s * p.each + r));
    return end;
}
// groups are counted from the 32 rows that hold the first one
__device__ __forceinline__ int groups_of(int start, int end) {
    return end > start ? (end - (start & ~31) + kGroup - 1) / kGroup : 0;
}
__device__ __forceinline__ int lane_groups(const QAttnParams& p, int s) {
    if (s >= p.n_seq) return 0;
    const int start = seq_start(p, s);
    return groups_of(start, seq_end(p, start, s));
}
__device__ __forceinline__ int wave_scan(int v) {   // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    return v;
}

// Several sequences: a workgroup's piece of the line of groups, and the sequence that it begins in.
struct Piece {
    int64_t begin, end, before;   // before: groups in front of sequence s
    int s;
};
__device__ __forceinline__ Piece piece_of(const QAttnParams& p, int j) {
    const int lane = threadIdx.x & 63;
    Piece w = {0, 0, 0, 0};
    int64_t total = 0;
    int incl = 0, mine = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        mine = lane_groups(p, s0 + lane);
        incl = wave_scan(mine);
        total += uniform(__shfl(incl, 63));
    }
    // few groups: one each
    w.begin = total < p.n_wg ? j : (j * total) >> p.log2_wg;
    w.end = total < p.n_wg ? min(total, (int64_t)j + 1) : ((j + 1) * total) >> p.log2_wg;
    if (w.begin >= w.end) return w;
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        if (p.n_seq > 64) {
            mine = lane_groups(p, s0 + lane);
            incl = wave_scan(mine);
        }
        const uint64_t past = __ballot(w.before + incl > w.begin);
        if (past) {
            const int at = __builtin_ctzll(past);
            w.s = s0 + at;
            w.before += uniform(__shfl(incl - mine, at));
            return w;
        }
        w.before += uniform(__shfl(incl, 63));
    }
    w.end = w.begin;   // not reached: the group is on the line
    return w;
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
    uint32_t ks[2][NB * 2];   // their scale bytes: of steps 2 i and 2 i + 1
    uint32_t vc[NB][8];       // codes of 8 elements of 8 keys
    u32x2 vs[NB];             // the 8 keys' scale bytes
};

// Byte `at` of w as a scale: the conversions look at the exponent bits alone, and 255 there is NaN.
__device__ __forceinline__ float scale_at(uint32_t w, int at) {
    return __uint_as_float(at < 3 ? w << (23 - 8 * at) : w >> 1);
}
__device__ __forceinline__ uint32_t byte_at(u32x2 w, int at) {
    return (w[at >> 2] >> (at & 3) * 8) & 255u;
}

template <typename T, int NB, int NC, bool WIDE>
__global__ __launch_bounds__(kWaves * 64) void qcache_attn_kernel(QAttnParams p) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int F = NB * 4;                      // contraction steps of a score
    __shared__ f32x4 s_o[kWaves / 2][NC * NB * 8][64];
    __shared__ float s_m[kWaves][NC * 16], s_l[kWaves][NC * 16];

    const int lane = threadIdx.x & 63;
    const int wave = uniform(threadIdx.x >> 6);
    const int g4 = lane >> 4, l16 = lane & 15;
    const int h = blockIdx.y, tile0 = blockIdx.z * (NC * 16);
    const int D = WIDE ? NB * 128 : p.D;
    const int code_row = D / 2, scale_row = D / kQBlock;

    // ---- where a lane's pieces of 32 keys lie ------------------------------------------------
    const int krow = 8 * (l16 >> 2) + (l16 & 3);
    const uint32_t k_off = (uint32_t)(krow * code_row + g4 * (WIDE ? 16 : 4));
    const uint32_t ks_off = (uint32_t)(krow * scale_row + (WIDE ? 2 * g4 : g4 >> 1));
    const uint32_t v_off = (uint32_t)(8 * g4 * code_row + 4 * l16);
    const uint32_t vs_off = (uint32_t)((g4 * scale_row + (l16 >> 1)) * 8);
    auto load = [&](int r0, Tile<NB>& t) {          // r0: a multiple of 32 below rows
        const int64_t row = (int64_t)h * p.rows + r0;
        const unsigned char* const kc = p.k_codes + row * code_row;
        const unsigned char* const ks = p.k_scales + row * scale_row;
        const unsigned char* const vc = p.v_codes + row * code_row;
        const unsigned char* const vs = p.v_scales + row * scale_row;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            if (WIDE) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const u32x4 c = *reinterpret_cast<const u32x4*>(kc + kt * 4 * code_row + nb * 64 + k_off);
#pragma unroll
                    for (int f = 0; f < 4; ++f) t.kc[kt][nb * 4 + f] = c[f];
                    t.ks[kt][nb * 2] =
                        *reinterpret_cast<const uint16_t*>(ks + kt * 4 * scale_row + nb * 8 + ks_off);
                }
            } else {
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const bool in = 32 * f + 8 * g4 < D;
                    t.kc[kt][f] = in ? *reinterpret_cast<const uint32_t*>(kc + kt * 4 * code_row + 16 * f + k_off) : 0u;
                    const uint32_t b = in ? ks[kt * 4 * scale_row + 2 * f + ks_off] : 127u;
                    if (f & 1) t.ks[kt][f >> 1] |= b << 8;
                    else t.ks[kt][f >> 1] = b;
                }
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const bool in = WIDE || 128 * nb + 8 * l16 < D;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                t.vc[nb][j] = in ? *reinterpret_cast<const uint32_t*>(vc + j * code_row + nb * 64 + v_off) : 0u;
            t.vs[nb] = in ? *reinterpret_cast<const u32x2*>(vs + nb * 64 + vs_off)
                          : u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
        }
    };

    // ---- the workgroup's groups ----------------------------------------------------------------
    const bool single = p.n_seq == 1;
    Piece piece = {0, 0, 0, 0};
    if (!single) {
        piece = piece_of(p, blockIdx.x);
        if (piece.begin >= piece.end) return;
    }
    for (;;) {
        const int s = piece.s, start = uniform(seq_start(p, s)), base = (start & ~31) + wave * 32;
        int g = single ? (int)blockIdx.x : (int)(piece.begin - piece.before);
        const int g_step = single ? p.n_wg : 1;
        Tile<NB> cur, next;
        const int r_first = base + g * kGroup;
        if (r_first < p.rows) load(r_first, cur);   // whether a row sees it turns out behind the loads

        // ---- this lane's columns ---------------------------------------------------------------
        int end[NC], end_min = 0x7fffffff, end_max = start;
        bf16x8 qf[NC][PARTS][F];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = tile0 + c * 16 + l16;
            const bool valid = col < p.cols;
            const int in_seq = valid ? col / p.group : 0;
            const int row = s * p.each + in_seq;
            const int head = h * p.group + (valid ? col - in_seq * p.group : 0);
            const T* q = static_cast<const T*>(p.q) + ((int64_t)row * p.hq + head) * D;
            end[c] = valid ? row_end(p, start, row) : start;
            end_max = max(end_max, end[c]);
            if (valid) end_min = min(end_min, end[c]);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int d = WIDE ? (f >> 2) * 128 + 32 * g4 + 8 * (f & 3) : 32 * f + 8 * g4;
                typedef typename Vec16<T>::type vec_t;
                vec_t v[8 / Vec16<T>::N] = {};
                if (valid && (WIDE || d < D))
#pragma unroll
                    for (int i = 0; i < 8 / Vec16<T>::N; ++i)
                        v[i] = reinterpret_cast<const vec_t*>(q + d)[i];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const T x = v[e / Vec16<T>::N][e % Vec16<T>::N];
                    if constexpr (PARTS == 1) {
                        qf[c][0][f][e] = x;
                    } else {
                        bf16_t part[PARTS];
                        split<PARTS>(x, part);
#pragma unroll
                        for (int i = 0; i < PARTS; ++i) qf[c][i][f][e] = part[i];
                    }
                }
            }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            end_min = min(end_min, __shfl_xor(end_min, o));
            end_max = max(end_max, __shfl_xor(end_max, o));
        }
        end_min = uniform(end_min);
        end_max = uniform(end_max);
        // all rows of the sequence have a say in the line's groups, this tile's in the single one's
        const int groups = single ? groups_of(start, end_max)
                                  : groups_of(start, uniform(seq_end(p, start, s)));
        const int g_end = single ? groups : (int)min((int64_t)groups, piece.end - piece.before);
        if (single && g > 0 && g >= groups) return;
        const bool whole = !single && g == 0 && g_end == groups;
        if (!single && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) {
            if (g == 0) p.held_by[s].x = blockIdx.x;
            if (g_end == groups) p.held_by[s].y = blockIdx.x;
        }

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

        // ---- the wave's steps, the next one's bytes on their way -----------------------------
        for (; g < g_end && base + g * kGroup < end_max; g += g_step) {
            const int r0 = base + g * kGroup, r1 = r0 + g_step * kGroup;
            if (g + g_step < g_end && r1 < end_max) load(r1, next);
            // keys in front of the sequence or behind what some column sees
            const bool edge = r0 < start || r0 + 32 > end_min;
            const int key0 = r0 + 8 * g4;      // of this lane's 8 scores and values
            f32x4 sc[NC][2];
#pragma unroll
            for (int c = 0; c < NC; ++c) sc[c][0] = sc[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const float scale = WIDE ? scale_at(cur.ks[kt][(f >> 2) * 2], (f & 3) >> 1)
                                             : scale_at(cur.ks[kt][f >> 1], f & 1);
                    u32x4 w;
#pragma unroll
                    for (int b = 0; b < 4; ++b) w[b] = cvt2(cur.kc[kt][f], scale, b);
                    const bf16x8 a = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int i = PARTS - 1; i >= 0; --i) sc[c][kt] = mfma16(a, qf[c][i][f], sc[c][kt]);
                }
            if (edge) {
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (key0 + j < start || key0 + j >= end[c]) sc[c][j >> 2][j & 3] = -INFINITY;
                // what no column sees may be any bytes; its weight is 0, and its scales become 1
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (key0 + j < start || key0 + j >= end_max)
                            cur.vs[nb][j >> 2] = (cur.vs[nb][j >> 2] & ~(255u << (j & 3) * 8)) |
                                                 127u << (j & 3) * 8;
            }
            bf16x8 pb[NC][PARTS];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, sc[c][j >> 2][j & 3]);
                top *= p.c2;
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
                    const float e = __builtin_amdgcn_exp2f(fmaf(sc[c][j >> 2][j & 3], p.c2, -ref));
                    bf16_t part[PARTS];
                    split<PARTS>(e, part);
                    l[c] += e;
#pragma unroll
                    for (int i = 0; i < PARTS; ++i) pb[c][i][j] = part[i];
                }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                u32x2 vs = cur.vs[nb];
                // scale bytes that stand for NaN: their keys count with another scale, and NaN goes into the
                // columns that see them by a product of its own (0 times NaN would reach the others)
                const u32x2 nan = ((vs & 0x7f7f7f7fu) + 0x01010101u) & vs & 0x80808080u;
                if (__any((nan[0] | nan[1]) != 0)) {
                    bf16x8 is_nan;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const bool n = byte_at(vs, j) == kQScaleNan;
                        is_nan[j] = (bf16_t)(n ? 1.f : 0.f);
                        if (n) vs[j >> 2] ^= 128u << (j & 3) * 8;
                    }
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        bf16x8 seen;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            seen[j] = (bf16_t)(key0 + j >= start && key0 + j < end[c] ? 1.f : 0.f);
                        const f32x4 n = mfma16(is_nan, seen, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (n[r] > 0.f)
#pragma unroll
                                for (int f = 0; f < 8; ++f) o[c][nb][f][r] = __builtin_nanf("");
                    }
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    u32x4 lo, hi;
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const uint32_t x0 = cvt2(cur.vc[nb][j], scale_at(vs[j >> 2], j & 3), b);
                        const uint32_t x1 = cvt2(cur.vc[nb][j + 1], scale_at(vs[j >> 2], (j & 3) + 1), b);
                        lo[j / 2] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
                        hi[j / 2] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
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
            cur = next;
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
                const int in_seq = col / p.group;
                const int64_t oc = (int64_t)(s * p.each + in_seq) * p.hq + h * p.group +
                                   (col - in_seq * p.group);
                // all of the row's keys are here
                const bool direct = single ? p.n_wg == 1 || groups_of(start, end[c]) <= 1 : whole;
                if (direct && single && blockIdx.x) continue;
                const int64_t part =
                    ((int64_t)(single ? blockIdx.x : blockIdx.x + s) * p.hkv + h) * p.cols + col;
                const float inv = l_all[c] == 0.f ? 0.f : 1.f / l_all[c];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int d = nb * 128 + 8 * (4 * g4 + r);
                        if (!WIDE && d >= D) continue;
                        if (direct) {
                            T* op = static_cast<T*>(p.out) + oc * D + d;
#pragma unroll
                            for (int e = 0; e < 8; e += Vec16<T>::N) {
                                typename Vec16<T>::type v;
#pragma unroll
                                for (int i = 0; i < Vec16<T>::N; ++i)
                                    v[i] = Elem<T>::from_f32(o[c][nb][e + i][r] * inv);
                                *reinterpret_cast<typename Vec16<T>::type*>(op + e) = v;
                            }
                        } else {
                            float* op = p.part_o + part * D + d;
#pragma unroll
                            for (int e = 0; e < 8; e += 4)
                                *reinterpret_cast<f32x4*>(op + e) =
                                    f32x4{o[c][nb][e][r], o[c][nb][e + 1][r], o[c][nb][e + 2][r],
                                          o[c][nb][e + 3][r]};
                        }
                    }
                if (g4 == 0) {
                    if (!direct) p.part_ml[part] = make_float2(m_all[c], l_all[c]);
                    else if (p.lse)
                        p.lse[oc] = l_all[c] == 0.f ? -INFINITY
                                                    : (m_all[c] + __builtin_amdgcn_logf(l_all[c])) *
                                                          0.69314718055994531f;
                }
            }
        }
        if (single) return;
        piece.begin = piece.before + g_end;
        if (piece.begin >= piece.end) return;
        piece.before += groups;
        do ++piece.s;                       // a group is left: one of them holds it
        while (piece.s < p.n_seq && uniform(lane_groups(p, piece.s)) == 0);
        if (piece.s >= p.n_seq) return;
    }
}

// A row and head of which several workgroups hold parts: eight waves share the parts and meet; rows
// of sequences without keys, which nobody took, are written here too.
template <typename T>
__global__ __launch_bounds__(kJoinWaves * 64) void qcache_attn_join_kernel(QAttnParams p) {
    __shared__ float s_o[kJoinWaves][256];
    __shared__ float2 s_ml[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t oc = blockIdx.x;
    const int row = (int)(oc / p.hq), head = (int)(oc % p.hq);
    const int s = row / p.each;
    T* out = static_cast<T*>(p.out) + oc * p.D;
    const int start = uniform(seq_start(p, s));
    int j0 = 0, j1, slot0 = 0;
    if (p.n_seq == 1) {
        j1 = min(p.n_wg, groups_of(start, uniform(row_end(p, start, row)))) - 1;
    } else {
        if (seq_end(p, start, s) == start) {
            if ((int)threadIdx.x < p.D) out[threadIdx.x] = Elem<T>::from_f32(0.f);
            if (threadIdx.x == 0 && p.lse) p.lse[oc] = -INFINITY;
            return;
        }
        const int2 by = p.held_by[s];
        j0 = uniform(by.x);
        j1 = uniform(by.y);
        slot0 = s;
    }
    if (j1 <= j0) return;                 // written by the workgroup that held it all
    const int h = head / p.group, col = (row - s * p.each) * p.group + head % p.group;
    const int64_t slot_rows = (int64_t)p.hkv * p.cols;
    const int64_t first = (int64_t)slot0 * slot_rows + (int64_t)h * p.cols + col;
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f, m = -INFINITY;
    for (int j = j0 + wave; j <= j1; j += 8 * kJoinWaves) {
        float2 ml[8];
        float x[8][4];
#pragma unroll
        for (int u = 0; u < 8; ++u) {          // eight parts at once
            const bool in = j + u * kJoinWaves <= j1;
            const int64_t at = first + (in ? j + u * kJoinWaves : j) * slot_rows;
            ml[u] = p.part_ml[at];
            if (!in) ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[u][i] = lane + 64 * i < p.D ? p.part_o[at * p.D + lane + 64 * i] : 0.f;
        }
        float mn = m;
#pragma unroll
        for (int u = 0; u < 8; ++u) mn = fmaxf(mn, ml[u].x);
        const float ref = mn == -INFINITY ? 0.f : mn, corr = __builtin_amdgcn_exp2f(m - ref);
        m = mn;
        l *= corr;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= corr;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float w = __builtin_amdgcn_exp2f(ml[u].x - ref);
            l += ml[u].y * w;
            if (j + u * kJoinWaves <= j1)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] += x[u][i] * w;
        }
    }
    if (lane == 0) s_ml[wave] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[wave][lane + 64 * i] = acc[i];
    __syncthreads();
    const int d = threadIdx.x;
    if (d >= p.D) return;
    float top = -INFINITY, sum = 0.f, a = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) top = fmaxf(top, s_ml[w].x);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_ml[w].x - ref);
        sum += s_ml[w].y * f;
        a += s_o[w][d] * f;
    }
    out[d] = Elem<T>::from_f32(sum == 0.f ? 0.f : a / sum);
    if (d == 0 && p.lse)
        p.lse[oc] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

template <typename T, int NB, int NC>
void launch_main(const QAttnParams& p, bool wide, dim3 grid, hipStream_t st) {
    if (wide)
        hipLaunchKernelGGL((qcache_attn_kernel<T, NB, NC, true>), grid, dim3(kWaves * 64), 0, st, p);
    else
        hipLaunchKernelGGL((qcache_attn_kernel<T, NB, NC, false>), grid, dim3(kWaves * 64), 0, st, p);
}

struct QPlan {
    int nb, nc, log2_wg;
    int64_t tiles;
    size_t parts;
};

QPlan plan(const pkv_layer_cfg& cfg, int64_t rows, int64_t m, int64_t n_seq) {
    QPlan pl;
    const int64_t cols = m / n_seq * (cfg.n_q_heads / cfg.n_kv_heads);
    pl.nb = cfg.head_dim > 128 ? 2 : 1;
    // columns of a workgroup: as many as there are, up to what the registers hold
    const int most = (cfg.dtype == PKV_F32 ? 2 : 4) / pl.nb;
    pl.nc = cols <= 16 || most == 1 ? 1 : cols <= 32 || most == 2 ? 2 : 4;
    pl.tiles = ceil_div(cols, 16 * pl.nc);
    // about two workgroups per CU, and no more than there can be groups
    const int64_t want = std::min(512 / std::max<int64_t>(1, cfg.n_kv_heads * pl.tiles),
                                  (ceil_div(rows, kGroup) + 1) * n_seq);
    pl.log2_wg = 0;
    while ((2 << pl.log2_wg) <= want) ++pl.log2_wg;
    pl.parts = (size_t)((1 << pl.log2_wg) + (n_seq > 1 ? n_seq : 0)) * cfg.n_kv_heads * cols;
    return pl;
}

}  // namespace

size_t qcache_attn_ws_bytes(const pkv_layer_cfg& cfg, int64_t rows, int64_t m, int64_t n_seq) {
    return plan(cfg, rows, m, n_seq).parts * (cfg.head_dim + 2) * sizeof(float) +
           (n_seq > 1 ? n_seq * sizeof(int2) : 0);
}

pkv_status launch_qcache_attn(const pkv_layer_cfg& cfg, const void* q, const pkv_qcache& cache,
                              const int32_t* row_pos, const int32_t* seq_start, void* out,
                              float* lse_out, int64_t m, int64_t n_seq, float scale, void* ws,
                              hipStream_t st) {
    const QPlan pl = plan(cfg, cache.rows, m, n_seq);
    // a workgroup per row and head joins: a launch holds less than 2^32 threads
    if (m * cfg.n_q_heads >= 1 << 23 || pl.tiles > 65535) return PKV_ERR_UNSUPPORTED;
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
    p.held_by = reinterpret_cast<int2*>(p.part_ml + pl.parts);
    p.rows = (int)cache.rows;
    p.each = (int)(m / n_seq);
    p.n_seq = (int)n_seq;
    p.hq = cfg.n_q_heads;
    p.hkv = cfg.n_kv_heads;
    p.group = p.hq / p.hkv;
    p.cols = p.each * p.group;
    p.D = cfg.head_dim;
    p.n_wg = 1 << pl.log2_wg;
    p.log2_wg = pl.log2_wg;
    p.c2 = scale * 1.4426950408889634f;
    const bool bf16 = cfg.dtype == PKV_BF16, wide = cfg.head_dim == 128 * pl.nb;
    const dim3 grid((unsigned)p.n_wg, (unsigned)cfg.n_kv_heads, (unsigned)pl.tiles);
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
    if (n_seq == 1 && p.n_wg == 1) return PKV_OK;
    const dim3 rows_heads((unsigned)(m * cfg.n_q_heads));
    if (bf16)
        hipLaunchKernelGGL((qcache_attn_join_kernel<bf16_t>), rows_heads, dim3(kJoinWaves * 64), 0, st, p);
    else
        hipLaunchKernelGGL((qcache_attn_join_kernel<float>), rows_heads, dim3(kJoinWaves * 64), 0, st, p);
    return launch_status();
}

}  // namespace pkv
