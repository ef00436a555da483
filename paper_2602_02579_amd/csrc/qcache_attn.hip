// Attention of a decoding step's rows over a cache held in 4 bits (qcache.h: the format).
//
//     S^T = K Q^T,   O^T += V^T P^T     (v_mfma_f32_16x16x32_bf16)
//
// 16 columns (row, head of the group) share the keys of a kv head.  A wave takes 32 keys at a time,
// straight from global memory into registers and from there, converted, into the matrix
// instructions: both layouts are such that no lane needs what another one loaded (head_dim 128):
//   Keys: lane (g4, l16) holds 32 consecutive elements of key 8 (l16 / 4) + l16 % 4 (+ 4 for the
//     second half), 16 bytes; contraction index 8 g4 + e of step f is element 32 g4 + 8 f + e, on
//     both sides.  Row 4 a + i of half kt being key 8 a + 4 kt + i, a lane ends with the scores of keys
//     8 g4 .. 8 g4 + 7 of its column: the B operand of the second product as they are.
//   Values: lane (g4, l16) holds elements 8 l16 .. + 7 of keys 8 g4 .. + 7; row i of output block f
//     is element 8 i + f.  A conversion gives two elements of one key, the operand wants two keys of
//     one element: a byte permutation per pair.  The scales of a lane's 8 keys are 8 adjacent bytes.
// Every value of the format is exact in bf16.  fp32: queries and weights go in as three bf16 parts
// (24 bits), so the products are as exact as fp32 ones.  bf16: the weights are rounded to bf16, the type of the
// product's operands (their sum is of the unrounded ones): error against 64 bits 0.0023 of the results' norm,
// with fp32 weights 0.0017.
//
// What bounds it: reading the cache, 4.5 bits an element.  One row over 131328 keys of 8 heads of 128, 151 MB,
// 28.3 us, 5.3 TB/s; over 32896 10.2 us, of which the bytes are 7.4 at a large copy's rate; 16 sequences of 0 to
// 12033 rows, 65 MB, 16.4 us (12.8).  The requests leave 1.1 us after a workgroup's start (several sequences:
// 2.2), the first bytes are there after 4, and the waves meet for 0.6.  32 keys are some 139 vector
// instructions, of which 64 convert codes and 32 bring two keys of an element together; without the
// latter the batch would take 0.6 us less.
//
// Other head sizes than 64, 128 and 256 load their pieces of keys one by one, and fp32 above 128 does not fit the
// registers (up to 327 of them go through memory).  One row over 32768 keys of 8 heads of 128, 256, 240 and 144:
// 12.2, 19.7, 31.2 and 28.4 us, fp32 14.3, 29.7, 44.3 and 41.9; 12 sequences of 7584 to 16384 rows 30.6, 53.4, 95
// and 88, fp32 35.0, 95, 158 and 146.
//
// The reference of a column's exponentials follows the running maximum only when that is 2^8 or more
// above it: few steps rescale, and the lanes of a column need not meet every step.  Behind the first
// scale of 2^65 or more a wave keeps it 2^40 higher still: 2^31 weights of up to 2^8 then sum to no more than
// the largest value, where they would leave the range before they are divided by their sum.
//
// Split.  The keys of a sequence come in groups of kGroup, a step of a workgroup.  One sequence: workgroup j
// of a kv head takes groups j, j + n_wg, ..: the first one's bytes are on their way before the
// sequence's length is known.  Several: their groups make one line that the workgroups share evenly,
// whatever the lengths; a workgroup's piece may begin and end inside sequences.  What several
// workgroups hold parts of goes to the workspace, and a second launch joins it (2.6 to 4 us).
#include <algorithm>
#include <atomic>

#include "lane_ops.h"
#include "qcache.h"

namespace pkv {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 8;
constexpr int kGroup = kWaves * 32;   // keys of a workgroup's step
constexpr float kLn2 = 0.69314718055994531f;

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

// The cache rows of a sequence from seq_start on; row_end: the first one that a row does not see
__device__ __forceinline__ int seq_start(const QAttnParams& p, int s) {
    return p.seq_start ? min(max(p.seq_start[s], 0), p.rows) : 0;
}
__device__ __forceinline__ int end_of(const QAttnParams& p, int start, int pos) {
    const int64_t e = (int64_t)start + pos + 1;
    return max(start, (int)min(e, (int64_t)p.rows));
}
__device__ __forceinline__ int row_end(const QAttnParams& p, int start, int row) {
    return end_of(p, start, p.row_pos[row]);
}
// groups are counted from the 32 rows that hold the first one
__device__ __forceinline__ int groups_of(int start, int end) {
    return end > start ? (end - (start & ~31) + kGroup - 1) / kGroup : 0;
}
// A sequence's first row and the groups that its rows see together
struct Seq {
    int start, groups;
};
__device__ __forceinline__ Seq seq_of(const QAttnParams& p, int s) {
    const int32_t* const row_pos = p.row_pos + (int64_t)s * p.each;
    const int start = seq_start(p, s);
    int pos = row_pos[0];
    for (int r = 1; r < p.each; r += 4)       // four at once
#pragma unroll
        for (int i = 0; i < 4; ++i) pos = max(pos, row_pos[min(r + i, p.each - 1)]);
    return {start, groups_of(start, end_of(p, start, pos))};
}
// Several sequences: a workgroup's piece of the line of groups, and the sequence that it is in.  To begin
// a sequence takes a workgroup as long as kBegin groups (its queries and first keys come, its waves have to
// meet), and so long is a sequence's place on the line: even pieces take even times.  Without it 16
// sequences of 0 to 12033 rows take 23.1 us in place of 20.2, 4 of 3333 to 16001 with 4 rows each 20.1 in
// place of 18.1; two of 20000 15.6 and 16.6.
constexpr int kBegin = 3;
struct Piece {
    int64_t begin, end, before;   // before: of the line, in front of the groups of sequence s
    int s, extra;                 // extra: what the line has in front of a sequence
    Seq seq;                      // of sequence s
    Seq of_lane;                  // up to 64 sequences: of the one of the lane's number
};
__device__ __forceinline__ Seq lane_seq(const QAttnParams& p, int s) {
    return s < p.n_seq ? seq_of(p, s) : Seq{0, 0};
}
__device__ __forceinline__ Piece piece_of(const QAttnParams& p, int j) {
    const int lane = threadIdx.x & 63;
    Piece w = {};
    int64_t total = 0;
    int incl = 0, some = 0;       // some: sequences that have groups
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        w.of_lane = lane_seq(p, s0 + lane);
        incl = wave_scan(w.of_lane.groups);
        total += last_lane(incl);
        some += __popcll(__ballot(w.of_lane.groups > 0));
    }
    // few groups: one each
    const bool few = total < p.n_wg;
    w.extra = few ? 0 : kBegin;
    total += (int64_t)some * w.extra;
    w.begin = few ? j : (j * total) >> p.log2_wg;
    w.end = few ? min(total, (int64_t)j + 1) : ((j + 1) * total) >> p.log2_wg;
    if (w.begin >= w.end) return w;
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        if (p.n_seq > 64) w.of_lane = lane_seq(p, s0 + lane);
        incl = wave_scan(w.of_lane.groups + (w.of_lane.groups > 0 ? w.extra : 0));
        const uint64_t past = __ballot(w.before + incl > w.begin);
        if (past) {
            const int at = __builtin_ctzll(past);
            w.s = s0 + at;
            w.seq.start = __builtin_amdgcn_readlane(w.of_lane.start, at);
            w.seq.groups = __builtin_amdgcn_readlane(w.of_lane.groups, at);
            w.before += __builtin_amdgcn_readlane(incl, at) - w.seq.groups;
            return w;
        }
        w.before += last_lane(incl);
    }
    w.end = w.begin;   // not reached: the place is on the line
    return w;
}
// The next sequence that has groups; false: there is none
__device__ __forceinline__ bool next_sequence(const QAttnParams& p, Piece& w) {
    w.before += w.seq.groups + w.extra;
    while (++w.s < p.n_seq) {
        if (p.n_seq <= 64) {
            w.seq.start = __builtin_amdgcn_readlane(w.of_lane.start, w.s);
            w.seq.groups = __builtin_amdgcn_readlane(w.of_lane.groups, w.s);
        } else {
            const Seq q = seq_of(p, w.s);
            w.seq.start = uniform(q.start);
            w.seq.groups = uniform(q.groups);
        }
        if (w.seq.groups) return true;
    }
    return false;
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

// What a lane holds of 32 keys: KE = DP / 4 elements of each of two, VE = DP / 16 of each of eight.
template <int DP>
struct Tile {
    uint32_t kc[2][DP / 32];                 // codes of a key's contraction steps
    uint32_t ks[2][DP < 256 ? 1 : 2];        // their scale bytes
    uint32_t vc[8][DP < 256 ? 1 : 2];        // codes of a value's elements
    u32x2 vs;                                // the 8 values' scale bytes
};

// Byte `at` of w as a scale: the conversions look at the exponent bits alone, and 255 there is NaN.
__device__ __forceinline__ float scale_at(uint32_t w, int at) {
    return __uint_as_float(at < 3 ? w << (23 - 8 * at) : w >> 1);
}
__device__ __forceinline__ uint32_t byte_at(u32x2 w, int at) {
    return (w[at >> 2] >> (at & 3) * 8) & 255u;
}

// A tensor from a uniform address on, for loads with a lane's offset in one register
__device__ __forceinline__ __amdgpu_buffer_rsrc_t from(const unsigned char* ptr) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(ptr), 0, 0x7fffffff,
                                             0x00027000);
}

// DP: 64, 128 or 256, at least head_dim.  EXACT: head_dim is DP, and a lane's piece of a key is contiguous;
// otherwise step f takes elements 32 f + 8 g4 .. of a key.  Pieces beyond head_dim are read from its
// beginning: the queries are 0 there, and nobody asks for those outputs.
template <typename T, int DP, bool EXACT, int NC, bool MULTI>
__global__ __launch_bounds__(kWaves * 64) void qcache_attn_kernel(QAttnParams p) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int F = DP / 32;                     // contraction steps of a score
    constexpr int VB = DP / 16;                    // output blocks: row i of block f is element VB i + f
    constexpr bool TWO_AHEAD = DP * NC <= 128;     // where the registers hold three tiles
    constexpr bool NEXT_AHEAD = DP * PARTS < 768;  // and two tiles and queries beside the results
    constexpr int kORow = DP + 4;                  // floats of a column's output in LDS
    extern __shared__ __align__(16) float s_o[];   // [kWaves][16][kORow]
    __shared__ float2 s_ml[kWaves][16];

    const int lane = threadIdx.x & 63;
    const int wave = uniform(threadIdx.x >> 6);
    const int g4 = lane >> 4, l16 = lane & 15;
    const int h = blockIdx.y, tile0 = blockIdx.z * (NC * 16);
    const int D = EXACT ? DP : p.D;
    const int code_row = D / 2, scale_row = D / kQBlock;

    // ---- where a lane's pieces of 32 keys lie ------------------------------------------------
    const int krow = 8 * (l16 >> 2) + (l16 & 3);
    int k_off[EXACT ? 1 : F], ks_off[EXACT ? 1 : F];
#pragma unroll
    for (int f = 0; f < (EXACT ? 1 : F); ++f) {
        const int d = EXACT ? g4 * (DP / 4) : 32 * f + 8 * g4 < D ? 32 * f + 8 * g4 : 0;
        k_off[f] = krow * code_row + d / 2;
        ks_off[f] = krow * scale_row + (EXACT ? d / kQBlock & ~3 : d / kQBlock);
    }
    // Scales come by whole words: what makes a number of fewer bits whole would move in front of the
    // loop's end and wait for the load there.
    const int ks_shift = EXACT ? (g4 * (DP / 4) / kQBlock & 3) * 8 : 0;
    const int vd = EXACT || l16 * VB < D ? l16 * VB : 0;
    const int v_off = 8 * g4 * code_row + (vd / 2 & ~3);
    const int v_shift = DP == 64 ? (vd / 2 & 3) * 8 : 0;
    const int vs_off = (g4 * scale_row + vd / kQBlock) * 8;
    auto load = [&](int r0, Tile<DP>& t) __attribute__((always_inline)) {
        const int64_t row = (int64_t)h * p.rows + r0;   // r0: a multiple of 32 below rows
        const auto kc = from(p.k_codes + row * code_row), ks = from(p.k_scales + row * scale_row);
        const auto vc = from(p.v_codes + row * code_row), vs = from(p.v_scales + row * scale_row);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int c0 = kt * 4 * code_row, s0 = kt * 4 * scale_row;
            if constexpr (!EXACT) {
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    t.kc[kt][f] = __builtin_amdgcn_raw_buffer_load_b32(kc, k_off[f], c0, 0);
                    const uint32_t b = __builtin_amdgcn_raw_buffer_load_b8(ks, ks_off[f], s0, 0);
                    t.ks[kt][f >> 2] = f & 3 ? t.ks[kt][f >> 2] | b << 8 * (f & 3) : b;
                }
            } else if constexpr (DP == 64) {
                const auto c = __builtin_amdgcn_raw_buffer_load_b64(kc, k_off[0], c0, 0);
                t.kc[kt][0] = c[0];
                t.kc[kt][1] = c[1];
                t.ks[kt][0] = __builtin_amdgcn_raw_buffer_load_b32(ks, ks_off[0], s0, 0);
            } else {
#pragma unroll
                for (int x = 0; x < F; x += 4) {
                    const auto c = __builtin_amdgcn_raw_buffer_load_b128(kc, k_off[0], c0 + 4 * x, 0);
#pragma unroll
                    for (int f = 0; f < 4; ++f) t.kc[kt][x + f] = c[f];
                }
                t.ks[kt][0] = __builtin_amdgcn_raw_buffer_load_b32(ks, ks_off[0], s0, 0);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (DP <= 128) {
                t.vc[j][0] = __builtin_amdgcn_raw_buffer_load_b32(vc, v_off, j * code_row, 0);
            } else {
                const auto c = __builtin_amdgcn_raw_buffer_load_b64(vc, v_off, j * code_row, 0);
                t.vc[j][0] = c[0];
                t.vc[j][1] = c[1];
            }
        }
        const auto c = __builtin_amdgcn_raw_buffer_load_b64(vs, vs_off, 0, 0);
        t.vs = u32x2{c[0], c[1]};
    };

    // ---- the workgroup's groups ----------------------------------------------------------------
    Piece piece = {};
    if constexpr (MULTI) {
        piece = piece_of(p, blockIdx.x);
        if (piece.begin >= piece.end) return;
    }
    auto first_group = [&]() __attribute__((always_inline)) {
        return MULTI ? (int)max(piece.begin - piece.before, (int64_t)0) : (int)blockIdx.x;
    };
    if (MULTI && piece.before + first_group() >= piece.end) return;   // it ends in front of the groups
    // Requests in the order of use: the first tile, the queries, the second tile (whether a row sees them
    // turns out behind the requests).
    typedef typename Vec16<T>::type vec_t;
    constexpr int QV = 8 / Vec16<T>::N;
    const int step = (MULTI ? 1 : p.n_wg) * kGroup;
    int s, start, r0, row0, down[NC];   // row0: the tile's first row; a lane's rows as seen from there
    Tile<DP> t0, t1, t2;
    vec_t q_in[NC][F][QV];
    auto request = [&]() __attribute__((always_inline)) {
        s = piece.s;
        start = MULTI ? piece.seq.start : uniform(seq_start(p, 0));
        r0 = (start & ~31) + wave * 32 + first_group() * kGroup;
        load(min(r0, p.rows - 32), t0);
        row0 = p.each == 1 ? s : s * p.each + tile0 / p.group;
        const T* const q0 = static_cast<const T*>(p.q) + ((int64_t)row0 * p.hq + h * p.group) * D;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            // this lane's columns (the last one again behind it)
            const int col = min(tile0 + c * 16 + l16, p.cols - 1);
            const int in_seq = p.each == 1 ? 0 : col / p.group;
            down[c] = s * p.each + in_seq - row0;
            const int q_at = down[c] * p.hq + col - in_seq * p.group;
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int d = EXACT ? g4 * (DP / 4) + 8 * f : 32 * f + 8 * g4;
                const vec_t* q = reinterpret_cast<const vec_t*>(q0 + (uint32_t)(q_at * D + d));
#pragma unroll
                for (int i = 0; i < QV; ++i) q_in[c][f][i] = EXACT || d < D ? q[i] : vec_t{};
            }
        }
        load(min(r0 + step, p.rows - 32), t1);
    };
    request();
    for (;;) {
        const int g = first_group();
        int end[NC], end_min, end_max;
        if (p.each == 1) {
            end_min = end_max = uniform(row_end(p, start, s));
#pragma unroll
            for (int c = 0; c < NC; ++c) end[c] = end_max;
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                end[c] = row_end(p, start, row0 + down[c]);
                end_min = c ? min(end_min, end[c]) : end[c];
                end_max = c ? max(end_max, end[c]) : end[c];
            }
            end_min = uniform(min16(end_min));
            end_max = uniform(max16(end_max));
        }
        bf16x8 qf[NC][PARTS][F];
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bf16_t part[PARTS];
                    if constexpr (PARTS == 1) part[0] = q_in[c][f][0][e];
                    else split<PARTS>(q_in[c][f][e / 4][e % 4], part);
#pragma unroll
                    for (int i = 0; i < PARTS; ++i) qf[c][i][f][e] = part[i];
                }
        // all rows of the sequence have a say in the line's groups, this tile's in the single one's
        const int groups = MULTI ? piece.seq.groups : groups_of(start, end_max);
        const int g_end = MULTI ? (int)min((int64_t)groups, piece.end - piece.before) : groups;
        if (!MULTI && g > 0 && g >= groups) return;
        const bool whole = MULTI ? g == 0 && g_end == groups : p.n_wg == 1;
        const int r_end = min(end_max, (start & ~31) + g_end * kGroup);

        float m2[NC], l[NC], above = 0.f;      // above: by how much the reference is kept over the maximum
        f32x4 o[NC][VB];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            m2[c] = -INFINITY;
            l[c] = 0.f;
#pragma unroll
            for (int f = 0; f < VB; ++f) o[c][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        auto use = [&](int r0, Tile<DP>& cur) __attribute__((always_inline)) {
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
                    const float scale = EXACT ? scale_at(cur.ks[kt][0] >> ks_shift, f >> 1)
                                              : scale_at(cur.ks[kt][f >> 2], f & 3);
                    u32x4 w;
#pragma unroll
                    for (int b = 0; b < 4; ++b) w[b] = cvt2(cur.kc[kt][f], scale, b);
                    const bf16x8 a = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int i = PARTS - 1; i >= 0; --i) sc[c][kt] = mfma16(a, qf[c][i][f], sc[c][kt]);
                }
            if (__builtin_expect(edge, 0)) {
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const uint32_t seen = bits_between(start - key0, end[c] - key0);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        sc[c][j >> 2][j & 3] = where_bit(seen, j, sc[c][j >> 2][j & 3]);
                }
                // what no column sees may be any bytes; its weight is 0, and its scales become 1
                const uint32_t some = bits_between(start - key0, end_max - key0);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t off = ~(uint32_t)__builtin_amdgcn_sbfe((int)some, j, 1) &
                                         255u << (j & 3) * 8;
                    cur.vs[j >> 2] = (cur.vs[j >> 2] & ~off) | (off & 0x7f7f7f7fu);
                }
            }
            bf16x8 pb[NC][PARTS];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, sc[c][j >> 2][j & 3]);
                top = fmaf(top, p.c2, above);
                if (__builtin_expect(__any(top > m2[c] + 8.f), 0)) {
                    float m = fmaxf(top, m2[c]);
                    m = fmaxf(m, __shfl_xor(m, 16));
                    m = fmaxf(m, __shfl_xor(m, 32));
                    const float corr = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m2[c] - m);
                    m2[c] = m;
                    l[c] *= corr;
#pragma unroll
                    for (int f = 0; f < VB; ++f) o[c][f] *= corr;
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
            // Scale bytes from 192 on: large values, for which the reference rises, and 255, which stands for NaN:
            // those keys count with another scale, and NaN goes into the columns that see them by a
            // product of its own (0 times NaN would reach the others).
            u32x2 vs = cur.vs;
            const u32x2 large = vs & (vs << 1) & 0x80808080u;
            if (__builtin_expect(__any((large[0] | large[1]) != 0), 0)) {
                if (above == 0.f) {
                    above = 40.f;
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        m2[c] += above;
                        l[c] *= 0x1p-40f;
#pragma unroll
                        for (int f = 0; f < VB; ++f) o[c][f] *= 0x1p-40f;
#pragma unroll
                        for (int i = 0; i < PARTS; ++i)
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                pb[c][i][j] = (bf16_t)((float)pb[c][i][j] * 0x1p-40f);
                    }
                }
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
                            for (int f = 0; f < VB; ++f) o[c][f][r] = __builtin_nanf("");
                }
            }
#pragma unroll
            for (int f = 0; f < VB; f += 2) {       // a conversion gives elements f and f + 1
                u32x4 lo, hi;
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint32_t x0 = cvt2(cur.vc[j][f >> 3] >> v_shift, scale_at(vs[j >> 2], j & 3),
                                             (f & 7) / 2);
                    const uint32_t x1 = cvt2(cur.vc[j + 1][f >> 3] >> v_shift,
                                             scale_at(vs[j >> 2], (j & 3) + 1), (f & 7) / 2);
                    lo[j / 2] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
                    hi[j / 2] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
                }
                const bf16x8 a0 = __builtin_bit_cast(bf16x8, lo), a1 = __builtin_bit_cast(bf16x8, hi);
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int i = PARTS - 1; i >= 0; --i) {
                        o[c][f] = mfma16(a0, pb[c][i], o[c][f]);
                        o[c][f + 1] = mfma16(a1, pb[c][i], o[c][f + 1]);
                    }
            }
        };

        // ---- the wave's steps, one or two more on their way -----------------------------------------
        // Behind the last one the loads go on, to rows that are there already: a load that may or may not
        // have been made would have to be waited for as if it were the one in question.  So would one
        // that some way through the loop leaves out: the loop has a single end.
        auto load_ahead = [&](Tile<DP>& t) __attribute__((always_inline)) {
            const int ahead = r0 + 2 * step;
            load(ahead < r_end ? ahead : r0, t);
        };
        if constexpr (TWO_AHEAD) {
            while (r0 + 2 * step < r_end) {
                load_ahead(t2);
                use(r0, t0);
                r0 += step;
                load_ahead(t0);
                use(r0, t1);
                r0 += step;
                load_ahead(t1);
                use(r0, t2);
                r0 += step;
            }
        } else {
            while (r0 + step < r_end) {
                use(r0, t0);
                load_ahead(t0);
                r0 += step;
                use(r0, t1);
                load_ahead(t1);
                r0 += step;
            }
        }
        if (r0 < r_end) use(r0, t0);
        if (TWO_AHEAD && r0 + step < r_end) use(r0 + step, t1);

        // the next sequence is on its way while the waves meet
        const int s_now = s;
        bool more = false;
        if constexpr (MULTI) {
            if (blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) {
                if (g == 0) p.held_by[s].x = blockIdx.x;
                if (g_end == groups) p.held_by[s].y = blockIdx.x;
            }
            piece.begin = piece.before + g_end;
            more = piece.begin < piece.end && next_sequence(p, piece) && piece.before < piece.end;
            if (more && NEXT_AHEAD) request();
        }

        // ---- the waves meet: 16 columns at a time through LDS, a wave per column, always in the same order
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int left = p.cols - tile0 - c * 16;
            if (left <= 0) break;
            l[c] += __shfl_xor(l[c], 16);
            l[c] += __shfl_xor(l[c], 32);
            if (MULTI || c) __syncthreads();     // the previous exchange has been read
            if (l16 < left) {
                // element VB (4 g4 + r) + f of the column
                float* const so = s_o + (wave * 16 + l16) * kORow + 4 * VB * g4;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int f = 0; f < VB; f += 4)
                        *reinterpret_cast<f32x4*>(so + VB * r + f) =
                            f32x4{o[c][f][r], o[c][f + 1][r], o[c][f + 2][r], o[c][f + 3][r]};
                if (g4 == 0) s_ml[wave][l16] = make_float2(m2[c], l[c]);
            }
            __syncthreads();
            for (int x = wave; x < min(left, 16); x += kWaves) {
                float m = -INFINITY, sum = 0.f, factor[kWaves];
#pragma unroll
                for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_ml[w][x].x);
                const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    factor[w] = __builtin_amdgcn_exp2f(s_ml[w][x].x - ref);
                    sum += s_ml[w][x].y * factor[w];
                }
                const int col = tile0 + c * 16 + x;
                f32x2 a[DP > 128 ? 2 : 1];
#pragma unroll
                for (int i = 0; i < (DP > 128 ? 2 : 1); ++i) {
                    a[i] = f32x2{0.f, 0.f};
                    const int d = DP < 128 ? 2 * (lane & 31) : 2 * lane + 128 * i;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) {
                        const f32x2 v = *reinterpret_cast<const f32x2*>(s_o + (w * 16 + x) * kORow + d);
                        a[i][0] += v[0] * factor[w];
                        a[i][1] += v[1] * factor[w];
                    }
                }
                if (whole) {
                    const int in_seq = p.each == 1 ? 0 : col / p.group;
                    const int64_t oc = (int64_t)(s_now * p.each + in_seq) * p.hq + h * p.group +
                                       (col - in_seq * p.group);
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                    for (int i = 0; i < (DP > 128 ? 2 : 1); ++i) {
                        const int d = 2 * lane + 128 * i;
                        if (d >= D) break;
                        typedef T pair_t __attribute__((ext_vector_type(2)));
                        *reinterpret_cast<pair_t*>(static_cast<T*>(p.out) + oc * D + d) =
                            pair_t{Elem<T>::from_f32(a[i][0] * inv), Elem<T>::from_f32(a[i][1] * inv)};
                    }
                    if (lane == 0 && p.lse)
                        p.lse[oc] = sum == 0.f ? -INFINITY
                                               : (m + __builtin_amdgcn_logf(sum)) * kLn2;
                } else {
                    const int64_t part =
                        ((int64_t)(MULTI ? blockIdx.x + s_now : blockIdx.x) * p.hkv + h) * p.cols + col;
#pragma unroll
                    for (int i = 0; i < (DP > 128 ? 2 : 1); ++i) {
                        const int d = 2 * lane + 128 * i;
                        if (d < D) *reinterpret_cast<f32x2*>(p.part_o + part * D + d) = a[i];
                    }
                    if (lane == 0) p.part_ml[part] = make_float2(m, sum);
                }
            }
        }
        if (!more) return;
        if (!NEXT_AHEAD) request();
    }
}

// A row and head of which several workgroups hold parts: the waves share the parts and meet; rows of
// sequences without keys, which nobody took, are written here too.
template <typename T, int kJoinWaves>
__global__ __launch_bounds__(kJoinWaves * 64) void qcache_attn_join_kernel(QAttnParams p) {
    __shared__ float s_o[kJoinWaves][256];
    __shared__ float2 s_ml[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t oc = blockIdx.x;
    const int row = (int)(oc / p.hq), head = (int)(oc % p.hq);
    const int s = row / p.each;
    T* out = static_cast<T*>(p.out) + oc * p.D;
    const bool single = p.n_seq == 1;
    const int h = head / p.group, col = (row - s * p.each) * p.group + head % p.group;
    const int64_t slot_rows = (int64_t)p.hkv * p.cols;
    const int64_t first = (int64_t)(single ? 0 : s) * slot_rows + (int64_t)h * p.cols + col;
    int2 by = {0, p.n_wg - 1};            // one sequence: the parts are requested before it is known
    if (!single) {                        // how many there are
        by = p.held_by[s];
        if (seq_of(p, s).groups == 0) {
            if ((int)threadIdx.x < p.D) out[threadIdx.x] = Elem<T>::from_f32(0.f);
            if (threadIdx.x == 0 && p.lse) p.lse[oc] = -INFINITY;
            return;
        }
        if (by.y <= by.x) return;         // written by the workgroup that held it all
    }
    const int j0 = uniform(by.x), j_most = uniform(by.y);
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f, m = -INFINITY;
    int j1 = j_most;
    for (int j = j0 + wave; j <= j1; j += 4 * kJoinWaves) {
        float2 ml[4];
        float x[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {          // four parts at once
            const int64_t at = first + min(j + u * kJoinWaves, j_most) * slot_rows;
            ml[u] = p.part_ml[at];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[u][i] = lane + 64 * i < p.D ? p.part_o[at * p.D + lane + 64 * i] : 0.f;
        }
        if (single) {                          // the first workgroup has a part even where there is no key
            const int start = seq_start(p, 0);
            j1 = min(j_most, max(0, uniform(groups_of(start, row_end(p, start, row))) - 1));
        }
        float mn = m;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (j + u * kJoinWaves > j1) ml[u] = make_float2(-INFINITY, 0.f);
            mn = fmaxf(mn, ml[u].x);
        }
        const float ref = mn == -INFINITY ? 0.f : mn, corr = __builtin_amdgcn_exp2f(m - ref);
        m = mn;
        l *= corr;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= corr;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float w = __builtin_amdgcn_exp2f(ml[u].x - ref);
            l += ml[u].y * w;
            if (j + u * kJoinWaves <= j1)      // what is behind them was never written
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
        p.lse[oc] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <typename T, int DP, bool EXACT, int NC, bool MULTI>
pkv_status launch_kernel(const QAttnParams& p, dim3 grid, hipStream_t st) {
    constexpr int kBytes = kWaves * 16 * (DP + 4) * sizeof(float);
    auto* const kernel = &qcache_attn_kernel<T, DP, EXACT, NC, MULTI>;
    static std::atomic<bool> configured{false};   // set twice at worst: the calls are idempotent
    if (!configured.load(std::memory_order_acquire)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                hipFuncAttributeMaxDynamicSharedMemorySize, kBytes) != hipSuccess)
            return PKV_ERR_LAUNCH;
        configured.store(true, std::memory_order_release);
    }
    hipLaunchKernelGGL(kernel, grid, dim3(kWaves * 64), kBytes, st, p);
    return launch_status();
}
template <typename T, int DP, int NC>
pkv_status launch_main(const QAttnParams& p, dim3 grid, hipStream_t st) {
    const bool multi = p.n_seq > 1;
    return p.D == DP ? (multi ? launch_kernel<T, DP, true, NC, true>(p, grid, st)
                              : launch_kernel<T, DP, true, NC, false>(p, grid, st))
                     : (multi ? launch_kernel<T, DP, false, NC, true>(p, grid, st)
                              : launch_kernel<T, DP, false, NC, false>(p, grid, st));
}
template <typename T>
pkv_status launch_main(const QAttnParams& p, int nc, dim3 grid, hipStream_t st) {
    if (p.D > 128) return launch_main<T, 256, 1>(p, grid, st);
    if (p.D > 64) {
        if constexpr (sizeof(T) == 2)
            if (nc == 2) return launch_main<T, 128, 2>(p, grid, st);
        return launch_main<T, 128, 1>(p, grid, st);
    }
    if constexpr (sizeof(T) == 2)
        if (nc == 2) return launch_main<T, 64, 2>(p, grid, st);
    return launch_main<T, 64, 1>(p, grid, st);
}

template <typename T, int WAVES>
pkv_status launch_join(const QAttnParams& p, int64_t m, hipStream_t st) {
    hipLaunchKernelGGL((qcache_attn_join_kernel<T, WAVES>), dim3((unsigned)(m * p.hq)), dim3(WAVES * 64), 0,
                       st, p);
    return launch_status();
}

struct QPlan {
    int nc, log2_wg;
    int64_t tiles;
    size_t parts;
};

QPlan plan(const pkv_layer_cfg& cfg, int64_t rows, int64_t m, int64_t n_seq) {
    QPlan pl;
    const int64_t cols = m / n_seq * (cfg.n_q_heads / cfg.n_kv_heads);
    // columns of a workgroup: as many as there are, up to what the registers hold
    pl.nc = cols <= 16 || cfg.dtype == PKV_F32 || cfg.head_dim > 128 ? 1 : 2;
    pl.tiles = ceil_div(cols, 16 * pl.nc);
    // about a workgroup per CU, and no more than there can be groups; one for a short cache, whose
    // few steps in a row cost less than a second launch
    int64_t want = std::min(256 / std::max<int64_t>(1, cfg.n_kv_heads * pl.tiles),
                            (ceil_div(rows, kGroup) + 1) * n_seq);
    if (n_seq == 1 && rows <= 8 * kGroup) want = 1;
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
    const bool bf16 = cfg.dtype == PKV_BF16;
    const dim3 grid((unsigned)p.n_wg, (unsigned)cfg.n_kv_heads, (unsigned)pl.tiles);
    const pkv_status status = bf16 ? launch_main<bf16_t>(p, pl.nc, grid, st)
                                   : launch_main<float>(p, pl.nc, grid, st);
    if (status != PKV_OK) return status;
    if (n_seq == 1 && p.n_wg == 1) return PKV_OK;
    // Waves for the parts that a row has: a dozen or more on average, a few, hardly any where there are more
    // sequences than workgroups (but a thread for each element).  Eight, four and two waves: one sequence of
    // 131328 rows 31.2, 31.8 and 33.1 us, 9 of 100 to 5000 on 128 workgroups 11.6, 12.0 and 12.3, 16 of 0 to
    // 12033 on 32 20.1, 19.8 and 19.6, four with four rows each 18.1, 17.3 and 17.9, 100 of 300 27.6, 25.5
    // and 24.4.
    if (n_seq * 12 <= p.n_wg || n_seq == 1)
        return bf16 ? launch_join<bf16_t, 8>(p, m, st) : launch_join<float, 8>(p, m, st);
    if (n_seq <= p.n_wg || p.D > 128)
        return bf16 ? launch_join<bf16_t, 4>(p, m, st) : launch_join<float, 4>(p, m, st);
    return bf16 ? launch_join<bf16_t, 2>(p, m, st) : launch_join<float, 2>(p, m, st);
}

}  // namespace pkv
