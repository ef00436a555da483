// Causal attention over a packed prompt: row i attends the row_pos[i] + 1 rows that end with itself.
// (Paper: Sec. 2 - the method's input are chunks that were prefilled one by one.)
//
// bf16: S^T = K Q^T,  O^T += V^T P^T  (v_mfma_f32_32x32x16_bf16), softmax along a lane's registers.
// A workgroup of four waves owns 128 consecutive (row, head of the group) columns of a kv head, 32 a
// wave, whichever sequences they belong to: many short sequences fill a tile as well as a long
// one, and the tiles are known without a look at the lengths.  It goes over the keys from the first
// that one of its rows sees to the last, 64 at a time; every column masks with its own two ends, and
// a wave skips what none of its columns sees.  K and V tiles come into LDS by direct loads, the
// next ones while some are used; 64 KB (head_dim 128) leave room for a second workgroup on the CU, whose
// products run under this one's exponentials.
//
// The reference of a column's exponentials follows the running maximum only when that is 2^8 or more
// above it: most tiles neither rescale nor exchange anything between lanes.  The weights go into the second
// product in bf16, which is what the matrix instructions take; their sum is of the unrounded ones.  Error against
// 64 bits 1.3 times that of fp32 weights (the timed cases: 0.0020 of the results' norm and 0.0016).
//
// Measured (32 heads on 8, head_dim 128, bf16): seven sequences of 17 to 8192 rows, 23344 together, 1.06 to
// 1.09 ms, 1.05 to 1.08 PFLOP/s, where a large product of the same box reaches 1.40 and these matrix
// instructions alone take 774 us: the power limit, then the exponentials (958 us without) and fills (933).
// Eight of 1 to 512 rows, 2914 together, 27.3 us (12 to read and write them once): a workgroup's set-up and
// results take 9000 of its 28000 clocks.  Few and short ones are a chain of half tiles, 1190 clocks each of
// which the products are 512; nine of 1 to 512 rows, 2000 together, of 8 heads on 2 take 12.9 us.
#include <atomic>
#include <type_traits>

#include "attn_common.h"
#include "attn_tile.h"
#include "lane_ops.h"

namespace pkv {

namespace {

// x is made here: the compiler would move what is used later behind the loop's matrix instructions.
template <typename V>
__device__ __forceinline__ void here(V& x) {
    asm volatile("" : "+v"(x));
}
// What is made from x is made where it is used: made in front of the loop, as the compiler would, it
// takes the place of accumulators.
template <typename V>
__device__ __forceinline__ void not_ahead(V& x) {
    here(x);
}

template <typename T>
struct PackedParams {
    const T *q, *k, *v;
    const int32_t* row_pos;
    T* out;
    float* lse;
    int m, hq, hkv, group, D, n_tiles;
    float c2;   // softmax scale * log2(e)
};

constexpr float kLn2 = 0.69314718055994531f;
constexpr int kThreads = 256;  // bf16

// The tile and kv head of a workgroup.  Later rows see more: first.  Where all workgroups run at once, `many`
// on a CU, every other 256 of them in the opposite order: a CU's are then of different lengths.  (One
// sequence of 2000 rows in fp32, 4 heads of 64: 41 -> 26 us with the work in front of the loop that went
// the same step, four of 512 in bf16, 32 heads on 8: 21.5 -> 19.0.)
__device__ __forceinline__ void job_of(int n_tiles, int hkv, int many, int* tile, int* g) {
    const int n = gridDim.x, first = blockIdx.x & ~255;
    int i = blockIdx.x;
    if (n <= 256 * many && first & 256) i = 2 * first + min(256, n - first) - 1 - i;
    *g = i % hkv;
    *tile = n_tiles - 1 - i / hkv;
}

// What a row sees: keys lo <= t < hi (nothing: hi == 0, and a lo that stays large minus a few tiles)
__device__ __forceinline__ void keys_of(const int32_t* row_pos, int row, bool valid, int* lo,
                                        int* hi) {
    *lo = 0x7fff0000;
    *hi = 0;
    if (!valid) return;
    const int pos = min(row_pos[row], row);
    if (pos < 0) return;
    *lo = row - pos;
    *hi = row + 1;
}

// Columns whose result is not finite though their weights are.  A value of a tile that is not finite comes into
// the products as 0 times infinity for the columns that do not see it, and sums of large values may leave
// the range before they are divided.  So those columns are attended once more by their wave, with
// weights that are divided first (a sum is then no larger than the values), values that are not finite left
// out of the products, and what the column sees of these counted by products with 1 for every key that
// is seen: an element is infinite or NaN where a seen value is.  Keys and values come straight from global
// memory, 32 (fp32: 16) at a time, and values element by element: one NaN that all of 8192 rows of 32 heads on 8
// see makes 3.2 ms of 0.53, NaN in all values 5.5 (fp32, 4 heads of 64: 3.1 and 4.8 of 0.33).  Columns whose
// weights are not finite (a key or query that is not) do not come here: they are NaN.
// ref, inv: of the column, the reference of its exponentials and 1 / their sum; mine: it is one of these.
__device__ __forceinline__ float seen_value(float x, bool plus, bool minus) {
    return plus ? (minus ? __builtin_nanf("") : INFINITY) : minus ? -INFINITY : x;
}

template <int DP>
__device__ __forceinline__ void attend_again(const PackedParams<bf16_t>& p, int row, int head, int g,
                                             int lo, int hi, float ref, float inv, bool mine) {
    constexpr int KC = DP / 16, DB = DP / 32;
    const int lane = threadIdx.x & 63, hh = lane >> 5, l32 = lane & 31;
    if (!mine) lo = 0x7fff0000, hi = 0;
    const int prow = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);   // swap_bits_2_3, as below
    const int64_t row_len = (int64_t)p.hkv * p.D;
    const uint16_t* const vh = reinterpret_cast<const uint16_t*>(p.v) + (int64_t)g * p.D;
    bf16_t* const out = p.out + ((int64_t)row * p.hq + head) * p.D;
    bf16x8 q[KC];
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)      // (out may be q: the other columns' are results by now)
        q[kc] = mine && kc * 16 < p.D
                    ? *reinterpret_cast<const bf16x8*>(
                          p.q + ((int64_t)row * p.hq + head) * p.D + kc * 16 + hh * 8)
                    : bf16x8{};
    f32x16 o[DB];
    uint32_t plus[DB], minus[DB];        // bit r: of o[.][r]
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        plus[db] = minus[db] = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
    }
    const int end = max32(hi);
#pragma unroll 1
    for (int key0 = min32(lo) & ~31; key0 < end; key0 += 32) {
        const bf16_t* const kp = p.k + min(key0 + prow, p.m - 1) * row_len + (int64_t)g * p.D + hh * 8;
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int kc = 0; kc < KC; ++kc)
            if (kc * 16 < p.D) s = mfma32(*reinterpret_cast<const bf16x8*>(kp + kc * 16), q[kc], s);
        const uint32_t bits = bits_between(lo - key0 - 8 * hh, hi - key0 - 8 * hh);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {             // 16 keys, 8 of them this lane's
            bf16x8 w, seen;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool on = bits >> (16 * kb + e) & 1;
                w[e] = (bf16_t)(on ? __builtin_amdgcn_exp2f(fmaf(s[8 * kb + e], p.c2, -ref)) * inv : 0.f);
                seen[e] = (bf16_t)(on ? 1.f : 0.f);
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const int d = db * 32 + l32;
                bf16x8 v, is_plus, is_minus;
                bool any = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = min(key0 + 16 * kb + 8 * hh + e, p.m - 1);
                    const uint16_t x = d < p.D ? vh[t * row_len + d] : 0;
                    const bool off = (x & 0x7f80) == 0x7f80, nan = off && (x & 0x7f);
                    v[e] = __builtin_bit_cast(bf16_t, off ? (uint16_t)0 : x);
                    is_plus[e] = (bf16_t)(nan || x == 0x7f80 ? 1.f : 0.f);
                    is_minus[e] = (bf16_t)(nan || x == 0xff80 ? 1.f : 0.f);
                    any = any || off;
                }
                o[db] = mfma32(v, w, o[db]);
                if (__any(any)) {
                    f32x16 n;
#pragma unroll
                    for (int r = 0; r < 16; ++r) n[r] = 0.f;
                    const f32x16 up = mfma32(is_plus, seen, n), down = mfma32(is_minus, seen, n);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        plus[db] |= (uint32_t)(up[r] > 0.f) << r;
                        minus[db] |= (uint32_t)(down[r] > 0.f) << r;
                    }
                }
            }
        }
    }
    if (!mine) return;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const int d = db * 32 + r4 * 8 + hh * 4;
            bf16x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * r4 + e;
                x[e] = (bf16_t)seen_value(o[db][r], plus[db] >> r & 1, minus[db] >> r & 1);
            }
            if (d < p.D) *reinterpret_cast<bf16x4*>(out + d) = x;
        }
}

__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <int DP>
__device__ __forceinline__ void attend_again_f32(const PackedParams<float>& p, int row, int head,
                                                 int g, int lo, int hi, float ref, float inv,
                                                 bool mine) {
    constexpr int CM = DP / 16;
    const int lane = threadIdx.x & 63, g4 = lane >> 4, l16 = lane & 15, C = p.D / 16;
    if (!mine) lo = 0x7fff0000, hi = 0;
    const int64_t row_len = (int64_t)p.hkv * p.D;
    float* const out = p.out + ((int64_t)row * p.hq + head) * p.D;
    f32x4 q[CM], o[CM];
    uint32_t plus[CM], minus[CM];
#pragma unroll
    for (int c = 0; c < CM; ++c) {
        o[c] = q[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        plus[c] = minus[c] = 0;
        if (mine && c < C)
            q[c] = *reinterpret_cast<const f32x4*>(p.q + ((int64_t)row * p.hq + head) * p.D + 16 * c +
                                                   4 * g4);
    }
    const int end = uniform(max16(hi));
#pragma unroll 1
    for (int t0 = uniform(min16(lo)) & ~15; t0 < end; t0 += 16) {
        const float* const kp = p.k + min(t0 + l16, p.m - 1) * row_len + (int64_t)g * p.D + 4 * g4;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CM; ++c)
            if (c < C) {
                const f32x4 k = *reinterpret_cast<const f32x4*>(kp + 16 * c);
#pragma unroll
                for (int j = 0; j < 4; ++j) s = mfma_f32(k[j], q[c][j], s);
            }
        const uint32_t bits = bits_between(lo - t0 - 4 * g4, hi - t0 - 4 * g4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool on = bits >> j & 1;
            const float w = on ? __builtin_amdgcn_exp2f(s[j] * p.c2 - ref) * inv : 0.f, seen = on ? 1.f : 0.f;
            const float* const vp = p.v + min(t0 + 4 * g4 + j, p.m - 1) * row_len + (int64_t)g * p.D +
                                    C * l16;
#pragma unroll
            for (int c = 0; c < CM; ++c)
                if (c < C) {
                    const float x = vp[c];
                    const bool off = !(fabsf(x) < INFINITY);
                    o[c] = mfma_f32(off ? 0.f : x, w, o[c]);
                    if (__any(off)) {
                        const f32x4 n = {0.f, 0.f, 0.f, 0.f};
                        const f32x4 up = mfma_f32(off && !(x < 0.f) ? 1.f : 0.f, seen, n);
                        const f32x4 down = mfma_f32(off && !(x > 0.f) ? 1.f : 0.f, seen, n);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            plus[c] |= (uint32_t)(up[r] > 0.f) << r;
                            minus[c] |= (uint32_t)(down[r] > 0.f) << r;
                        }
                    }
                }
        }
    }
    if (!mine) return;
#pragma unroll
    for (int c = 0; c < CM; ++c)
        if (c < C)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                out[C * (4 * g4 + r) + c] = seen_value(o[c][r], plus[c] >> r & 1, minus[c] >> r & 1);
}

// DP: head_dim rounded up to 64, 128 or 256.  Elements between are 0 in the queries; in the tiles they
// repeat others of the same row.  S: 1, or 2 where the tiles are so few that half of the CUs would idle: two
// waves own 64 columns and every other tile of keys, the other two the rest, and their parts meet in LDS.
template <int DP, int S>
__global__ __launch_bounds__(kThreads, DP == 256 || S == 2 ? 1 : 2) void packed_attn_kernel(
    PackedParams<bf16_t> p) {
    constexpr int W = 4 / S;                  // waves that go over the same keys
    constexpr int kCols = 32 * W;
    constexpr int KC = DP / 16;               // contraction steps of a score
    constexpr int DB = DP / 32;               // 32-row blocks of O^T
    constexpr int CH = DP / 8;                // 16-byte pieces of a row
    constexpr int kRow = DP * 2;              // bytes of a row in LDS
    constexpr int kTile = kBN * kRow;         // 64 keys of K or of V
    constexpr int FILLS = kTile / 1024 / W;   // instructions of a wave for a tile
    constexpr int RPI = 64 / CH;              // rows of a fill instruction
    extern __shared__ __align__(16) unsigned char smem_all[];
    __shared__ int s_lo[4], s_hi[4];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = uniform(tid >> 6) % W, grp = uniform(tid >> 6) / W;   // of the group; the group
    unsigned char* const smem = smem_all + grp * 4 * kTile;
    const int hh = lane >> 5, l32 = lane & 31;
    int tile, g;
    job_of(p.n_tiles, p.hkv, S == 2 || DP == 256 ? 1 : DP == 128 ? 2 : 3, &tile, &g);
    const uint32_t col0 = (uint32_t)tile * kCols, n_cols = (uint32_t)p.m * p.group;

    // ---- global -> LDS -----------------------------------------------------------------------------
    // Keys are counted down from the tile's last row: that end is known before anything is read.  Half
    // tile u of the group holds the 32 keys from key_of(u) on; tile t of values halves 2 t + 1 and 2 t.
    // Piece c of K row r lies at c ^ swizzle: the rows of one operand read are in different banks.  V
    // likewise, for the four rows of a transposing read.
    const int k_end = (int)((min(col0 + kCols, n_cols) - 1) / p.group) + 1;
    auto key_of = [&](int u) __attribute__((always_inline)) {
        return k_end - 32 * ((S == 1 ? u : 2 * S * (u >> 1) + 2 * grp + (u & 1)) + 1);
    };
    auto k_swz = [](int r) { return DP == 64 ? (r >> 1) & 7 : r & 15; };
    auto v_swz = [](int r) { return DP == 64 ? 2 * (r & 2) : 4 * (r & 3); };
    const uint32_t lds = uniform((uint32_t)(uintptr_t)smem);
    const uint32_t row_bytes = (uint32_t)p.hkv * p.D * 2;
    const int fill_row = wave * FILLS * RPI + lane / CH;
    const uint32_t k_piece = (uint32_t)((lane % CH) ^ k_swz(fill_row)) * 16;
    const uint32_t v_piece = (uint32_t)((lane % CH) ^ v_swz(fill_row)) * 16;
    // instruction i takes rows RPI i further, whose swizzle differs by these bits
    auto k_bits = [](int i) { return (uint32_t)(DP == 64 ? 64 * (i & 1) : 16 * (RPI * i & 15)); };
    auto v_bits = [](int i) { return (uint32_t)(DP == 256 ? 128 * (i & 1) : 0); };
    const unsigned char* const k_head = reinterpret_cast<const unsigned char*>(p.k + (int64_t)g * p.D);
    const unsigned char* const v_head = reinterpret_cast<const unsigned char*>(p.v + (int64_t)g * p.D);
    // Keys lie in four places for 32 (a half tile), values in two places for 64 behind them.  This wave's
    // rows of a 64-row fill that begins at key `row0`, to lds_dst; head: the head's keys or values
    auto fill = [&](const unsigned char* head, uint32_t piece, auto bits, uint32_t dst, int row0) {
        const unsigned char* const base = head + (int64_t)max(row0, 0) * row_bytes;
        if (row0 >= 0 && p.D == DP) {         // (a row is a multiple of kRow: the bits are the piece's)
            uint32_t off = (uint32_t)fill_row * row_bytes + piece;
            not_ahead(off);
#pragma unroll
            for (int i = 0; i < FILLS; ++i)
                dma16(base + (uint32_t)(i * RPI) * row_bytes, off ^ bits(i), dst + i * 1024);
        } else if (row0 > -kBN) {             // the first row for those in front of it, pieces likewise
            int row = fill_row + min(row0, 0);
            not_ahead(row);
            not_ahead(piece);
#pragma unroll
            for (int i = 0; i < FILLS; ++i)
                dma16(base, (uint32_t)max(row + i * RPI, 0) * row_bytes +
                                min(piece ^ bits(i), (uint32_t)p.D * 2 - 16), dst + i * 1024);
        }
    };
    // key halves u and u + 1, of which the upper half of the waves fill the first; values of tile t
    const bool upper = wave >= W / 2;
    const uint32_t in_half = wave % (W / 2) * FILLS * 1024;
    auto fill_k = [&](int u) {
        const uint32_t dst = lds + ((u + (upper ? 0 : 1)) & 3) * (kTile / 2) + in_half;
        fill(k_head, k_piece, k_bits, dst, upper ? key_of(u) - 32 : key_of(u + 1));
    };
    auto fill_v = [&](int t) {
        fill(v_head, v_piece, v_bits, lds + (2 + (t & 1)) * kTile + wave * FILLS * 1024,
             key_of(2 * t + 1));
    };
    if (upper) fill(k_head, k_piece, k_bits, lds + in_half, key_of(0) - 32);   // half 0
    fill_k(1);

    // ---- this lane's column ---------------------------------------------------------------------
    int lo, hi;
    bf16x8 qreg[KC];
    {
        const uint32_t col = col0 + wave * 32 + l32;
        const int row = col / (uint32_t)p.group, head = g * p.group + (int)(col - (uint32_t)row * p.group);
        keys_of(p.row_pos, row, col < n_cols, &lo, &hi);
        // rows behind the last one: the last one's queries, for nobody
        const bf16_t* qp = p.q + ((int64_t)min(row, p.m - 1) * p.hq + head) * p.D + hh * 8;
#pragma unroll
        for (int kc = 0; kc < KC; ++kc)
            qreg[kc] = kc * 16 + hh * 8 < p.D ? *reinterpret_cast<const bf16x8*>(qp + kc * 16) : bf16x8{};
    }
    // what some column of the wave sees, and what all of them that see anything do
    const int w_lo = min32(lo), w_hi = max32(hi);
    const int in_lo = max32(hi ? lo : 0), in_hi = min32(hi ? hi : 0x7fffffff);
    if (lane == 0) {
        s_lo[grp * W + wave] = w_lo;
        s_hi[grp * W + wave] = w_hi;
    }

    // ---- LDS -> operands -----------------------------------------------------------------------------
    // A row i of a 32-key block is key swap_bits_2_3(i): a lane's 16 scores are then the keys 8 hh + 0..7
    // and 16 + 8 hh + 0..7, the B operands of the second product
    const int prow = (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
    const uint32_t kaddr = (uint32_t)(prow * kRow + ((hh ^ k_swz(prow)) * 16));   // ^ 32 kc
    uint32_t vaddr[DB];
    {
        const int e = (lane >> 2) & 3, j = lane & 3, gh = (lane >> 4) & 1;
#pragma unroll
        for (int db = 0; db < DB; ++db)
            vaddr[db] = (uint32_t)(2 * kTile + (8 * hh + e) * kRow +
                                   ((db * 4 + gh * 2 + (j >> 1)) ^ v_swz(e)) * 16 + (j & 1) * 8);
    }

    float m2 = -INFINITY, l_run = 0.f;     // l_run: this lane's keys only
    f32x16 o_acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o_acc[db][r] = 0.f;

    // The scores of the next half tile are multiplied while the exponentials of this one are worked out, its
    // values while the maximum of those scores is found: each matrix instruction has vector instructions
    // to run beside it.  So keys are half a tile ahead of values.
    // Halves first .. last - 1 of the group hold keys that some column sees.
    int first = 0x7fffffff, last = 0;
    if (w_hi > w_lo) {
        auto of_group = [&](int n) {          // how many of the workgroup's first n halves
            return S == 1 ? n : n / (2 * S) * 2 + min(max(n % (2 * S) - 2 * grp, 0), 2);
        };
        const int a = of_group((k_end - w_hi) / 32), b = of_group((k_end - 1 - w_lo) / 32 + 1);
        if (S == 1 || a < b) first = a, last = b;
    }
    auto k_op = [&](int u, int kc) __attribute__((always_inline)) {
        return *reinterpret_cast<const bf16x8*>(smem + (u & 3) * (kTile / 2) + (kaddr ^ 32 * kc));
    };
    auto v_op = [&](int u, int i) __attribute__((always_inline)) {   // i: block of elements, then of keys
        const unsigned char* a = smem + (u >> 1 & 1) * kTile + (~u & 1) * 32 * kRow +
                                 16 * (i / DB) * kRow + vaddr[i % DB];
        const bf16x4 x = lds_read_tr(a), y = lds_read_tr(a + 4 * kRow);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto largest = [&](const f32x16& s) __attribute__((always_inline)) {
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        return top;
    };
    // the ends of the columns' keys, and the reference; s: of half u, top: its largest
    auto settle = [&](int u, f32x16& s, float top, auto begins) __attribute__((always_inline)) {
        const int key0 = key_of(u);
        if (__builtin_expect(key0 < in_lo || key0 + 32 > in_hi, 0)) {
            // element r is key 16 (r / 8) + 8 hh + r % 8
            const uint32_t seen = bits_between(lo - key0 - 8 * hh, hi - key0 - 8 * hh);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = where_bit(seen, 16 * (r / 8) + r % 8, s[r]);
            top = largest(s);
        }
        top *= p.c2;
        if (__builtin_expect(__any(top > m2 + 8.f), 0)) {
            float mx = fmaxf(top, m2);
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float corr = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m2 - mx);
            m2 = mx;
            if (decltype(begins)::value) return;   // nothing has been added up
            l_run *= corr;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) o_acc[db][r] *= corr;
        }
    };
    // Half u (its number modulo 4 is a constant), of which s are the scores, and `next`, those of the half
    // behind it: a product, its share of the vector work, a product.  Operands are requested AHEAD
    // products ahead (LDS answers after some 200 clocks, a product takes 32), those of the next half's
    // keys too where they are there; a weight is summed and packed one product behind its exponential.
    // A wave skips the halves that none of its columns sees.
    constexpr int NK = KC, NV = 2 * DB, AHEAD = DP == 256 ? 4 : DP == 128 ? 6 : 4;
    bf16x8 op[AHEAD];
    auto half = [&](auto u4, int u, const f32x16& s, f32x16& next) __attribute__((always_inline)) {
        constexpr int U = decltype(u4)::value;
        if (u + 1 < first || u >= last) return;
        const float ref = m2 == -INFINITY ? 0.f : m2;
        bf16x8 pb[2];
        f32x16 zero;
        float e[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) zero[r] = 0.f;
        auto exponential = [&](int r) __attribute__((always_inline)) {
            e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.c2, -ref));
            here(e[r]);
        };
        auto sum = [&](int r) __attribute__((always_inline)) {
            l_run += e[r];
            here(l_run);
            pb[r / 8][r % 8] = (bf16_t)e[r];
        };
        if (U % 2 == 0 || u < first) {          // (else the half before has)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) op[i] = k_op(U + 1, i);
        }
#pragma unroll
        for (int i = 0; i < NK; ++i) {          // with the first eight weights
            __builtin_amdgcn_sched_barrier(0);
            next = mfma32(op[i % AHEAD], qreg[i], i ? next : zero);
            op[i % AHEAD] = i + AHEAD < NK ? k_op(U + 1, i + AHEAD) : v_op(U, i + AHEAD - NK);
#pragma unroll
            for (int r = i * 8 / NK; r < (i + 1) * 8 / NK; ++r) {
                exponential(r);
                if (r) sum(r - 1);
            }
        }
        sum(7);
        float top = -INFINITY;
        bf16x8 after[AHEAD];
#pragma unroll
        for (int i = 0; i < NV; ++i) {          // with the other eight, and then the maximum
            __builtin_amdgcn_sched_barrier(0);
            o_acc[i % DB] = mfma32(op[(i + NK) % AHEAD], pb[i / DB], o_acc[i % DB]);
            if (i + AHEAD < NV) op[(i + NK) % AHEAD] = v_op(U, i + AHEAD);
            else if (U % 2 == 0) after[i + AHEAD - NV] = k_op(U + 2, i + AHEAD - NV);
            if (i < DB) {
#pragma unroll
                for (int r = 8 + i * 8 / DB; r < 8 + (i + 1) * 8 / DB; ++r) {
                    exponential(r);
                    if (r > 8) sum(r - 1);
                }
                if (i == DB - 1) sum(15);
            } else {
#pragma unroll
                for (int r = (i - DB) * 16 / DB; r < (i - DB + 1) * 16 / DB; ++r)
                    top = fmaxf(top, next[r]);
                here(top);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (U % 2 == 0) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) op[i] = after[i];
        }
        settle(u + 1, next, top, std::false_type{});
    };
    f32x16 s0, s1;      // scores of even halves, of odd ones; weights of 0 in front of the first
#pragma unroll
    for (int r = 0; r < 16; ++r) s0[r] = s1[r] = -INFINITY;
    wait_vm<0>();
    // the queries have come too, and nothing waits for them inside the loop, behind fills on their way
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) here(qreg[kc]);
    fill_v(0);      // not before: the queries would come behind it (50 chunks of 100 rows 26.0 -> 25.4 us)
    __syncthreads();
    const int k_lo = uniform(min(min(s_lo[0], s_lo[1]), min(s_lo[2], s_lo[3])));
    const int k_hi = uniform(max(max(s_hi[0], s_hi[1]), max(s_hi[2], s_hi[3])));
    const int n_iter = k_hi > k_lo ? (k_end - k_lo + S * kBN - 1) / (S * kBN) : 0;   // both groups
    // tile t begins: its values and the key halves 2 t + 1 and 2 t + 2 are there, everybody is done with
    // what the next fills replace
    auto begin_tile = [&](int t) __attribute__((always_inline)) {
        wait_vm<0>();
        __syncthreads();
        if (t + 1 < n_iter) {
            fill_k(2 * t + 3);
            fill_v(t + 1);
        }
    };
    if (n_iter > 0) {
        if (first == 0) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s0[r] = 0.f;
#pragma unroll
            for (int kc = 0; kc < KC; ++kc) s0 = mfma32(k_op(0, kc), qreg[kc], s0);
            settle(0, s0, largest(s0), std::true_type{});
        }
        for (int t = 0; t < n_iter; t += 2) {
            begin_tile(t);
            half(std::integral_constant<int, 0>{}, 2 * t, s0, s1);
            half(std::integral_constant<int, 1>{}, 2 * t + 1, s1, s0);
            if (t + 1 == n_iter) break;
            begin_tile(t + 1);
            half(std::integral_constant<int, 2>{}, 2 * t + 2, s0, s1);
            half(std::integral_constant<int, 3>{}, 2 * t + 3, s1, s0);
        }
    }

    // ---- the groups' parts: the second leaves its own in the place of its tiles -------------------------
    if constexpr (S == 2) {
        __shared__ float s_m[W][64], s_l[W][64];
        float* const part = reinterpret_cast<float*>(smem_all + 4 * kTile) + wave * DB * 16 * 64 + lane;
        wait_vm<0>();
        __syncthreads();
        if (grp == 1) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) part[(db * 16 + r) * 64] = o_acc[db][r];
            s_m[wave][lane] = m2;
            s_l[wave][lane] = l_run;
        }
        __syncthreads();
        if (grp == 1) return;
        const float mo = s_m[wave][lane], mx = fmaxf(m2, mo), ref = mx == -INFINITY ? 0.f : mx;
        const float a = __builtin_amdgcn_exp2f(m2 - ref), b = __builtin_amdgcn_exp2f(mo - ref);
        m2 = mx;
        l_run = l_run * a + s_l[wave][lane] * b;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                o_acc[db][r] = o_acc[db][r] * a + part[(db * 16 + r) * 64] * b;
    }

    // ---- results: through LDS, so that a column goes out in one piece ------------------------------------
    const float l = l_run + __shfl_xor(l_run, 32);
    const float inv = hi ? 1.f / l : 0.f;
    float checks[4] = {0.f, 0.f, 0.f, 0.f};    // 0 as long as all are finite
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            o_acc[db][r] *= inv;
            checks[r % 4] = fmaf(o_acc[db][r], 0.f, checks[r % 4]);
        }
    const float check = (checks[0] + checks[1]) + (checks[2] + checks[3]);
    int at = l32;
    not_ahead(at);
    const uint32_t col = col0 + wave * 32 + at;
    const int row = col / (uint32_t)p.group, head = g * p.group + (int)(col - (uint32_t)row * p.group);
    // not finite: NaN where the weights are, otherwise attended once more
    const bool again = check != 0.f && col < n_cols && (l > 0.f || !hi);
    const uint64_t not_fine = __ballot(again);
    const uint32_t once_more = (uint32_t)(not_fine | not_fine >> 32);   // by column
    const bool mine = col < n_cols && !(once_more >> at & 1);
    const int oc = mine ? row * p.hq + head : -1;
    if constexpr (S == 1) {
        wait_vm<0>();                          // (tiles without keys: of the first fills)
        __syncthreads();
    }
    unsigned char* const so = smem + wave * 32 * kRow;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            bf16x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (bf16_t)o_acc[db][4 * r4 + e];
            *reinterpret_cast<bf16x4*>(so + at * kRow + ((db * 4 + r4) ^ k_swz(at)) * 16 + hh * 8) = x;
        }
    if (hh == 0 && col < n_cols && p.lse)
        p.lse[(int64_t)row * p.hq + head] = hi ? (m2 + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    int to[CH / 2];
    bf16x8 x[CH / 2];
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {         // all requested before the first goes out
        const int c = i * RPI + lane / CH, piece = lane % CH;
        to[i] = __shfl(oc, c);
        x[i] = *reinterpret_cast<const bf16x8*>(so + c * kRow + (piece ^ k_swz(c)) * 16);
    }
#pragma unroll
    for (int i = 0; i < CH / 2; ++i)
        if (to[i] >= 0 && lane % CH * 8 < p.D)
            *reinterpret_cast<bf16x8*>(p.out + (int64_t)to[i] * p.D + lane % CH * 8) = x[i];
    if (once_more)
        attend_again<DP>(p, row, head, g, lo, hi, m2 == -INFINITY ? 0.f : m2, l > 0.f ? 1.f / l : 0.f,
                         once_more >> at & 1);
}

// ---- fp32 ----------------------------------------------------------------------------------------
// v_mfma_f32_16x16x4_f32: a workgroup owns 16 columns of a kv head, its four waves take every fourth tile of
// 16 keys and meet in LDS; two (head_dim 128) to four (64) workgroups on a CU work while others begin or
// end.  Operands come from global memory as they lie there: lane group g4 of a contraction takes elements
// 4 g4 .. + 3 of every 16, a lane's scores (keys 4 g4 + r) are the B operand of the second product, and
// row i of output block c is element C i + c of the head, so that a lane's piece of a value row is C
// consecutive floats.  A tile is requested before the one in front of it is used.  WIDE: head_dim is DP.
//
// Four sequences of 1 to 143 rows, 300 together, 4 heads of 64: 5.8 us, below the host's time for a call.
// Sixteen of 512, 2.1 GFLOP: 40 us, 54 TFLOP/s (153 in a large product); one of 2000 25, of 8192 302, 114.
// Few short ones are bound by the 1.5 us until the first bytes are there and the steps behind one another;
// many by the bytes that every tile reads from L2 (12 TB/s) and, as much, by the products.  With
// 16 waves and one workgroup on a CU four of 512 took 21.8 us in place of 10.6, one of 4096 103 and 80.
constexpr int kF32Waves = 4;

template <int DP, bool WIDE>
__global__ __launch_bounds__(kF32Waves * 64) void packed_attn_f32_kernel(PackedParams<float> p) {
    constexpr int NW = kF32Waves, CM = DP / 16, kColRow = 17;       // 17: the join reads down the columns
    extern __shared__ __align__(16) float s_part[];   // [NW][DP][17]
    __shared__ float s_m[NW][16], s_l[NW][16];
    __shared__ int s_col[16][4];                    // row, head, lo, hi
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g4 = lane >> 4, l16 = lane & 15;
    int tile, g;
    job_of(p.n_tiles, p.hkv, !WIDE || DP == 256 ? 1 : DP == 128 ? 2 : 4, &tile, &g);
    const int D = WIDE ? DP : p.D, C = D / 16;
    const uint32_t col = (uint32_t)tile * 16 + l16;
    const int row = col / (uint32_t)p.group, head = g * p.group + (int)(col - (uint32_t)row * p.group);
    const bool valid = row < p.m;
    // Keys in tiles of 16 counted down from those that hold the last row's: known before anything is read
    const int last_row = (int)((min((uint32_t)tile * 16 + 16, (uint32_t)p.m * p.group) - 1) / p.group);
    const int k_end = (last_row | 15) + 1;

    // A tile's keys and values by offsets from its first row, the same ones for every tile; behind the last
    // row the loads return 0, and in front of the first tile too: no load depends on a condition, so that
    // none is waited for before its own turn.
    const int row_bytes = p.hkv * D * 4;
    const int k_off = l16 * row_bytes + 16 * g4;
    int v_off[4];   // (an offset for all lanes would not be looked at by the check of the bounds)
#pragma unroll
    for (int j = 0; j < 4; ++j) v_off[j] = (4 * g4 + j) * row_bytes + 4 * C * l16;
    const unsigned char* const kb = reinterpret_cast<const unsigned char*>(p.k + (int64_t)g * D);
    const unsigned char* const vb = reinterpret_cast<const unsigned char*>(p.v + (int64_t)g * D);
    struct Keys {
        f32x4 k[CM];
        float v[4][CM];
    };
    auto load = [&](int t0, Keys& x) __attribute__((always_inline)) {
        const int rows = t0 < 0 ? 0 : min(p.m - t0, 16);
        const int bytes = rows ? (rows - 1) * row_bytes + 4 * D : 0;
        const int64_t at = (int64_t)(rows ? t0 : 0) * row_bytes;
        const auto k = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(kb + at), 0, bytes,
                                                         0x00027000);
        const auto v = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(vb + at), 0, bytes,
                                                         0x00027000);
#pragma unroll
        for (int c = 0; c < CM; ++c)
            if (WIDE || c < C)
                x.k[c] = __builtin_bit_cast(
                    f32x4, __builtin_amdgcn_raw_buffer_load_b128(k, k_off + 64 * c, 0, 0));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (WIDE) {
#pragma unroll
                for (int c = 0; c < CM; c += 4) {
                    const f32x4 y = __builtin_bit_cast(
                        f32x4, __builtin_amdgcn_raw_buffer_load_b128(v, v_off[j] + 4 * c, 0, 0));
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.v[j][c + i] = y[i];
                }
            } else {
#pragma unroll
                for (int c = 0; c < CM; ++c)
                    if (c < C)
                        x.v[j][c] = __uint_as_float(
                            __builtin_amdgcn_raw_buffer_load_b32(v, v_off[j] + 4 * c, 0, 0));
            }
        }
    };
    constexpr int kStep = NW * 16;
    Keys a, b;
    int t = k_end - 16 * (wave + 1);
    load(t, a);

    int lo, hi;
    keys_of(p.row_pos, row, valid, &lo, &hi);
    f32x4 q4[CM], o_acc[CM];
    {
        const float* const qp = p.q + ((int64_t)(valid ? row : 0) * p.hq + head) * D + 4 * g4;
#pragma unroll
        for (int c = 0; c < CM; ++c) {
            o_acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
            q4[c] = o_acc[c];
            if (valid && (WIDE || c < C)) q4[c] = *reinterpret_cast<const f32x4*>(qp + 16 * c);
        }
    }
    const int k_lo = uniform(min16(lo));
    float m2 = -INFINITY, sum = 0.f;                // sum: this lane group's keys only
    auto use = [&](int t, const Keys& x) __attribute__((always_inline)) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, s2 = s;     // two chains: half the latency
#pragma unroll
        for (int c = 0; c < CM; ++c)
            if (WIDE || c < C)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c & 1) s2 = mfma_f32(x.k[c][j], q4[c][j], s2);
                    else s = mfma_f32(x.k[c][j], q4[c][j], s);
                }
        s += s2;
        float top = -INFINITY;
        const uint32_t seen = bits_between(lo - t - 4 * g4, hi - t - 4 * g4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            s[r] = where_bit(seen, r, s[r] * p.c2);
            top = fmaxf(top, s[r]);
        }
        if (__any(top > m2 + 8.f)) {
            float m = fmaxf(top, m2);
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            const float corr = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m2 - m);
            m2 = m;
            sum *= corr;
#pragma unroll
            for (int c = 0; c < CM; ++c) o_acc[c] *= corr;
        }
        const float ref = m2 == -INFINITY ? 0.f : m2;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] - ref);
            sum += s[r];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < CM; ++c)
                if (WIDE || c < C) o_acc[c] = mfma_f32(x.v[j][c], s[j], o_acc[c]);
    };
    while (t + 16 > k_lo) {
        load(t - kStep, b);
        use(t, a);
        load(t - 2 * kStep, a);
        if (t - kStep + 16 > k_lo) use(t - kStep, b);
        t -= 2 * kStep;
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (g4 == 0) {
        s_m[wave][l16] = m2;
        s_l[wave][l16] = sum;
        if (wave == 0) {
            s_col[l16][0] = valid ? row : -1;
            s_col[l16][1] = head;
            s_col[l16][2] = lo;
            s_col[l16][3] = hi;
        }
    }
#pragma unroll
    for (int c = 0; c < CM; ++c)
        if (WIDE || c < C)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                s_part[(wave * DP + C * (4 * g4 + r) + c) * kColRow + l16] = o_acc[c][r];
    __syncthreads();
    // All columns at once, TPC threads each: of one wave, so that a row of queries that its result replaces is
    // still there where the column has to be attended once more
    constexpr int TPC = NW * 64 / 16, EPT = DP / TPC;
    const int cc = tid / TPC, e0 = tid % TPC;
    const int r = s_col[cc][0], h = s_col[cc][1];
    const bool sees = s_col[cc][3] > 0;
    float top = -INFINITY, l = 0.f, f[NW], x[EPT];
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_m[w][cc]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        f[w] = __builtin_amdgcn_exp2f(s_m[w][cc] - ref);
        l += s_l[w][cc] * f[w];
    }
    const float inv = sees ? 1.f / l : 0.f;
    bool fine = true;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
        const int d = e0 + i * TPC;
        x[i] = 0.f;
        if ((WIDE || d < D) && sees) {
#pragma unroll
            for (int w = 0; w < NW; ++w) x[i] += s_part[(w * DP + d) * kColRow + cc] * f[w];
            x[i] *= inv;
            fine = fine && (fabsf(x[i]) < INFINITY || !(l > 0.f));   // weights that are NaN: so is the result
        }
    }
    const uint64_t not_fine = __ballot(!fine && r >= 0);
    const int64_t oc = (int64_t)r * p.hq + h;
    const auto once_more = [&](int c) {    // column c of the wave's
        return (not_fine >> c * TPC & ((1ull << TPC) - 1)) != 0;
    };
    if (r >= 0 && !once_more(lane / TPC)) {
#pragma unroll
        for (int i = 0; i < EPT; ++i)
            if (WIDE || e0 + i * TPC < D) p.out[oc * D + e0 + i * TPC] = x[i];
    }
    if (r >= 0 && e0 == 0 && p.lse)
        p.lse[oc] = sees ? (top + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    if (not_fine) {
        constexpr int CPW = 64 / TPC;
        float mx = -INFINITY, sum_all = 0.f;
        for (int w = 0; w < NW; ++w) mx = fmaxf(mx, s_m[w][l16]);
        for (int w = 0; w < NW; ++w)
            sum_all += s_l[w][l16] * __builtin_amdgcn_exp2f(s_m[w][l16] - (mx == -INFINITY ? 0.f : mx));
        attend_again_f32<DP>(p, s_col[l16][0], s_col[l16][1], g, s_col[l16][2], s_col[l16][3],
                             mx == -INFINITY ? 0.f : mx, sum_all > 0.f ? 1.f / sum_all : 0.f,
                             l16 / CPW == wave && once_more(l16 % CPW));
    }
}

template <typename T>
PackedParams<T> params(const pkv_layer_cfg& cfg, const void* q, const void* k, const void* v,
                       const int32_t* row_pos, void* out, float* lse, int64_t m, float scale) {
    PackedParams<T> p = {};
    p.q = static_cast<const T*>(q);
    p.k = static_cast<const T*>(k);
    p.v = static_cast<const T*>(v);
    p.row_pos = row_pos;
    p.out = static_cast<T*>(out);
    p.lse = lse;
    p.m = (int)m;
    p.hq = cfg.n_q_heads;
    p.hkv = cfg.n_kv_heads;
    p.group = p.hq / p.hkv;
    p.D = cfg.head_dim;
    p.c2 = scale * 1.4426950408889634f;
    return p;
}

// more LDS than a kernel gets unasked; set twice at worst, the calls are idempotent
template <typename Kernel>
bool allow_lds(Kernel kernel, int bytes, std::atomic<bool>* done) {
    if (done->load(std::memory_order_acquire)) return true;
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                            hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess)
        return false;
    done->store(true, std::memory_order_release);
    return true;
}

template <int DP, int S>
pkv_status launch_tiles(PackedParams<bf16_t> p, hipStream_t st) {
    constexpr int kBytes = S * 4 * kBN * DP * 2;
    static std::atomic<bool> done{false};
    if (!allow_lds(packed_attn_kernel<DP, S>, kBytes, &done)) return PKV_ERR_LAUNCH;
    p.n_tiles = (int)ceil_div((int64_t)p.m * p.group, 128 / S);
    const int64_t grid = (int64_t)p.n_tiles * p.hkv;
    if (grid >= (int64_t)1 << 24) return PKV_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((packed_attn_kernel<DP, S>), dim3((unsigned)grid), dim3(kThreads), kBytes, st, p);
    return launch_status();
}

template <int DP, bool WIDE>
pkv_status launch_f32(PackedParams<float> p, hipStream_t st) {
    constexpr int kBytes = kF32Waves * DP * 17 * 4;
    static std::atomic<bool> done{false};
    if (!allow_lds(packed_attn_f32_kernel<DP, WIDE>, kBytes, &done)) return PKV_ERR_LAUNCH;
    p.n_tiles = (int)ceil_div((int64_t)p.m * p.group, 16);
    const int64_t grid = (int64_t)p.n_tiles * p.hkv;
    if (grid >= 1 << 23) return PKV_ERR_UNSUPPORTED;   // a launch holds less than 2^32 threads
    hipLaunchKernelGGL((packed_attn_f32_kernel<DP, WIDE>), dim3((unsigned)grid), dim3(kF32Waves * 64), kBytes, st,
                       p);
    return launch_status();
}

}  // namespace

pkv_status launch_packed_attn(const pkv_layer_cfg& cfg, const void* q, const void* k,
                              const void* v, const int32_t* row_pos, void* out, float* lse_out,
                              int64_t m, float scale, hipStream_t st) {
    const int d = cfg.head_dim;
    if (cfg.dtype == PKV_BF16) {
        const auto p = params<bf16_t>(cfg, q, k, v, row_pos, out, lse_out, m, scale);
        if (d > 128) return launch_tiles<256, 1>(p, st);
        // Half as wide tiles, their keys split, where all of them run at once (head_dim 128: 128 KB of LDS, one
        // on a CU).  Then 512 rows of 32 heads on 8 take 10.9 us in place of 13.2, one sequence of 2000 of 8
        // on 2 25.8 in place of 36.1, four of 512 11.5 and 13.6; where they do not, two of 512 of 32 on 8 take
        // 17.6 in place of 14.3, eight of 8 on 2 21.9 and 15.4 (one of 4096 alone would gain: 53 and 70).
        // head_dim 64: 2000 rows of 16 heads on 4 19.5 and 27.9, four of 512 10.7 and 10.6.
        if (ceil_div(m * p.group, 64) * p.hkv <= (d <= 64 ? 512 : 256))
            return d <= 64 ? launch_tiles<64, 2>(p, st) : launch_tiles<128, 2>(p, st);
        return d <= 64 ? launch_tiles<64, 1>(p, st) : launch_tiles<128, 1>(p, st);
    }
    const auto p = params<float>(cfg, q, k, v, row_pos, out, lse_out, m, scale);
    if (d == 64) return launch_f32<64, true>(p, st);
    if (d == 128) return launch_f32<128, true>(p, st);
    if (d == 256) return launch_f32<256, true>(p, st);
    if (d < 64) return launch_f32<64, false>(p, st);
    return d < 128 ? launch_f32<128, false>(p, st) : launch_f32<256, false>(p, st);
}

}  // namespace pkv
