// page_attn.hpp -- kernels of splice_page_attn (splice_pages.h): the spliced
// attention of cells' new tokens over a cache in 4-bit pages.
//
// Per page of 64 keys and 16 rows (columns of every product):
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, K's codes expanded to bf16 in registers: a
//                 lane's 16 bytes are a block of 32 values of a key and give four operands as they
//                 lie.  (The instructions that take codes and their exponents directly,
//                 v_mfma_scale_f32_16x16x128_f8f6f4 with q as two e4m3 terms, do not
//                 sum exactly: what lies 2^-15 below the largest product is lost, which put lse
//                 1e-3 off behind a key of 50 times the others' size.)
//   P             online softmax in fp32, base 2; a running maximum moves only when a
//                 score passes it by 2^8.  S^T's registers are P^T's as the second product takes it.
//   O^T += V^T P^T  v_mfma_f32_16x16x32_bf16, V's codes expanded to bf16 (exact) in
//                 registers, whose order the page's layout is made for.
// Two forms of work group, four waves each:
//   narrow  R x 16 rows, the waves take pages in turn and are joined at the end through LDS;
//   wide    every wave R x 16 rows of its own, all walk the same pages; a wave expands a
//           quarter of V (and of K, but for heads of 256) and hands it to the others
//           through LDS, in operand order.
// Measured (32 q heads, 8 KV heads of 128, with the join where there is one): narrow, 64 cells of up to
// 16384 rows, 0.56 GB of pages, 120 us, 4.7 TB/s: bound by the bytes; wide, 4096 tokens of one cell over
// themselves, 137 GFLOP, 133 us, 1030 TFLOP/s: bound by the matrix products and the softmax beside them.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "device_common.hpp"
#include "page_plan.hpp"

namespace splice_dev {

using splice::kPageRows;
using splice::PageLayout;

constexpr float kLowest = -3.0e38f;   // a running maximum before the first key
constexpr float kMostWeight = 256.f;  // 2^kSlack

struct PageCall {
    const char *q;
    const uint8_t *pool;
    const int32_t *tables, *clean, *donor;
    __bf16 *out;
    float *lse;
    float *part;       // [parts][C][T][Hq][D], then [parts][C][T][Hq] of (m, l), part_stride floats a part
    int64_t part_stride;
    int C, T, G, Hkv, Tp, span_lo, span_hi, window, zero_donor, n_pages, table_len, n_active;
    int shared, own_rows, own_each, own_per, own_parts;
    int rows_u, tiles_u, tiles_s, prompt_per, prompt_parts, parts;
    float qk_scale;
};

// Cells in words (see tree_plan.hpp); tile: a cell's first own tile, the cell's index above it.
struct PageArgs {
    PageCall call;
    uint32_t step[SPLICE_MAX_CELLS], count_split[SPLICE_MAX_CELLS], cell_tile[SPLICE_MAX_CELLS];
};

// ---------------------------------------------------------------- what a tile walks

// Up to four runs of keys that lie in pages of one table.  Positions count
// prompt slots, then the cell's rows.
struct PageWalk {
    const int32_t *table[4];
    int page0[4], lo[4], hi[4], first[5];   // first page, positions [lo, hi), ordinal of the first page
    int shift;                              // the last run's row 0 is position Tp
    int n;
};

struct PageTile {
    int id;               // page, -1: none
    int pos, lo, hi;      // position of its first row, which of its positions count
    const int32_t *entry; // in its table
    int end;              // the walk's number of the page behind its run
};

// Nobody writes tables meanwhile: scalar loads, which no wait for pages' bytes waits for.
__device__ __forceinline__ int entry_of(const int32_t *table) {
    return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)table;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Page `at` of the walk; behind `end` none.  A table's entry is read on every path (one of a
// walk with pages), so that waits for loads can be counted.  Everything is taken from the walk before
// anything is chosen, and the choice is the same for a whole wave: it stays in scalar registers.
__device__ __forceinline__ PageTile tile_of(const PageWalk &w, int at, int end) {
    const int32_t *t0 = w.table[0], *t1 = w.table[1], *t2 = w.table[2], *t3 = w.table[3];
    const int f1 = w.first[1], f2 = w.first[2], f3 = w.first[3], p0 = w.page0[0], p1 = w.page0[1], p2 = w.page0[2], p3 = w.page0[3];
    const int l0 = w.lo[0], l1 = w.lo[1], l2 = w.lo[2], l3 = w.lo[3], h0 = w.hi[0], h1 = w.hi[1], h2 = w.hi[2], h3 = w.hi[3];
    const int i = uniform(min(at, end - 1));
    PageTile t;
    int page = p0 + i;
    const int32_t *table = t0;
    t.lo = l0;
    t.hi = h0;
    t.end = f1;
    if (i >= f1) {
        page = p1 + i - f1;
        table = t1;
        t.lo = l1;
        t.hi = h1;
        t.end = f2;
    }
    if (i >= f2) {
        page = p2 + i - f2;
        table = t2;
        t.lo = l2;
        t.hi = h2;
        t.end = f3;
    }
    t.pos = page * kPageRows;
    if (i >= f3) {
        page = p3 + i - f3;
        table = t3;
        t.pos = page * kPageRows + w.shift;
        t.lo = l3;
        t.hi = h3;
        t.end = w.n;
    }
    t.entry = table + page;
    t.id = entry_of(t.entry);
    if (at >= end) t.id = -1;
    return t;
}

// Page `at`, STEP pages behind t (pages of one run lie evenly apart: the usual case).
template <int STEP>
__device__ __forceinline__ PageTile tile_after(const PageWalk &w, const PageTile &t, int at, int end) {
    if (at >= min(t.end, end)) return tile_of(w, at, end);
    PageTile n = t;
    n.pos += STEP * kPageRows;
    n.entry += STEP;
    n.id = entry_of(n.entry);
    return n;
}

// ---------------------------------------------------------------- operands

// Places of a lane's share of K, of D / 32 products: row lane % 16, values 8 j .. 8 j + 7 of its
// block; D = 64 has blocks for two lanes each.
template <int D>
struct KeyShare {
    static constexpr int CH = D == 256 ? 2 : 1, W = D == 64 ? 2 : 4;   // pieces of 128 values, dwords of codes of each
    static constexpr int N = CH * W;                                    // products a tile
    static __device__ __forceinline__ int first(int quad) { return D == 64 ? 16 * quad : 32 * quad; }   // value of a piece
};

// q's row as the other operand of those products.
template <int D>
struct QueryRow {
    bf16x8_t v[KeyShare<D>::N];
};

template <int D>
__device__ __forceinline__ void load_query(const char *row, int quad, QueryRow<D> &q) {
    static_for<0, KeyShare<D>::CH>([&](auto c) {
        static_for<0, KeyShare<D>::W>([&](auto j) {
            q.v[c * KeyShare<D>::W + j] = *reinterpret_cast<const bf16x8_t *>(row + (c * 128 + KeyShare<D>::first(quad) + 8 * j) * 2);
        });
    });
}

// A lane's places in the bytes of a page's head, unsigned words: added to a base in scalar registers by the loads.
template <int D>
struct LanePlaces {
    uint32_t key, key_exp, value, value_exp;   // of tile 0, piece 0
    __device__ __forceinline__ explicit LanePlaces(int lane) {
        const uint32_t col = lane & 15, quad = lane >> 4;
        key = col * (D / 2) + (D == 64 ? 8 * quad : 16 * quad);
        key_exp = PageLayout<D>::kKScale + (col * PageLayout<D>::kChunkBlocks + (D == 64 ? quad >> 1 : quad)) * 4;
        value = PageLayout<D>::kV + lane * 16;
        value_exp = PageLayout<D>::kVScale + (quad * 2 + (col >> 3)) * (D / 8);
    }
};

// The lane's codes of 16 keys (tile t of a page).
template <int D>
__device__ __forceinline__ void load_codes(const uint8_t *head, uint32_t at, uint32_t (&w)[KeyShare<D>::N]) {
    if constexpr (D == 64) {
        const uint2 x = *reinterpret_cast<const uint2 *>(head + at);
        w[0] = x.x;
        w[1] = x.y;
    } else {
        static_for<0, KeyShare<D>::CH>([&](auto c) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(head + at + c * 64);
            static_for<0, 4>([&](auto j) { w[4 * c + j] = x[(int)j]; });
        });
    }
}

// The lane's exponent bytes of each piece, a byte a tile of the page.
template <int D>
__device__ __forceinline__ void load_exponents(const uint8_t *head, uint32_t at, uint32_t (&s)[KeyShare<D>::CH]) {
    static_for<0, KeyShare<D>::CH>([&](auto c) { s[c] = *reinterpret_cast<const uint32_t *>(head + at + c * 256); });
}

// Byte n of a word as the power of two that it stands for; 255: infinity, which makes what it scales NaN or infinite.
template <int N>
__device__ __forceinline__ float power(uint32_t w) {
    constexpr int up = 23 - 8 * N;
    return __uint_as_float((up >= 0 ? w << (up & 31) : w >> (-up & 31)) & 0x7f800000u);
}

// Eight codes as eight bf16 values.
__device__ __forceinline__ bf16x8_t expand(uint32_t w, float f) {
    return __builtin_bit_cast(bf16x8_t, u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 0)),
                                                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 1)),
                                                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 2)),
                                                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 3))});
}

// S^T of 16 keys and 16 rows: the lane's row lane % 16, keys 4 (lane / 16) + r.
template <int D, int TL, int R>
__device__ __forceinline__ void scores(const uint32_t (&w)[KeyShare<D>::N], const uint32_t (&e)[KeyShare<D>::CH],
                                       const QueryRow<D> (&q)[R], f32x4_t (&s)[R][4]) {
    static_for<0, R>([&](auto r) { s[r][TL] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
    static_for<0, KeyShare<D>::N>([&](auto n) {
        const bf16x8_t k = expand(w[n], power<TL>(e[n / KeyShare<D>::W]));
        static_for<0, R>([&](auto r) { s[r][TL] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[r].v[n], s[r][TL], 0, 0, 0); });
    });
}

// Whether any byte is 255 (the exponent of a row that is NaN).
__device__ __forceinline__ bool has_nan(uint32_t w) { return ((~w - 0x01010101u) & w & 0x80808080u) != 0; }

// Keys of a page whose exponent bytes are 255, a bit each (a lane's word: those of its column in the four tiles).
__device__ __forceinline__ uint64_t nan_keys(uint32_t w) {
    uint64_t keys = 0;
    if (__any(has_nan(w))) static_for<0, 4>([&](auto t) {
        keys |= (__ballot(((w >> (8 * t)) & 255u) == 255u) & 0xffffull) << (16 * t);
    });
    return keys;
}

// Scale bytes of four keys, position of the first one and of those that
// count: what does not count, and NaN (its scores say so), become 2^-127.
__device__ __forceinline__ uint32_t finite_scales(uint32_t w, int pos, int lo, int hi) {
    uint32_t keep = 0;
    static_for<0, 4>([&](auto f) {
        const int p = pos + f;
        if (p >= lo && p < hi && ((w >> (8 * f)) & 255u) != 255u) keep |= 255u << (8 * f);
    });
    return w & keep;
}

// V's 8 keys x 4 values of a lane as operands m = 0..3 (values 4 i + m).  DW: how many
// dwords (two keys each) of the codes.
template <int DW>
__device__ __forceinline__ void value_operands(const uint32_t (&code)[DW], const uint32_t (&scale)[DW / 2], uint32_t (&op)[4][DW]) {
    static_for<0, DW>([&](auto w) {
        const uint32_t s = scale[w / 2];
        const float f0 = power<2 * (w % 2)>(s), f1 = power<2 * (w % 2) + 1>(s);
        const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[w], f0, 0));
        const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[w], f0, 1));
        const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[w], f1, 2));
        const uint32_t d = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[w], f1, 3));
        op[0][w] = __builtin_amdgcn_perm(c, a, 0x05040100);
        op[1][w] = __builtin_amdgcn_perm(c, a, 0x07060302);
        op[2][w] = __builtin_amdgcn_perm(d, b, 0x05040100);
        op[3][w] = __builtin_amdgcn_perm(d, b, 0x07060302);
    });
}

__device__ __forceinline__ bf16x8_t as_operand(const uint32_t (&w)[4]) {
    return __builtin_bit_cast(bf16x8_t, u32x4_t{w[0], w[1], w[2], w[3]});
}

// ---------------------------------------------------------------- rows

// Rows of a wave: of the lane's column in each of its R sets of 16.
template <int R>
struct PageRowsOf {
    int64_t at[R];     // (cell, token, q head) as an index of out's rows; -1: no row
    int lo[R], hi[R];  // positions it sees
    int zeros[R];      // keys of the ZERO donor it sees, in this part
};

// State of a wave's softmax and second product.
template <int D, int R>
struct PageState {
    f32x4_t o[R][D / 64][4];   // register r of [b][m]: value 64 b + 16 quad + 4 r + m
    float m[R], l[R];          // l: over the lane's own keys
};

template <int D, int R>
__device__ __forceinline__ void start(PageState<D, R> &st, const PageRowsOf<R> &rows, bool first, int quad) {
    static_for<0, R>([&](auto r) {
        static_for<0, D / 64>([&](auto b) {
            static_for<0, 4>([&](auto m) { st.o[r][b][m] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
        });
        const bool zeros = first && rows.zeros[r] > 0;   // keys that score 0, with values 0
        st.m[r] = zeros ? 0.f : kLowest;
        st.l[r] = zeros && quad == 0 ? (float)rows.zeros[r] : 0.f;
    });
}

// What a page's scores are worth to some rows: from, to: the lane's visible keys, counted from its first one of the
// page; nan: keys that are NaN.
__device__ __forceinline__ void mark(f32x4_t (&s)[4], int from, int to, uint64_t nan, int quad) {
    if (nan) static_for<0, 4>([&](auto t) {
        static_for<0, 4>([&](auto r) {
            if ((nan >> (16 * t + r)) >> (4 * quad) & 1) s[t][(int)r] = __uint_as_float(0x7fc00000u);
        });
    });
    static_for<0, 4>([&](auto t) {
        static_for<0, 4>([&](auto r) { s[t][(int)r] = 16 * t + r >= from && 16 * t + r < to ? s[t][(int)r] : -INFINITY; });
    });
}

// The running maxima raised to what the page's scores ask for: those of rows whose own weights do, so that a row's
// result does not depend on the rows beside it.
template <int D, int R>
__device__ __forceinline__ void raise(PageState<D, R> &st, const f32x4_t (&s)[R][4], const float (&sum)[R], float qk) {
    static_for<0, R>([&](auto r) {
        float top = s[r][0][0];
        static_for<1, 16>([&](auto i) { top = fmaxf(top, s[r][i / 4][i % 4]); });
        top *= qk;
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const uint64_t lanes = __ballot(!(sum[r] <= kMostWeight));   // a row's are 16 apart
        const uint32_t half = (uint32_t)lanes | (uint32_t)(lanes >> 32);
        const float now = (half | half >> 16) >> (threadIdx.x & 15) & 1 ? fmaxf(top, st.m[r]) : st.m[r], f = fast_exp2(st.m[r] - now);
        st.m[r] = now;
        st.l[r] *= f;
        static_for<0, D / 64>([&](auto b) { static_for<0, 4>([&](auto m) { st.o[r][b][m] *= f; }); });
    });
}

// Weights of a page as the second product's operands (two of 32 keys); their sums to the rows'.  The operands are
// bf16, off by 2^-8 of a weight at most: a second term each would double the second product's instructions.  That is what sets the
// results' errors, up to 1.41 times those with weights of 32 bits; the sums are of the unrounded weights, as lse is of 32 bits.  The scores'
// maximum is looked for only where a lane's weights sum to more than 2^8 (or to NaN): one of them may then.
template <int D, int R>
__device__ __forceinline__ void weights(PageState<D, R> &st, const f32x4_t (&s)[R][4], float qk, bf16x8_t (&p)[R][2]) {
    typedef float f32x8_t __attribute__((ext_vector_type(8)));
    float sum[R];
    auto all = [&]() {
        static_for<0, R>([&](auto r) {
            static_for<0, 2>([&](auto h) {
                f32x8_t w;
                static_for<0, 8>([&](auto i) { w[(int)i] = fast_exp2(fmaf(s[r][2 * h + i / 4][i % 4], qk, -st.m[r])); });
                const float x = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                sum[r] = h ? sum[r] + x : x;
                p[r][h] = __builtin_convertvector(w, bf16x8_t);
            });
        });
    };
    all();
    bool up = false;
    static_for<0, R>([&](auto r) { up |= !(sum[r] <= kMostWeight); });
    if (__any(up)) {
        raise<D, R>(st, s, sum, qk);
        all();
    }
    static_for<0, R>([&](auto r) { st.l[r] += sum[r]; });
}

// A row's values are there before what follows: a wait in a loop would take later loads with it.
template <int D, int R>
__device__ __forceinline__ void settle(const QueryRow<D> (&q)[R]) {
    static_for<0, R>([&](auto r) {
        static_for<0, KeyShare<D>::N>([&](auto n) {
            const u32x4_t w = __builtin_bit_cast(u32x4_t, q[r].v[n]);
            asm volatile("" ::"v"(w));
        });
    });
}

// Least and largest over the wave's rows.
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) x = min(x, __shfl_xor(x, o));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x) { return -wave_min(-x); }

// ---------------------------------------------------------------- results

// 16 values of a row to out, or to its partial result.
template <int D>
__device__ __forceinline__ void put16(const PageCall &a, int part, int64_t at, int d, const float (&x)[16], float by) {
    if (part < 0) {
        typedef float f32x8_t __attribute__((ext_vector_type(8)));
        static_for<0, 2>([&](auto h) {
            f32x8_t y;
            static_for<0, 8>([&](auto i) { y[(int)i] = x[8 * h + i] * by; });
            *reinterpret_cast<bf16x8_t *>(a.out + at * D + d + 8 * h) = __builtin_convertvector(y, bf16x8_t);
        });
        return;
    }
    float *p = a.part + part * a.part_stride + at * D + d;
    static_for<0, 4>([&](auto i) {
        *reinterpret_cast<f32x4_t *>(p + 4 * i) = f32x4_t{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    });
}

template <int D>
__device__ __forceinline__ void put_record(const PageCall &a, int part, int64_t at, float m, float l) {
    if (part < 0) {
        a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
        return;
    }
    float2 *rec = reinterpret_cast<float2 *>(a.part + part * a.part_stride + (int64_t)a.C * a.T * a.G * a.Hkv * D);
    rec[at] = make_float2(m, l);
}

// What a row's sum is divided by: nothing seen gives 0.
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }

// ---------------------------------------------------------------- narrow

template <int D, int R>
struct NarrowShared {
    float o[4][16 * R][D + 4];
    float m[4][16 * R], l[4][16 * R];
    int64_t at[16 * R];
};

// Pages that a wave has in registers or on their way there.  Two hide the memory's latency behind the other's
// products (64 cells of 8k rows, D = 128, a part a cell: 181 us with one, 126 with two; 120 with the plan of now); what they take of registers beside two
// sets of rows, or rows of 256, leaves room for one.
constexpr int narrow_pages(int D, int R) { return D == 64 || (D == 128 && R == 1) ? 2 : 1; }

// Pages [i0, i1) of the walk for R x 16 rows, the waves a page each in turn.
template <int D, int R>
__device__ __forceinline__ void narrow(const PageCall &a, const PageWalk &walk, int i0, int i1, int h, const PageRowsOf<R> &rows,
                                       bool first, int part, NarrowShared<D, R> &sh) {
    constexpr int B = D / 64, PF = narrow_pages(D, R), STEP = 4 * PF;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    const int64_t page_bytes = (int64_t)a.Hkv * PageLayout<D>::kBytes;
    const uint8_t *pool = a.pool + (int64_t)h * PageLayout<D>::kBytes;
    const LanePlaces<D> at(lane);
    QueryRow<D> q[R];
    int lo_most = rows.lo[0], hi_least = rows.hi[0];
    static_for<0, R>([&](auto r) {
        load_query<D>(a.q + (rows.at[r] < 0 ? 0 : rows.at[r]) * D * 2, quad, q[r]);
        lo_most = max(lo_most, rows.lo[r]);
        hi_least = min(hi_least, rows.hi[r]);
    });
    lo_most = wave_max(lo_most);
    hi_least = wave_min(hi_least);
    PageState<D, R> st;
    start<D, R>(st, rows, first && wave == 0, quad);
    struct Slot {
        PageTile now, next;   // the page in the registers, and the one that follows it there
        uint32_t kc[4][KeyShare<D>::N], ke[KeyShare<D>::CH];
        u32x4_t vc[2][B];
        uint32_t vs[2][B][2];
    };
    auto there = [&](const PageTile &t) { return t.id >= 0 && t.id < a.n_pages; };
    auto head_of = [&](const PageTile &t) { return pool + (uint64_t)(uint32_t)(there(t) ? t.id : 0) * (uint64_t)page_bytes; };
    auto load_keys = [&](Slot &p, const uint8_t *head) {
        static_for<0, 4>([&](auto t) { load_codes<D>(head, at.key + t * (8 * D), p.kc[t]); });
        load_exponents<D>(head, at.key_exp, p.ke);
    };
    auto load_values = [&](Slot &p, const uint8_t *head) {
        static_for<0, 2>([&](auto t) {
            static_for<0, B>([&](auto b) {
                p.vc[t][b] = *reinterpret_cast<const u32x4_t *>(head + at.value + (t * B + b) * 1024);
                const uint2 s = *reinterpret_cast<const uint2 *>(head + at.value_exp + t * D + b * 8);
                p.vs[t][b][0] = s.x;
                p.vs[t][b][1] = s.y;
            });
        });
    };
    // The page of a slot, number i of the walk; the bytes of page i + STEP take its place.
    auto page = [&](Slot &slot, int i) {
        const PageTile now = slot.now;
        f32x4_t s[R][4];
        static_for<0, 4>([&](auto t) { scores<D, decltype(t)::value, R>(slot.kc[t], slot.ke, q, s); });
        const uint64_t nan = nan_keys(slot.ke[0]);
        const uint8_t *head = head_of(slot.next);
        load_keys(slot, head);
        slot.now = slot.next;
        slot.next = tile_after<STEP>(walk, slot.now, i + 2 * STEP, i1);
        if (there(now)) {
            const bool edge = now.pos < now.lo || now.pos + kPageRows > now.hi;
            if (edge || nan || now.pos < lo_most || now.pos + kPageRows > hi_least) {
                if (edge || nan) static_for<0, 2>([&](auto t) {
                    static_for<0, B>([&](auto b) {
                        static_for<0, 2>([&](auto e) {
                            slot.vs[t][b][e] = finite_scales(slot.vs[t][b][e], now.pos + 32 * t + 16 * e + 4 * quad, now.lo, now.hi);
                        });
                    });
                });
                const int base = now.pos + 4 * quad;
                static_for<0, R>([&](auto r) {
                    mark(s[r], max(now.lo, rows.lo[r]) - base, min(now.hi, rows.hi[r]) - base, nan, quad);
                });
            }
            bf16x8_t p[R][2];
            weights<D, R>(st, s, a.qk_scale, p);
            static_for<0, 2>([&](auto t) {
                static_for<0, B>([&](auto b) {
                    const uint32_t code[4] = {slot.vc[t][b][0], slot.vc[t][b][1], slot.vc[t][b][2], slot.vc[t][b][3]};
                    uint32_t op[4][4];
                    value_operands<4>(code, slot.vs[t][b], op);
                    static_for<0, 4>([&](auto m) {
                        static_for<0, R>([&](auto r) {
                            st.o[r][b][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_operand(op[m]), p[r][t], st.o[r][b][m], 0, 0, 0);
                        });
                    });
                });
            });
        }
        load_values(slot, head);
    };
    Slot slot[PF];
    int i = i0 + wave;
    if (i < i1) {
        static_for<0, PF>([&](auto n) {
            slot[n].now = tile_of(walk, i + 4 * n, i1);
            slot[n].next = tile_after<STEP>(walk, slot[n].now, i + 4 * n + STEP, i1);
        });
        static_for<0, PF>([&](auto n) {
            load_keys(slot[n], head_of(slot[n].now));
            load_values(slot[n], head_of(slot[n].now));
            __builtin_amdgcn_sched_barrier(0);   // in the loop's order, so that its waits count as few of them
        });
        settle<D, R>(q);   // asked for before the pages
        for (; i < i1; i += STEP) static_for<0, PF>([&](auto n) { page(slot[n], i + 4 * n); });
    }
    // the four waves' results are one
    static_for<0, R>([&](auto r) {
        st.l[r] += __shfl_xor(st.l[r], 16);
        st.l[r] += __shfl_xor(st.l[r], 32);
        if (quad == 0) {
            sh.m[wave][16 * r + col] = st.m[r];
            sh.l[wave][16 * r + col] = st.l[r];
            if (wave == 0) sh.at[16 * r + col] = rows.at[r];
        }
    });
    __syncthreads();
    static_for<0, R>([&](auto r) {
        const int row = 16 * r + col;
        const float top = fmaxf(fmaxf(sh.m[0][row], sh.m[1][row]), fmaxf(sh.m[2][row], sh.m[3][row]));
        const float f = fast_exp2(st.m[r] - top);
        static_for<0, B>([&](auto b) {
            static_for<0, 4>([&](auto n) {
                *reinterpret_cast<f32x4_t *>(&sh.o[wave][row][64 * b + 16 * quad + 4 * n]) =
                    f32x4_t{st.o[r][b][0][(int)n] * f, st.o[r][b][1][(int)n] * f, st.o[r][b][2][(int)n] * f,
                            st.o[r][b][3][(int)n] * f};
            });
        });
    });
    __syncthreads();
    for (int u = threadIdx.x; u < 16 * R * (D / 16); u += kThreads) {
        const int row = u / (D / 16), d = 16 * (u % (D / 16));
        const int64_t at = sh.at[row];
        if (at < 0) continue;
        const float top = fmaxf(fmaxf(sh.m[0][row], sh.m[1][row]), fmaxf(sh.m[2][row], sh.m[3][row]));
        float l = 0.f;
        static_for<0, 4>([&](auto w) { l += sh.l[w][row] * fast_exp2(sh.m[w][row] - top); });
        if (d == 0) put_record<D>(a, part, at, top, l);
        if (part >= 0 && l == 0.f) continue;
        float x[16];
        static_for<0, 4>([&](auto j) {
            f32x4_t y = {0.f, 0.f, 0.f, 0.f};
            static_for<0, 4>([&](auto w) { y += *reinterpret_cast<const f32x4_t *>(&sh.o[w][row][d + 4 * j]); });
            static_for<0, 4>([&](auto n) { x[4 * j + n] = y[(int)n]; });
        });
        put16<D>(a, part, at, d, x, inverse(l));
    }
}

// ---------------------------------------------------------------- wide

// K's operands too go through LDS while two pages of both leave room for two work groups.
template <int D>
struct WideShared {
    static constexpr bool kKeys = D <= 128;
    u32x4_t k[kKeys ? 2 : 1][kKeys ? 4 * KeyShare<D>::N : 1][64];   // operands (16-key tile, product), a lane's 16 bytes each
    u32x4_t v[2][2 * (D / 64) * 4][64];                             // operands (32-key tile, 64 values, m)
};

// Pages [i0, i1) of the walk, every wave R x 16 rows of its own.  Page i + 1 is expanded
// while page i is computed with, its bytes loaded a page before.
template <int D, int R>
__device__ __forceinline__ void wide(const PageCall &a, const PageWalk &walk, int i0, int i1, int h, const PageRowsOf<R> &rows,
                                     bool first, int part, WideShared<D> &sh) {
    constexpr int B = D / 64, UNITS = D >= 128 ? D / 128 : 1;   // pieces of V a wave expands
    constexpr int DW = D == 64 ? 2 : 4;                         // ... dwords of codes a lane has of each
    constexpr int N = KeyShare<D>::N, CH = KeyShare<D>::CH, KT = WideShared<D>::kKeys ? 1 : 4;   // 16-key tiles of K a wave expands
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;
    const int64_t page_bytes = (int64_t)a.Hkv * PageLayout<D>::kBytes;
    const uint8_t *pool = a.pool + (int64_t)h * PageLayout<D>::kBytes;
    const LanePlaces<D> place(lane);
    QueryRow<D> q[R];
    int lo_most = rows.lo[0], hi_least = rows.hi[0], lo_least = rows.lo[0], hi_most = rows.hi[0];
    static_for<0, R>([&](auto r) {
        load_query<D>(a.q + (rows.at[r] < 0 ? 0 : rows.at[r]) * D * 2, quad, q[r]);
        lo_most = max(lo_most, rows.lo[r]);
        lo_least = min(lo_least, rows.lo[r]);
        hi_least = min(hi_least, rows.hi[r]);
        hi_most = max(hi_most, rows.hi[r]);
    });
    lo_most = wave_max(lo_most);
    lo_least = wave_min(lo_least);
    hi_least = wave_min(hi_least);
    hi_most = wave_max(hi_most);
    bool some = false;   // a wave without rows hands over its share of the pages, and computes nothing
    static_for<0, R>([&](auto r) { some |= rows.at[r] >= 0; });
    if (!__any(some)) hi_most = -1;
    PageState<D, R> st;
    start<D, R>(st, rows, first, quad);
    uint32_t kc[KT][N], ke[CH], vc[UNITS][DW], vs[UNITS][DW / 2];
    uint32_t kn = 0;   // with K's bytes loaded a page later than V's: exponents that tell of NaN
    auto there = [&](const PageTile &t) { return t.id >= 0 && t.id < a.n_pages; };
    auto head_of = [&](const PageTile &t) { return pool + (uint64_t)(uint32_t)(there(t) ? t.id : 0) * (uint64_t)page_bytes; };
    auto load_keys = [&](const uint8_t *head) {
        static_for<0, KT>([&](auto t) { load_codes<D>(head, place.key + (KT == 1 ? wave * (8 * D) : t * (8 * D)), kc[t]); });
        load_exponents<D>(head, place.key_exp, ke);
    };
    // piece u of wave w: D = 64 (32-key tile w / 2, half w % 2 of its keys), else (tile, 64 values) w * UNITS + u
    auto load_values = [&](const uint8_t *head) {
        if constexpr (KT == 4) kn = *reinterpret_cast<const uint32_t *>(head + place.key_exp);
        if constexpr (D == 64) {
            const int t = wave >> 1, e = wave & 1;
            const uint2 c = *reinterpret_cast<const uint2 *>(head + (place.value + t * 1024 + e * 8));
            vc[0][0] = c.x;
            vc[0][1] = c.y;
            vs[0][0] = *reinterpret_cast<const uint32_t *>(head + (place.value_exp + t * D + e * 4));
        } else {
            static_for<0, UNITS>([&](auto u) {
                const int n = wave * UNITS + u, t = n / B, b = n % B;
                const u32x4_t c = *reinterpret_cast<const u32x4_t *>(head + (place.value + n * 1024));
                const uint2 s = *reinterpret_cast<const uint2 *>(head + (place.value_exp + t * D + b * 8));
                static_for<0, 4>([&](auto j) { vc[u][j] = c[(int)j]; });
                vs[u][0] = s.x;
                vs[u][1] = s.y;
            });
        }
    };
    // What of the values' exponents stands for nothing, out of the way.
    auto clean = [&](const PageTile &t) {
        static_for<0, UNITS>([&](auto u) {
            const int n = D == 64 ? wave >> 1 : wave * UNITS + u;
            static_for<0, DW / 2>([&](auto e) {
                const int half = D == 64 ? wave & 1 : (int)e;
                vs[u][e] = finite_scales(vs[u][e], t.pos + 32 * (n / B) + 16 * half + 4 * quad, t.lo, t.hi);
            });
        });
    };
    auto at_edge = [&](const PageTile &t) { return t.pos < t.lo || t.pos + kPageRows > t.hi; };
    // The wave's share of a page to LDS.
    auto hand_over = [&](int at) {
        if constexpr (WideShared<D>::kKeys) static_for<0, N>([&](auto n) {
            const float f = __uint_as_float((ke[n / KeyShare<D>::W] >> (8 * wave) & 255u) << 23);
            sh.k[at][wave * N + n][lane] = __builtin_bit_cast(u32x4_t, expand(kc[0][n], f));
        });
        static_for<0, UNITS>([&](auto u) {
            const int n = D == 64 ? wave >> 1 : wave * UNITS + u;
            uint32_t op[4][DW];
            value_operands<DW>(vc[u], vs[u], op);
            static_for<0, 4>([&](auto m) {
                if constexpr (D == 64) {
                    reinterpret_cast<uint2 *>(&sh.v[at][n * 4 + m][lane])[wave & 1] = make_uint2(op[m][0], op[m][1]);
                } else {
                    sh.v[at][n * 4 + m][lane] = u32x4_t{op[m][0], op[m][1], op[m][2], op[m][3]};
                }
            });
        });
    };
    PageTile now{}, next{}, after{};
    uint64_t nan = 0;
    if (i0 < i1) {
        now = tile_of(walk, i0, i1);
        next = tile_of(walk, i0 + 1, i1);
        after = tile_of(walk, i0 + 2, i1);
        load_keys(head_of(now));
        load_values(head_of(now));
        nan = nan_keys(KT == 4 ? kn : ke[0]);
        if (at_edge(now) || nan) clean(now);
        hand_over(0);
        if (KT == 1) load_keys(head_of(next));
        load_values(head_of(next));
        settle<D, R>(q);
    }
    for (int i = i0; i < i1; ++i) {
        const int at = (i - i0) & 1;
        const bool seen = there(now) && now.pos < hi_most && now.pos + kPageRows > lo_least;   // by some row of the wave
        const bool masked = at_edge(now) || now.pos < lo_most || now.pos + kPageRows > hi_least;
        const uint64_t nan_next = nan_keys(KT == 4 ? kn : ke[0]);
        if (at_edge(next) || nan_next) clean(next);
        __syncthreads();   // page i is in LDS, and of page i - 1 nothing is read any more
        // the next page is handed over (behind the last one some page, which nobody reads), the one behind it asked for
        auto go_on = [&]() {
            hand_over(at ^ 1);
            if (KT == 1) load_keys(head_of(after));
            load_values(head_of(after));
        };
        if (!seen) {
            if constexpr (KT == 4) load_keys(head_of(next));
            go_on();
        } else {
            // Ahead of the compute unit's other waves up to the softmax: what all waves of the group wait for at the
            // next barrier is done early, and one wave's products fall beside another's softmax.  32/8 heads of 128:
            // 4096 nodes of one cell 131 us against 153 without, 2 cells of 4096 262 against 274, 4 of 1024 62 against
            // 59; through the second product too 134, let go before the expansion 157.
            __builtin_amdgcn_s_setprio(1);
            f32x4_t s[R][4];
            if constexpr (KT == 4) {
                // K is the wave's own: this page's, then the next one's bytes
                static_for<0, 4>([&](auto t) { scores<D, decltype(t)::value, R>(kc[KT == 4 ? (int)t : 0], ke, q, s); });
                load_keys(head_of(next));
            } else {
                static_for<0, 4>([&](auto t) {
                    static_for<0, R>([&](auto r) { s[r][t] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
                    static_for<0, N>([&](auto n) {
                        const bf16x8_t k = __builtin_bit_cast(bf16x8_t, sh.k[at][t * N + n][lane]);
                        static_for<0, R>([&](auto r) { s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[r].v[n], s[r][t], 0, 0, 0); });
                    });
                });
            }
            go_on();
            if (masked || nan) {
                const int base = now.pos + 4 * quad;
                static_for<0, R>([&](auto r) {
                    mark(s[r], max(now.lo, rows.lo[r]) - base, min(now.hi, rows.hi[r]) - base, nan, quad);
                });
            }
            bf16x8_t p[R][2];
            __builtin_amdgcn_s_setprio(0);
            weights<D, R>(st, s, a.qk_scale, p);
            static_for<0, 2>([&](auto t) {
                static_for<0, B>([&](auto b) {
                    static_for<0, 4>([&](auto m) {
                        const bf16x8_t v = __builtin_bit_cast(bf16x8_t, sh.v[at][(t * B + b) * 4 + m][lane]);
                        static_for<0, R>([&](auto r) {
                            st.o[r][b][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[r][t], st.o[r][b][m], 0, 0, 0);
                        });
                    });
                });
            });
        }
        now = next;
        next = after;
        after = tile_after<1>(walk, next, i + 3, i1);
        nan = nan_next;
    }
    static_for<0, R>([&](auto r) {
        float l = st.l[r];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (rows.at[r] < 0) return;
        if (quad == 0) put_record<D>(a, part, rows.at[r], st.m[r], l);
        if (part >= 0 && l == 0.f) return;
        const float by = inverse(l);
        static_for<0, B>([&](auto b) {
            float x[16];
            static_for<0, 16>([&](auto n) { x[n] = st.o[r][b][n % 4][n / 4]; });
            put16<D>(a, part, rows.at[r], 64 * b + 16 * quad, x, by);
        });
    });
}

// ---------------------------------------------------------------- the kernel

// The walk of a tile whose rows see positions from `low` on: the prompt
// (spliced or not) and, with rows to show, a cell's own.
__device__ __forceinline__ PageWalk walk_of(const PageCall &a, bool prompt, bool spliced, int low, const int32_t *table, int rows) {
    PageWalk w;
    const int v0 = max(0, min(low, a.Tp)), g0 = max(0, low - a.Tp);
    const bool cut = spliced && prompt;
    // runs: clean up to the span (or to the end), donor, clean behind it, the cell's rows
    const int lo[4] = {v0, max(v0, a.span_lo), max(v0, a.span_hi), a.Tp + g0};
    const int hi[4] = {!prompt ? v0 : (cut ? a.span_lo : a.Tp), cut && !a.zero_donor ? a.span_hi : 0, cut ? a.Tp : 0, a.Tp + rows};
    w.table[0] = w.table[2] = a.clean;
    w.table[1] = a.donor;
    w.table[3] = table;
    w.shift = a.Tp;
    w.first[0] = 0;
    static_for<0, 4>([&](auto s) {
        const int off = s == 3 ? a.Tp : 0, n = hi[s] > lo[s] ? (hi[s] - 1 - off) / kPageRows - (lo[s] - off) / kPageRows + 1 : 0;
        w.lo[s] = lo[s];
        w.hi[s] = hi[s];
        w.page0[s] = (lo[s] - off) / kPageRows;
        w.first[s + 1] = w.first[s] + n;
    });
    w.n = w.first[4];
    return w;
}

// Keys of the ZERO donor that a row sees.
__device__ __forceinline__ int zeros_of(const PageCall &a, bool spliced, int low) {
    return spliced && a.zero_donor ? max(0, a.span_hi - max(a.span_lo, low)) : 0;
}

template <int D, int OWN, bool SHARED>
struct PageMode {
    static constexpr int WR = D <= 128 ? 2 : 1;   // row sets of a wave in wide tiles
    static constexpr bool kWide = OWN == 0 || SHARED;
    static constexpr int NR = OWN ? OWN : 1;
    union Memory {
        NarrowShared<D, NR> narrow;
        WideShared<D> wide;
    };
    static constexpr size_t kBytes = OWN == 0 ? sizeof(WideShared<D>) : (SHARED ? sizeof(Memory) : sizeof(NarrowShared<D, NR>));
};

template <int D, int OWN, bool SHARED>
__global__ __launch_bounds__(kThreads, 2) void page_attn_kernel(PageArgs args) {
    using Mode = PageMode<D, OWN, SHARED>;
    constexpr int WR = Mode::WR;
    __shared__ __attribute__((aligned(16))) char s_mem[Mode::kBytes];
    const PageCall &a = args.call;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15;
    int x = blockIdx.x;
    const int h = x % a.Hkv;
    x /= a.Hkv;
    const int Hq = a.Hkv * a.G, ahead = a.window > 0 ? a.window - 1 : 0;
    auto low_of = [&](int pos) { return a.window > 0 ? pos - ahead : 0; };
    if constexpr (SHARED) {
        const int n_prompt = (a.tiles_u + a.tiles_s) * a.prompt_parts;
        if (x < n_prompt) {
            // rows of any cells: cells' numbers of rows before this one, in LDS
            const int part = x % a.prompt_parts, tile = x / a.prompt_parts;
            const bool spliced = tile >= a.tiles_u;
            int *s_sum = reinterpret_cast<int *>(s_mem), *s_low = s_sum + SPLICE_MAX_CELLS;
            const int tid = threadIdx.x;
            int mine = 0;
            if (tid < a.n_active) {
                const int count = (int)(args.count_split[tid] & 0xffffu), split = (int)(args.count_split[tid] >> 16);
                mine = (spliced ? count - split : split) * a.G;
            }
            int sum = mine;
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(sum, o);
                if (lane >= o) sum += y;
            }
            if (lane == 63) s_low[wave] = sum;
            __syncthreads();
            for (int w = 0; w < wave; ++w) sum += s_low[w];
            s_sum[tid] = sum;            // rows of cells 0 .. tid
            __syncthreads();
            const int total = s_sum[a.n_active - 1];
            PageRowsOf<WR> rows;
            int low = 0x7fffffff;
            static_for<0, WR>([&](auto r) {
                const int want = (spliced ? tile - a.tiles_u : tile) * (64 * WR) + (wave * WR + r) * 16 + col;
                const int row = min(want, total - 1);
                int ci = 0;
                for (int step = SPLICE_MAX_CELLS / 2; step > 0; step >>= 1)
                    if (ci + step <= a.n_active - 1 && s_sum[ci + step - 1] <= row) ci += step;
                const int in = row - (ci ? s_sum[ci - 1] : 0), split = (int)(args.count_split[ci] >> 16);
                const int t = in / a.G + (spliced ? split : 0), g = in % a.G, pos = a.Tp + (int)args.step[ci] + t;
                rows.at[r] = want < total ? ((int64_t)(args.cell_tile[ci] >> 24) * a.T + t) * Hq + h * a.G + g : -1;
                rows.lo[r] = low_of(pos);
                rows.hi[r] = pos + 1;
                rows.zeros[r] = zeros_of(a, spliced, rows.lo[r]);
                low = min(low, rows.lo[r]);
            });
            low = wave_min(low);
            if (lane == 0) s_low[4 + wave] = low;
            __syncthreads();
            low = min(min(s_low[4], s_low[5]), min(s_low[6], s_low[7]));
            low = __builtin_amdgcn_readfirstlane(low);
            __syncthreads();
            const PageWalk walk = walk_of(a, true, spliced, low, nullptr, 0);
            const int i0 = min(part * a.prompt_per, walk.n), i1 = part == a.prompt_parts - 1 ? walk.n : min(i0 + a.prompt_per, walk.n);
            wide<D, WR>(a, walk, i0, i1, h, rows, part == 0, part, *reinterpret_cast<WideShared<D> *>(s_mem));
            return;
        }
        x -= n_prompt;
    }
    // rows of one cell
    const int part = x % a.own_parts, tile = x / a.own_parts;
    int ci = 0;
    if (a.own_each > 0) ci = tile / a.own_each;
    else
        for (int step = SPLICE_MAX_CELLS / 2; step > 0; step >>= 1)
            if (ci + step < a.n_active && (int)(args.cell_tile[ci + step] & 0xffffffu) <= tile) ci += step;
    const int count = (int)(args.count_split[ci] & 0xffffu), s0 = (int)args.step[ci], cell = (int)(args.cell_tile[ci] >> 24);
    const int split = a.shared ? count : (int)(args.count_split[ci] >> 16);
    const int tiles_u = (split * a.G + a.own_rows - 1) / a.own_rows, all = tiles_u + ((count - split) * a.G + a.own_rows - 1) / a.own_rows;
    const int in = all - 1 - (tile - (int)(args.cell_tile[ci] & 0xffffffu));   // the longest lists first
    const bool spliced = in >= tiles_u;
    const int per = a.own_rows / a.G, t0 = spliced ? split + (in - tiles_u) * per : in * per, t1 = min(spliced ? count : split, t0 + per);
    const int low = low_of(a.Tp + s0 + t0);
    const PageWalk walk = walk_of(a, !a.shared, spliced, low, a.tables + (int64_t)cell * a.table_len, s0 + t1);
    const int i0 = min(part * a.own_per, walk.n), i1 = part == a.own_parts - 1 ? walk.n : min(i0 + a.own_per, walk.n);
    const int out_part = a.parts > 1 ? a.prompt_parts + part : -1;
    auto row = [&](int r, int64_t &at, int &lo, int &hi, int &zeros) {
        const int t = t0 + r / a.G, pos = a.Tp + s0 + min(t, t1 - 1);
        at = t < t1 ? ((int64_t)cell * a.T + t) * Hq + h * a.G + r % a.G : -1;
        lo = low_of(pos);
        hi = pos + 1;
        zeros = a.shared ? 0 : zeros_of(a, spliced, lo);
    };
    if constexpr (OWN == 0) {
        PageRowsOf<WR> rows;
        static_for<0, WR>([&](auto r) { row((wave * WR + r) * 16 + col, rows.at[r], rows.lo[r], rows.hi[r], rows.zeros[r]); });
        wide<D, WR>(a, walk, i0, i1, h, rows, part == 0, out_part, *reinterpret_cast<WideShared<D> *>(s_mem));
    } else {
        PageRowsOf<OWN> rows;
        static_for<0, OWN>([&](auto r) { row(r * 16 + col, rows.at[r], rows.lo[r], rows.hi[r], rows.zeros[r]); });
        narrow<D, OWN>(a, walk, i0, i1, h, rows, part == 0, out_part, *reinterpret_cast<NarrowShared<D, OWN> *>(s_mem));
    }
}

// Joins rows' partial results, W waves a row: blockIdx.y the cell.  A lane has four values of a row, so that a
// load of a wave takes 256 / D parts, and up to eight loads are on their way.
template <int D, int W>
__global__ __launch_bounds__(kThreads) void page_join_kernel(PageArgs args) {
    constexpr int L = D / 4, PP = 64 / L, AHEAD = 8;
    __shared__ f32x4_t s_sum[W == 1 ? 1 : kWaves][L];
    const PageCall &a = args.call;
    const int ci = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, Hq = a.Hkv * a.G, sub = lane / L, d = lane % L;
    const int row = W == 1 ? blockIdx.x * kWaves + wave : blockIdx.x, w0 = W == 1 ? 0 : wave;
    if (row >= (int)(args.count_split[ci] & 0xffffu) * Hq) return;
    const int64_t at = (int64_t)(args.cell_tile[ci] >> 24) * a.T * Hq + row;
    const int64_t records = (int64_t)a.C * a.T * Hq * D;
    float m = kLowest, l = 0.f;
    if (lane < a.parts) {
        const float2 rec = reinterpret_cast<const float2 *>(a.part + lane * a.part_stride + records)[at];
        m = rec.x;
        l = rec.y;
    }
    float top = l == 0.f ? kLowest : m;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float w = l == 0.f ? 0.f : fast_exp2(m - top);
    float sum = l * w;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    // (the whole wave goes round as often: a lane that had left would have no weight to give)
    for (int first = w0 * PP; first < a.parts; first += AHEAD * W * PP) {
        const int p0 = first + sub;
        f32x4_t y[AHEAD];
        static_for<0, AHEAD>([&](auto k) {
            const int p = min(p0 + k * (W * PP), a.parts - 1);
            y[k] = reinterpret_cast<const f32x4_t *>(a.part + p * a.part_stride + at * D)[d];
        });
        static_for<0, AHEAD>([&](auto k) {
            const int p = p0 + k * (W * PP);
            const float f = __shfl(w, p & 63);
            if (p < a.parts && f != 0.f) o += f * y[k];   // a part that saw nothing has no values
        });
    }
    static_for<0, 4>([&](auto i) {
#pragma unroll
        for (int x = L; x < 64; x <<= 1) o[(int)i] += __shfl_xor(o[(int)i], x);
    });
    if constexpr (W > 1) {
        if (lane < L) s_sum[wave][d] = o;
        __syncthreads();
        o = s_sum[0][d] + s_sum[1][d] + s_sum[2][d] + s_sum[3][d];
    }
    if (w0 > 0 || lane >= L) return;
    const float by = inverse(sum);
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4_t *>(a.out + at * D + 4 * d) = __builtin_convertvector(o * by, bf16x4_t);
    if (lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

template <int D>
bool launch_page_attn(const PageArgs &args, const splice::PagePlan &p, int most_count, hipStream_t stream) {
    const dim3 grid((unsigned)p.blocks), block(kThreads);
    auto go = [&](auto own, auto shared) {
        hipLaunchKernelGGL((page_attn_kernel<D, decltype(own)::value, decltype(shared)::value>), grid, block, 0, stream, args);
    };
    auto pick = [&](auto own) {
        if (p.shared) go(own, std::true_type{});
        else go(own, std::false_type{});
    };
    if (p.own == 0) go(std::integral_constant<int, 0>{}, std::false_type{});   // such tiles are not shared
    else if (D <= 128 && p.own == 2) pick(std::integral_constant<int, D <= 128 ? 2 : 1>{});
    else pick(std::integral_constant<int, 1>{});
    if (hipGetLastError() != hipSuccess) return false;
    if (p.parts == 1) return true;
    // four waves a row where the rows alone do not fill the GPU (32 rows of 64 parts: one wave each, one load at a time 19.6 us)
    const int64_t rows = (int64_t)most_count * args.call.Hkv * args.call.G;
    const bool few = rows * args.call.n_active <= 1024;
    const dim3 join((unsigned)(few ? rows : (rows + kWaves - 1) / kWaves), (unsigned)args.call.n_active);
    if (few) hipLaunchKernelGGL((page_join_kernel<D, kWaves>), join, block, 0, stream, args);
    else hipLaunchKernelGGL((page_join_kernel<D, 1>), join, block, 0, stream, args);
    return hipGetLastError() == hipSuccess;
}

bool launch_page_attn_d64(const PageArgs &, const splice::PagePlan &, int, hipStream_t);
bool launch_page_attn_d128(const PageArgs &, const splice::PagePlan &, int, hipStream_t);
bool launch_page_attn_d256(const PageArgs &, const splice::PagePlan &, int, hipStream_t);

}  // namespace splice_dev
