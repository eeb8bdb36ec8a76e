// tree_attn.hpp -- attention of a tree of drafted nodes per cell over the
// cell's spliced prompt, its generated rows and the tree's own rows
// (splice_tree_attn): out = sum_j 2^(s_j - m) v_j / l with s_j = scale log2(e) q.k_j
// over the keys j that a node sees, l = sum_j 2^(s_j - m), in one pass with
// a running m.
//
// The queries of a (cell, KV head) are its T * G (node, head) rows.  A work
// group takes 32 RW of them (RW waves of 32 rows; the other 4 / RW waves of a
// row take other keys) over a chunk of the cell's list of keys, which it walks
// tile by tile.  Per wave and 32 keys
//   S^T = K Q^T   v_mfma_f32_32x32x16_bf16, A = K from LDS, B = Q^T: lane (half
//                 h, r) gets row r's scores of the keys 8 b + 4 h + i, so a
//                 row's statistics take one exchange between the halves, and
//                 that only where its maximum rises by more than kSlack;
//   softmax       sums in fp32;
//   O^T += V^T P  A = V^T by transposing LDS reads, in the order of keys in
//                 which P lies in the lanes; P rounded to bf16, the type of V: a
//                 weight is off by 2^-8 of itself at most, a result by 2^-8
//                 sum p |v| (12 nodes a cell, window 1024, D = 256, against 64
//                 bits: 2.3e-3 of the results' size, of which rounding the
//                 result alone makes 1.7e-3).  The weights' sum is not rounded.
// RW = 1: every wave has a tile of its own, with the next one (of 8-bit rows the
// next two) in registers, and waits for no other; else a tile is for all waves, and bf16 rows go straight
// to one of two buffers in LDS while the other is computed.
//
// The list has up to five segments (prompt before, in and behind the span, each
// span form that the work group's rows need, the generated rows with the
// tree's behind them); only tiles that some row does not see wholly are masked.
// It is walked as if all values were finite, and again, with the values of those
// tiles looked at, where a result is not (0 * inf is no 0).
//
// Packed calls: the prompt is the same for all cells, so work groups of 128
// rows of any cells walk chunks of it, and the cells' generated rows have work groups
// of their own.  Chunks' results go to memory in 16 bits and tree_join_kernel joins them.
//
// What bounds it: where many rows share keys the tile loop, whose matrix products
// (40% busy) and vector operations (45%) overlap in part only: 47 cells of 16 nodes, 32 heads of
// 128 over 8k slots 137 us in the kernel (780 TFLOP/s); with small trees the generated
// rows' bytes, 64 cells of 5 nodes, 4.4 TB/s of bf16 rows and 3.3 TB/s of 8-bit ones, 5.3 and 4.5
// over longer lists (4.2 with one 8-bit tile in flight a wave; with half the bytes a key the
// chain from codes through LDS to the products counts for more); in small calls
// the chain of loads before the first tile (7.1 us with one tile).
#pragma once

#include <atomic>

#include "kv_format.hpp"
#include "tree_plan.hpp"
#include "prompt_wide.hpp"

namespace splice_dev {

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

struct TreeCall {
    const char *q, *ck, *cv, *dk, *dv, *gk, *gv;
    const uint8_t *gke, *gve;
    const int32_t *depth;
    const uint64_t *visible;
    __bf16 *out;
    float *lse;
    // Partial results, [slot][node][q head]: o / l (a convex combination of
    // value rows) in fp16, times a power of two sc that brings a row's
    // largest value to 2^14 .. 2^15, and m, l, 1 / sc.  A rounding of 2^-11 of
    // a value is small beside the bf16 result's 2^-8, and 32 bits would be 1.9 times the
    // bytes that a call of many chunks writes and reads again.
    _Float16 *part;
    float4 *record;
    int T, G, lgG, Hkv, Tp, cap, span_lo, span_hi, window, zero_donor, n_active, row_tiles, per;
    int n_p, p_tiles, p_heavy0, p_heavy;   // packed calls: chunks of the prompt, tiles of 128 rows, those that may walk
                                           // the span twice (first, number); else 0
    bool split;
    float qk_scale;   // scale * log2(e)
};
struct TreeArgs {
    TreeCall call;
    int32_t step[SPLICE_MAX_CELLS];   // of the active cells
    splice::TreeSlots slots;
};

// Where a work group is in its list of keys: the segment (0 the prompt before the span, or all
// of it; 1 the span, clean; 2 the span from the donor; 3 the prompt behind it; 4
// the generated rows with the tree's behind them), the rows left of it, the next tile's rows and
// first key (a prompt position, or in segment 4 a generated row).
struct TreeSegment {
    const char *k, *v;
    int key0, len;
};
struct TreeWalk {
    const char *k, *v;
    int seg, rem, key0;
};
struct TreeTileRef {
    int seg, key0, n;
    bool edge;     // some row's view begins or ends in it, or it is not full
    bool other;    // the span's form of nodes on one side of the onset, in a list with nodes on both
    bool dead;     // it holds rows of nodes that are not there
    bool differ;   // some row does not see some key of it
};

template <int D, int RW, bool F8>
struct TreeTile {
    static constexpr bool OWN = RW == 1;                       // every wave has tiles of its own
    static constexpr int KW = 4 / RW;                          // waves over keys
    static constexpr int KB = splice::tree_key_blocks(D, RW);  // 32-key blocks of a wave
    static constexpr int TK = splice::tree_tile_keys(D, RW);   // keys of a tile
    static constexpr int ROW = 2 * D;                          // bytes of a staged row
    static constexpr int CPR = D / 8;                          // 16-byte chunks of a row
    static constexpr int TILE = TK * ROW;                      // bytes of a K (or V) tile
    // Buffers of tiles for all waves: two, or one where two would leave room for a single work group on a compute unit (D =
    // 256, tiles of 64 keys; two groups then cover each other's loads. 8-bit rows in flight take the registers that a
    // second group would need)
    static constexpr int NBUF = OWN || (D > 128 && RW == 2 && !F8) ? 1 : 2;
    static constexpr int TILES = (OWN ? 4 : NBUF) * 2 * TILE;  // K and V: a tile a wave, or NBUF for all
    static constexpr int LDS = TILES + (OWN ? 32 * ROW : 0);   // ... and Q, for which a wave with a tile in
                                                               // registers has none left
    static constexpr int NT = OWN ? 64 : 256;                  // threads that load a tile
    static constexpr int NL = TK * CPR / NT;                   // chunks a thread loads of a K (or V) tile
    static constexpr int NL8 = NL / 2;                         // ... of 8-bit rows
    static constexpr int NR = OWN ? NL : NL8;                  // ... by way of registers
    static constexpr bool DEEP = OWN && F8;                    // two 8-bit tiles fit the registers of a bf16 one
    static constexpr int NE = OWN ? 2 : NL8;                   // exponents a thread holds: of a key of each tile, or a chunk
    static constexpr int EARLY = !OWN && D <= 128 ? 2 : 0;     // 16-key steps whose values are read before the softmax
    static constexpr int ND = D / 32;                          // 32-wide d blocks of the output
    static constexpr int PARTS = KW > 1 && KW * 32 * RW * D * 4 > TILES ? 2 : 1;   // in which the waves' results are joined
    static_assert(RW * KW == 4 && NL8 >= 1 && (KW == 1 || KW * 32 * RW * D * 4 <= TILES * PARTS), "");
};

// Chunk-slot swizzles (XOR on the 16-byte chunk index) of key r: the 16 rows
// that a quarter-wave reads of K, and the four rows that a 16-lane group reads
// 32 bytes each of V, fall into different banks.
template <int D>
__device__ __forceinline__ constexpr int tree_swz_k(int r) { return D == 64 ? (r >> 1) & 7 : r & 15; }
template <int D>
__device__ __forceinline__ constexpr int tree_swz_v(int r) { return D == 64 ? ((r >> 1) & 1) * 5 : (r & 3) << 2 | (r & 1); }

// ... and chunks 8 to 15 of every 16 in pairs the other way round, so that the
// eight lanes that store every second chunk of an 8-bit row meet every bank.
__device__ __forceinline__ constexpr int tree_pair(int chunk) { return chunk ^ ((chunk >> 3) & 1); }

// Bits [b, e) of a word, for any b and e.
__device__ __forceinline__ uint64_t bits(int b, int e) {
    b = max(b, 0);
    e = min(e, 64);
    if (e <= b) return 0;
    return (e - b == 64 ? ~0ull : (1ull << (e - b)) - 1) << b;
}
__device__ __forceinline__ uint64_t shifted(uint64_t x, int by) {   // left, or right when by < 0
    if (by >= 64 || by <= -64) return 0;
    return by >= 0 ? x << by : x >> -by;
}

// |x|, 0 for an infinity or NaN; and the power of two, 2^60 at most, that
// brings a largest value to 2^14 .. 2^15.
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
__device__ __forceinline__ float half_scale(float top) {
    return __uint_as_float((uint32_t)min(127 + 14 + 127 - (int)(__float_as_uint(top) >> 23), 127 + 60) << 23);
}

// A pointer that is the same in every lane, in scalar registers (a buffer
// descriptor from vector registers costs a loop a load).
__device__ __forceinline__ const char *uniform(const char *p) {
    const uint64_t x = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32));
    return reinterpret_cast<const char *>(((uint64_t)hi << 32) | lo);
}

// Which words of two bf16 values hold an infinity or NaN.
__device__ __forceinline__ bool has_non_finite(u32x4_t w) {
    bool bad = false;
    static_for<0, 4>([&](auto i) {
        bad |= (w[(int)i] & 0x7f80u) == 0x7f80u || (w[(int)i] & 0x7f800000u) == 0x7f800000u;
    });
    return bad;
}

// 1.0 where a value is +inf or NaN (above) or -inf or NaN (under), else 0.
__device__ __forceinline__ void find_non_finite(u32x4_t w, u32x4_t &above, u32x4_t &under) {
    static_for<0, 4>([&](auto i) {
        uint32_t up = 0, down = 0;
        static_for<0, 2>([&](auto h) {
            const uint32_t x = (w[(int)i] >> (16 * h)) & 0xffffu;
            const bool bad = (x & 0x7f80u) == 0x7f80u, nan = bad && (x & 0x7fu);
            up |= (bad && (nan || !(x >> 15)) ? 0x3f80u : 0u) << (16 * h);
            down |= (bad && (nan || (x >> 15)) ? 0x3f80u : 0u) << (16 * h);
        });
        above[(int)i] = up;
        under[(int)i] = down;
    });
}

// The words with 0 for every infinity and NaN.
__device__ __forceinline__ u32x4_t finite_only(u32x4_t w) {
    static_for<0, 4>([&](auto i) {
        uint32_t x = w[(int)i];
        if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
        if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
        w[(int)i] = x;
    });
    return w;
}

// One work group's item.  PACKED: 128 rows of any cells of a KV head over a chunk of
// the prompt; otherwise rows of one cell over a chunk of its list, which in a
// packed call is that of its generated rows.
template <int D, int RW, bool F8, bool PACKED>
__device__ __forceinline__ void tree_item(const TreeArgs &args, int rest) {
    using X = TreeTile<D, RW, F8>;
    constexpr int KW = X::KW, KB = X::KB, TK = X::TK, ND = X::ND, NST = D / 16;
    extern __shared__ __align__(16) char lds[];
    __shared__ int s_bad, s_again;
    __shared__ TreeSegment s_seg[5];
    __shared__ int s_rows[PACKED ? 4 : 1][4];
    __shared__ float s_ml[KW > 1 ? KW : 1][32 * RW][3];
    const TreeCall a = args.call;   // what the lambdas use: captured, the whole arguments would go to memory
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 31, h = lane >> 5, rw = wave % RW, kw = wave / RW;

    // ---- which rows: KV heads run fastest (blockIdx.x), so that with eight (or a multiple) an XCD keeps to its own.
    // What a division takes counts here: a work group may have few tiles
    const int g = blockIdx.x, rows = a.T << a.lgG, G1 = a.G - 1;
    int row0, row, chunk, slot, step = 0, node, depth, low, low_all, low_max;
    int64_t node0, pair = 0;
    bool last_chunk = false, valid, spliced, any_clean, any_donor;
    uint64_t alive = 0, word = 0;
    if constexpr (PACKED) {
        // tiles that walk both forms of the span come first: begun late, they would end long after the others
        const int heavy = a.p_heavy * a.n_p;
        const bool first = rest < heavy;
        const int of = first ? rest : rest - heavy, among = first ? a.p_heavy : a.p_tiles - a.p_heavy;
        chunk = of / among;
        row0 = 0;
        int rt = of - chunk * among;
        if (first) rt += a.p_heavy0;
        else if (rt >= a.p_heavy0) rt += a.p_heavy;
        const int at = 32 * RW * rt + 32 * rw + r, n_rows = a.n_active * rows;
        const int ci = min(at, n_rows - 1) / rows;
        row = at - ci * rows;
        const uint32_t info = args.slots.info[ci];
        const int at_step = args.step[ci];
        node0 = (int64_t)(info & 255) * a.T;
        slot = (int)(info >> 16) + chunk;
        node = min(row >> a.lgG, a.T - 1);
        depth = min(a.depth[node0 + node], a.T - 1);
        valid = at < n_rows && depth >= 0;
        spliced = depth >= (int)((info >> 8) & 255);
        low = a.window > 0 ? a.Tp + at_step + max(depth, 0) - a.window + 1 : 0;   // first position the row sees
        int lo = valid ? low : INT32_MAX, hi = valid ? low : INT32_MIN;
        for (int o = 32; o > 0; o >>= 1) {
            lo = min(lo, __shfl_xor(lo, o));
            hi = max(hi, __shfl_xor(hi, o));
        }
        const int clean = __any(valid && !spliced), donor = __any(valid && spliced);
        if (lane == 0) {
            s_rows[wave][0] = lo;
            s_rows[wave][1] = hi;
            s_rows[wave][2] = clean;
            s_rows[wave][3] = donor;
        }
        __syncthreads();
        static_for<0, 4>([&](auto w) {
            lo = min(lo, s_rows[w][0]);
            hi = max(hi, s_rows[w][1]);
        });
        any_clean = __builtin_amdgcn_readfirstlane(s_rows[0][2] | s_rows[1][2] | s_rows[2][2] | s_rows[3][2]) != 0;
        any_donor = __builtin_amdgcn_readfirstlane(s_rows[0][3] | s_rows[1][3] | s_rows[2][3] | s_rows[3][3]) != 0;
        if (!any_clean && !any_donor) return;
        low_all = __builtin_amdgcn_readfirstlane(max(lo, 0));   // some row sees from here on,
        low_max = __builtin_amdgcn_readfirstlane(hi);           // every row from here on
    } else {
        const int place = a.row_tiles == 1 ? rest : rest / a.row_tiles, rt = rest - place * a.row_tiles;
        const uint32_t here = args.slots.order[place >> 1] >> (16 * (place & 1));
        const int ci = here & 255;
        chunk = (here >> 8) & 255;
        const uint32_t info = args.slots.info[ci];
        const int c = info & 255, onset = (info >> 8) & 255;
        slot = (int)(info >> 16) + a.n_p + chunk;
        step = args.step[ci];
        last_chunk = slot + 1 == (int)(args.slots.info[ci + 1] >> 16);
        row0 = 32 * RW * rt;
        row = row0 + 32 * rw + r;
        node0 = (int64_t)c * a.T;
        pair = (int64_t)c * a.Hkv + g;
        node = min(row >> a.lgG, a.T - 1);
        int d_node = lane < a.T ? a.depth[node0 + lane] : -1;   // lane u: node u's depth
        word = a.visible[node0 + node];
        d_node = min(d_node, a.T - 1);
        alive = __ballot(d_node >= 0);
        // the work group's nodes
        const uint64_t mine = bits(row0 >> a.lgG, (min(row0 + 32 * RW - 1, rows - 1) >> a.lgG) + 1) & alive;
        if (mine == 0) return;
        depth = __shfl(d_node, node);
        const int p0 = a.Tp + step;
        valid = row < rows && depth >= 0;
        spliced = depth >= onset;
        low = a.window > 0 ? p0 + max(depth, 0) - a.window + 1 : 0;
        word = valid ? word & alive : 0;
        if (a.window > 0 && a.window < a.T) {
            for (int u = 0; u < a.T; ++u)
                if (depth - __shfl(d_node, u) >= a.window) word &= ~(1ull << u);
        }
        // of the work group's nodes: the least and the largest depth, and whether spliced and unspliced ones are there
        const bool in = (mine >> lane) & 1;
        int d_min = in ? d_node : SPLICE_MAX_NODES, d_max = in ? d_node : 0;
        for (int o = 32; o > 0; o >>= 1) {
            d_min = min(d_min, __shfl_xor(d_min, o));
            d_max = max(d_max, __shfl_xor(d_max, o));
        }
        d_min = __builtin_amdgcn_readfirstlane(d_min);
        d_max = __builtin_amdgcn_readfirstlane(d_max);
        any_clean = d_min < onset;
        any_donor = d_max >= onset;
        low_all = a.window > 0 ? max(p0 + d_min - a.window + 1, 0) : 0;
        low_max = a.window > 0 ? p0 + d_max - a.window + 1 : 0;
    }

    // ---- the list of keys: segments 0 to 4, walked tile by tile
    const int b0 = min(low_all, a.Tp), sa = min(max(a.span_lo, b0), a.Tp), sb = max(a.span_hi, sa);
    const int g0 = min(max(low_all - a.Tp, 0), step);
    const size_t head_p = (size_t)g * a.Tp * X::ROW;
    const bool prompt = PACKED || a.n_p == 0;   // a packed call's prompt has items of its own
    if (tid < 5) {
        const int i = tid, row_bytes = F8 && i == 4 ? D : X::ROW;
        int begin = i == 0 ? b0 : (i == 3 ? sb : (i == 4 ? g0 : sa)), end = begin;
        if (i == 4) end = PACKED ? begin : step + a.T;
        else if (!prompt) end = begin;
        else if (i == 0) end = any_donor ? sa : a.Tp;
        else if (any_donor) end = i == 3 ? a.Tp : ((i == 1 ? any_clean : !a.zero_donor) ? sb : begin);
        const char *k = i == 4 ? a.gk + pair * a.cap * row_bytes : pick_base(i == 2, a.ck, a.dk) + head_p;
        const char *v = i == 4 ? a.gv + pair * a.cap * row_bytes : pick_base(i == 2, a.cv, a.dv) + head_p;
        s_seg[i] = TreeSegment{k + (size_t)begin * row_bytes, v + (size_t)begin * row_bytes, begin, end - begin};
    }
    if (tid == 0) s_bad = s_again = 0;
    __syncthreads();
    int n_tiles = 0;
    static_for<0, 5>([&](auto i) { n_tiles += (s_seg[i].len + TK - 1) / TK; });
    n_tiles = __builtin_amdgcn_readfirstlane(n_tiles);
    const int t0 = PACKED ? n_tiles * chunk / a.n_p : min(chunk * a.per, n_tiles);
    const int t1 = PACKED ? n_tiles * (chunk + 1) / a.n_p : (last_chunk ? n_tiles : min(t0 + a.per, n_tiles));
    TreeWalk w;
    // `skip` tiles on from the end of segment i - 1, over the segments that are shorter
    auto enter = [&](int i, int skip) {
        TreeSegment x = s_seg[i];
        while (i < 4 && skip * TK >= x.len) {
            skip -= (x.len + TK - 1) / TK;
            x = s_seg[++i];
        }
        const int row_bytes = F8 && i == 4 ? D : X::ROW;
        w.seg = __builtin_amdgcn_readfirstlane(i);
        w.k = uniform(x.k + (size_t)skip * TK * row_bytes);
        w.v = uniform(x.v + (size_t)skip * TK * row_bytes);
        w.key0 = __builtin_amdgcn_readfirstlane(x.key0 + skip * TK);
        w.rem = __builtin_amdgcn_readfirstlane(x.len - skip * TK);
    };
    // The tile under way: how many keys, which, and what has to be looked at.
    auto tile = [&](int seg, int key0, int rem) {
        TreeTileRef x;
        x.seg = seg;
        x.key0 = key0;
        x.n = min(TK, rem);
        x.other = any_clean && any_donor && (seg == 1 || seg == 2);
        const bool gen = !PACKED && seg == 4;
        x.dead = gen && key0 + TK > step && alive != bits(0, a.T);
        x.differ = x.other || (gen ? a.Tp + key0 < low_max || key0 + TK > step : key0 < low_max);
        x.edge = x.n < TK || (x.differ && !x.other) || (x.other && key0 < low_max);
        return x;
    };
    auto tile_of = [&]() { return tile(w.seg, w.key0, w.rem); };
    auto generated = [&](int key0) { return tile(4, key0, step + a.T - key0); };
    auto advance = [&]() {   // to the wave's next tile
        const int row_bytes = F8 && w.seg == 4 ? D : X::ROW;
        constexpr int N = X::OWN ? 4 : 1;
        w.k += N * TK * row_bytes;
        w.v += N * TK * row_bytes;
        w.key0 += N * TK;
        w.rem -= N * TK;
        if (w.rem <= 0 && w.seg < 4) enter(w.seg + 1, -w.rem / TK);
    };

    // ---- tiles into LDS.  A tile for all waves: bf16 rows go there straight
    // from memory (lds_dma16: a lane names 16 bytes for chunk slot 64 q + lane)
    // into the other of two buffers, 8-bit ones by way of registers, where they
    // become bf16.  Tiles of a wave's own: the next one or two wait in registers,
    // so that one buffer a wave is enough, two work groups fit a compute unit and
    // no wave waits for another.
    int ltid = X::OWN ? lane : tid;
    char *const own = lds + (X::OWN ? wave * 2 * X::TILE : 0);
    const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_offset(lds));
    int k_src[X::NL], v_src[X::NL];
    if constexpr (!X::OWN) {
        static_for<0, X::NL>([&](auto i) {
            const int u = (int)i * 256 + tid, key = u / X::CPR, slot_of = u % X::CPR;
            k_src[i] = key * X::ROW + (tree_pair(slot_of ^ tree_swz_k<D>(key)) << 4);
            v_src[i] = key * X::ROW + (tree_pair(slot_of ^ tree_swz_v<D>(key)) << 4);
        });
    }
    u32x4_t kr[X::NR], vr[X::NR];
    uint8_t ke[X::NE], ve[X::NE];   // bytes: made words where they are loaded, they would be waited for there
    constexpr std::integral_constant<int, 0> kFirst{};
    constexpr std::integral_constant<int, 1> kSecond{};
    auto load8 = [&](auto set) {   // the walk's tile of 8-bit rows; nothing behind the list's end
        const int n = __builtin_amdgcn_readfirstlane(X::DEEP ? max(min(TK, w.rem), 0) : min(TK, w.rem));
        const int64_t ex = pair * a.cap + w.key0;
        const __amdgpu_buffer_rsrc_t rk = rows_rsrc(uniform(w.k), n * D), rv = rows_rsrc(uniform(w.v), n * D);
        const __amdgpu_buffer_rsrc_t re = rows_rsrc(uniform(reinterpret_cast<const char *>(a.gke + ex)), n);
        const __amdgpu_buffer_rsrc_t rf = rows_rsrc(uniform(reinterpret_cast<const char *>(a.gve + ex)), n);
        constexpr int at = decltype(set)::value * X::NL8;
        static_for<0, X::NL8>([&](auto i) {
            const int u = (int)i * X::NT + ltid;
            kr[at + i] = row_load<0>(rk, u * 16);
            vr[at + i] = row_load<0>(rv, u * 16);
            if constexpr (!X::OWN) {
                ke[i] = __builtin_amdgcn_raw_buffer_load_b8(re, u / (D / 16), 0, 0);
                ve[i] = __builtin_amdgcn_raw_buffer_load_b8(rf, u / (D / 16), 0, 0);
            }
        });
        if constexpr (X::OWN) {
            ke[set] = __builtin_amdgcn_raw_buffer_load_b8(re, r, 0, 0);
            ve[set] = __builtin_amdgcn_raw_buffer_load_b8(rf, r, 0, 0);
        }
    };
    auto load16 = [&]() {   // ... of a wave's own
        const int n = min(TK, w.rem);
        const __amdgpu_buffer_rsrc_t rk = rows_rsrc(w.k, n * X::ROW), rv = rows_rsrc(w.v, n * X::ROW);
        static_for<0, X::NL>([&](auto i) {
            kr[i] = row_load<0>(rk, ((int)i * X::NT + ltid) * 16);
            vr[i] = row_load<0>(rv, ((int)i * X::NT + ltid) * 16);
        });
    };
    auto load = [&](int b) {   // the walk's tile
        if (F8 && w.seg == 4) {
            load8(kFirst);
        } else if constexpr (X::OWN) {
            load16();
        } else {
            const int n = min(TK, w.rem);
            const u32x4_t rk = rows_desc(w.k, n * X::ROW), rv = rows_desc(w.v, n * X::ROW);
            const uint32_t base = lds0 + b * 2 * X::TILE;
            static_for<0, X::NL>([&](auto i) {
                const uint32_t at = base + (((int)i * 4 + wave) << 10);
                lds_dma16(rk, at, k_src[i]);
                lds_dma16(rv, at + X::TILE, v_src[i]);
            });
        }
    };
    // ---- addresses of the operands within a buffer: K at k_at ^ 16 tree_pair(2 st), V at v_at ^ 16 tree_pair(4 db)
    int k_at = ((X::OWN ? 0 : kw * 32 * KB) + r) * X::ROW + ((h ^ tree_swz_k<D>(r)) << 4), v_at;
    {
        const int vrow = (X::OWN ? 0 : kw * 32 * KB) + 4 * h + ((lane & 15) >> 2);
        const int chunk_of = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        v_at = X::TILE + vrow * X::ROW + ((chunk_of ^ tree_swz_v<D>(vrow)) << 4) + 8 * (lane & 1);
    }

    // What load() left in registers, into the tile: 8-bit rows two neighbouring
    // chunks a lane.  A lane's i-th key is i * step rows behind its first, whose
    // swizzle differs by a constant: one address each of K and V, and constants.
    auto store8 = [&](char *buf, auto set) {
        constexpr int LPR = D / 16, STEP = X::NT / LPR;
        const int key = ltid / LPR, ch = 2 * (ltid % LPR);
        const int at_k = key * X::ROW + ((tree_pair(ch) ^ tree_swz_k<D>(key)) << 4);
        const int at_v = key * X::ROW + ((tree_pair(ch) ^ tree_swz_v<D>(key)) << 4);
        static_for<0, X::NL8>([&](auto i) {
            constexpr int from = decltype(set)::value * X::NL8 + i;
            const u32x4_t k = kr[from], v = vr[from];
            uint32_t ek, ev;
            if constexpr (X::OWN) {
                ek = __shfl((int)ke[set], key + i * STEP);
                ev = __shfl((int)ve[set], key + i * STEP);
            } else {
                ek = ke[i];
                ev = ve[i];
            }
            static_for<0, 2>([&](auto j) {
                constexpr int ck = (j ^ tree_swz_k<D>(i * STEP)) << 4, cv = (j ^ tree_swz_v<D>(i * STEP)) << 4;
                char *const to = buf + i * STEP * X::ROW;
                *reinterpret_cast<u32x4_t *>(to + (at_k ^ ck)) = e4m3_to_bf16(j ? make_uint2(k.z, k.w) : make_uint2(k.x, k.y), ek);
                *reinterpret_cast<u32x4_t *>(to + X::TILE + (at_v ^ cv)) =
                    e4m3_to_bf16(j ? make_uint2(v.z, v.w) : make_uint2(v.x, v.y), ev);
            });
        });
    };
    auto store16 = [&](char *buf) {
        constexpr int STEP = X::NT / X::CPR;
        const int key = ltid / X::CPR, ch = ltid % X::CPR;
        const int at_k = key * X::ROW + ((tree_pair(ch) ^ tree_swz_k<D>(key)) << 4);
        const int at_v = key * X::ROW + ((tree_pair(ch) ^ tree_swz_v<D>(key)) << 4);
        static_for<0, X::NL>([&](auto i) {
            constexpr int ck = tree_swz_k<D>(i * STEP) << 4, cv = tree_swz_v<D>(i * STEP) << 4;
            char *const to = buf + i * STEP * X::ROW;
            *reinterpret_cast<u32x4_t *>(to + (at_k ^ ck)) = kr[i];
            *reinterpret_cast<u32x4_t *>(to + X::TILE + (at_v ^ cv)) = vr[i];
        });
    };
    auto store = [&](char *buf, int seg) {
        if (F8 && seg == 4) store8(buf, kFirst);
        else if constexpr (X::OWN) store16(buf);
    };
    // Values that are looked at: those of nodes that are not there become 0, and
    // so do infinities and NaN, which must not reach the rows that do not see
    // them (0 * inf); s_bad tells that there were some, and the rows that do
    // see them are settled behind the loop.
    auto look = [&](const TreeTileRef &x, char *buf) {
        static_for<0, X::NL>([&](auto i) {
            const int u = (int)i * X::NT + ltid, key = u / X::CPR, nd = x.key0 + key - step;
            u32x4_t *p = reinterpret_cast<u32x4_t *>(buf + X::TILE + u * 16);
            const u32x4_t v = *p;
            if (!PACKED && x.seg == 4 && nd >= 0 && (nd >= 64 || !((alive >> nd) & 1))) {
                *p = u32x4_t{0, 0, 0, 0};
            } else if (has_non_finite(v)) {
                *p = finite_only(v);
                s_bad = 1;
            }
        });
    };
    // Bit k: the lane's row sees key k of the tile, from the wave's first key on.
    auto seen = [&](const TreeTileRef &x) {
        const int skip = X::OWN ? 0 : kw * 32 * KB, first = x.key0 + skip, n = x.n - skip;
        if (!PACKED && x.seg == 4)
            return bits(low - a.Tp - first, min(step - first, n)) | (shifted(word, step - first) & bits(step - first, n));
        return x.other && (x.seg == 2) != spliced ? 0 : bits(low - first, n);
    };
    auto values = [&](const char *buf, int db, int kk) {   // 32 d of 16 keys, in the lanes of the A operand
        const char *at = buf + (v_at ^ (tree_pair(4 * db) << 4)) + 16 * kk * X::ROW;
        const u32x2_t lo = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)at));
        const u32x2_t hi = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(at + 8 * X::ROW)));
        return u32x4_t{lo.x, lo.y, hi.x, hi.y};
    };
    auto product = [&](u32x4_t x, bf16x8_t p, f32x16_t acc) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), p, acc, 0, 0, 0);
    };

    const int t_first = X::OWN ? t0 + kw : t0;
    constexpr int t_step = X::OWN ? 4 : 1;
    TreeTileRef cur;
    // Two tiles of 8-bit rows: always both, so that the number of loads in flight is known where the first is waited for.
    auto two = [&]() {
        load8(kFirst);
        advance();
        __builtin_amdgcn_sched_barrier(0);   // in this order
        load8(kSecond);
        advance();
    };
    auto begin = [&]() {   // the wave's first tile
        enter(0, t_first);
        cur = tile_of();
        if (t_first >= t1) return;
        if (X::DEEP && cur.seg == 4) {
            two();
        } else {
            if constexpr (X::DEEP) load16();
            else load(0);
            advance();
        }
    };
    begin();

    // ---- Q^T, in the lanes of the B operand: row r, d = 16 st + 8 h ..
    bf16x8_t qb[X::OWN ? 1 : NST];
    char *const s_q = lds + X::TILES;   // chunk slots as those of K
    {
        const int64_t q_row = (node0 + node) * (a.Hkv * a.G) + g * a.G + (row & G1);
        if constexpr (X::OWN) {
            for (int ch = 2 * kw + h; ch < X::CPR; ch += 8) {
                u32x4_t x = {0, 0, 0, 0};
                if (valid) x = *reinterpret_cast<const u32x4_t *>(a.q + (q_row * D + 8 * ch) * 2);
                *reinterpret_cast<u32x4_t *>(s_q + r * X::ROW + ((tree_pair(ch) ^ tree_swz_k<D>(r)) << 4)) = x;
            }
            __syncthreads();
        } else {
            static_for<0, NST>([&](auto st) {
                u32x4_t x = {0, 0, 0, 0};
                if (valid) x = *reinterpret_cast<const u32x4_t *>(a.q + (q_row * D + 16 * (int)st + 8 * h) * 2);
                qb[st] = __builtin_bit_cast(bf16x8_t, x);
            });
        }
    }
    const bool wave_clean = __any(valid && !spliced), wave_donor = __any(valid && spliced);

    // The list is walked as if every value were finite. If a row's result then
    // is not, it is walked once more, and the values of every tile that
    // rows see differently are looked at.
    f32x16_t o[ND];   // o[db][i] is d = 32 db + 8 (i / 4) + 4 h + i % 4 of the row
    float m, l;       // its maximum; its sum, of which either half has a share
    for (bool careful = false;; careful = true) {
        static_for<0, ND>([&](auto db) { static_for<0, 16>([&](auto i) { o[db][(int)i] = 0.f; }); });
        m = -INFINITY;
        l = 0.f;
        // keys of the ZERO donor score 0 and add nothing to o
        if (a.zero_donor && prompt && spliced && chunk == 0 && kw == 0) {
            const int n_zero = a.span_hi - max(a.span_lo, max(low, 0));
            if (n_zero > 0) {
                m = 0.f;
                l = h == 0 ? (float)n_zero : 0.f;
            }
        }

        // the tile cur, which is in buf
        auto work = [&](char *buf) {
            if (careful ? cur.differ : cur.dead) {
                look(cur, buf);
                if constexpr (X::OWN) wave_fence();
                else __syncthreads();
            }
            // (a wave may have no row that sees its tile)
            if (!cur.other || (cur.seg == 2 ? wave_donor : wave_clean)) {
                f32x16_t s[KB];
                static_for<0, KB>([&](auto kb) {
                    u32x4_t ka[NST];
                    static_for<0, NST>([&](auto st) {
                        ka[st] = *reinterpret_cast<const u32x4_t *>(buf + (k_at ^ (tree_pair(2 * (int)st) << 4)) + (int)kb * 32 * X::ROW);
                    });
                    static_for<0, 16>([&](auto i) { s[kb][(int)i] = 0.f; });
                    static_for<0, NST>([&](auto st) {
                        bf16x8_t q;
                        if constexpr (X::OWN) q = *reinterpret_cast<const bf16x8_t *>(s_q + (k_at ^ (tree_pair(2 * (int)st) << 4)));
                        else q = qb[st];
                        s[kb] = product(ka[st], q, s[kb]);
                    });
                });
                // with registers to spare the values are on their way while the softmax runs
                u32x4_t vv[X::EARLY > 0 ? X::EARLY : 1][ND];
                if constexpr (X::EARLY > 0) {
                    static_for<0, X::EARLY>([&](auto kk) { static_for<0, ND>([&](auto db) { vv[kk][db] = values(buf, db, kk); }); });
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
                if (cur.edge || (careful && cur.other)) {
                    const uint64_t see = seen(cur) >> 4 * h;
                    static_for<0, KB>([&](auto kb) {
                        static_for<0, 16>([&](auto i) {
                            constexpr int key = 32 * kb + 8 * (i >> 2) + (i & 3);
                            if (!((see >> key) & 1)) s[kb][(int)i] = -INFINITY;
                        });
                    });
                }
                float mt = -INFINITY;
                static_for<0, KB>([&](auto kb) { static_for<0, 16>([&](auto i) { mt = fmaxf(mt, s[kb][(int)i]); }); });
                mt *= a.qk_scale;
                const bool hidden = cur.other && (cur.seg == 2) != spliced;   // the row sees none of it
                if (hidden) mt = -INFINITY;
                if (__any(mt > m + kSlack)) {
                    mt = fmaxf(mt, __shfl_xor(mt, 32));
                    const bool need = mt > m + kSlack;
                    const float mn = need ? mt : m;
                    const float al = need ? fast_exp2(m - mn) : 1.f;
                    l *= al;
                    static_for<0, ND>([&](auto db) { o[db] *= al; });
                    m = mn;
                }
                const float ms = hidden ? INFINITY : (m == -INFINITY ? 0.f : m);
                bf16x8_t pb[2 * KB];
                static_for<0, KB>([&](auto kb) {
                    static_for<0, 16>([&](auto i) {
                        const float p = fast_exp2(fmaf(s[kb][(int)i], a.qk_scale, -ms));
                        l += p;
                        pb[2 * kb + i / 8][i % 8] = (__bf16)p;
                    });
                });
                static_for<0, 2 * KB>([&](auto kk) {
                    static_for<0, ND>([&](auto db) {
                        if constexpr (kk < X::EARLY) o[db] = product(vv[kk][db], pb[kk], o[db]);
                        else o[db] = product(values(buf, db, kk), pb[kk], o[db]);
                    });
                });
            }
        };
        if constexpr (!X::OWN && X::NBUF == 2) {
            wait_vmcnt<0>();   // this wave's part of the first tile
            if (t_first < t1) store(own, cur.seg);
        }
        int t = t_first;
        for (; !X::DEEP && t < t1; t += t_step) {
            const int b = X::NBUF == 1 ? 0 : (t - t0) & 1;
            char *const buf = own + b * 2 * X::TILE;
            // addresses are worked out anew for every tile: kept, they would take the registers of the tile in flight
            asm volatile("" : "+v"(ltid), "+v"(k_at), "+v"(v_at));
            if constexpr (X::OWN) {
                wave_fence();   // the wave has read the tile before
                store(buf, cur.seg);
                wave_fence();
            } else if constexpr (X::NBUF == 1) {
                wait_vmcnt<0>();
                store(buf, cur.seg);
                __syncthreads();
            } else {
                __syncthreads();   // every wave's part of tile t is in LDS, and tile t - 1 has been read
            }
            const TreeTileRef next = tile_of();
            // the matrix products of one wave go before the softmax of another on its SIMD
            __builtin_amdgcn_s_setprio(1);
            if (t + t_step < t1 && (X::OWN || X::NBUF == 2)) {
                load(b ^ 1);
                advance();
            }
            work(buf);
            cur = next;
            if constexpr (!X::OWN && X::NBUF == 1) {
                __syncthreads();   // tile t has been read
                if (t + 1 < t1) {
                    cur = tile_of();
                    load(0);
                    advance();
                }
            } else if constexpr (!X::OWN) {
                wait_vmcnt<0>();
                if (t + 1 < t1) store(own + (b ^ 1) * 2 * X::TILE, cur.seg);
            }
        }
        if constexpr (X::DEEP) {
            // the prompt's tiles
            bool turn = false;
            if (t < t1 && cur.seg != 4) {
                TreeTileRef next;
                for (;; t += t_step) {
                    asm volatile("" : "+v"(ltid), "+v"(k_at), "+v"(v_at));
                    wave_fence();
                    store16(own);
                    wave_fence();
                    next = tile_of();
                    __builtin_amdgcn_s_setprio(1);
                    turn = t + t_step < t1 && next.seg == 4;
                    if (turn) break;
                    const bool more = t + t_step < t1;
                    if (more) {
                        load16();
                        advance();
                    }
                    work(own);
                    cur = next;
                    if (!more) break;
                }
                if (turn) {
                    two();
                    work(own);
                    cur = next;
                } else {
                    wait_vmcnt<0>();
                }
                t += t_step;
            }
            // the generated rows, to the list's end: two tiles are in registers, the third is asked for as the first goes to LDS
            // (a pair of steps without a way out between them, on which loads in flight would be taken to be others)
            auto step_of = [&](auto set) {
                const bool on = decltype(set)::value == 0 || t < t1;
                asm volatile("" : "+v"(ltid), "+v"(k_at), "+v"(v_at));
                if (on) {
                    wave_fence();
                    store8(own, set);
                    wave_fence();
                }
                __builtin_amdgcn_s_setprio(1);
                load8(set);
                advance();
                if (on) work(own);
                t += t_step;
                cur = generated(cur.key0 + t_step * TK);
            };
            while (t < t1) {
                step_of(kFirst);
                step_of(kSecond);
            }
            wait_vmcnt<0>();   // what was asked for behind the end: else a walk that follows would seem to have it in flight
        }
        __syncthreads();
        if (careful) break;
        float zero = 0.f * l;   // NaN if anything is not finite
        static_for<0, ND>([&](auto db) { static_for<0, 16>([&](auto i) { zero = fmaf(0.f, o[db][(int)i], zero); }); });
        if (valid && zero != zero) s_again = 1;
        __syncthreads();
        if (!s_again) break;
        begin();
    }
    if (s_bad) {
        // infinities and NaN among the values of tiles that rows see differently:
        // the tiles once more, and which of them each row sees
        enter(0, t_first);
        for (int t = t_first; t < t1; t += t_step) {
            const TreeTileRef x = tile_of();
            if (x.differ) {
                if constexpr (!X::OWN) __syncthreads();
                load(0);
                wait_vmcnt<0>();
                if constexpr (X::OWN) wave_fence();
                store(own, x.seg);
                if constexpr (X::OWN) wave_fence();
                else __syncthreads();
                const uint64_t see = seen(x) >> 4 * h;
                bf16x8_t on[2 * KB];
                static_for<0, 32 * KB / 2>([&](auto i) {
                    constexpr int key = 32 * (i / 16) + 8 * ((i % 16) >> 2) + (i & 3);
                    on[i / 8][i % 8] = (__bf16)((see >> key) & 1 ? 1.f : 0.f);
                });
                static_for<0, ND>([&](auto db) {
                    f32x16_t up, down;
                    static_for<0, 16>([&](auto i) { up[(int)i] = down[(int)i] = 0.f; });
                    static_for<0, 2 * KB>([&](auto kk) {
                        u32x4_t above, under;
                        find_non_finite(values(own, db, kk), above, under);
                        up = product(above, on[kk], up);
                        down = product(under, on[kk], down);
                    });
                    static_for<0, 16>([&](auto i) {
                        if (up[(int)i] > 0.f) o[db][(int)i] += INFINITY;
                        if (down[(int)i] > 0.f) o[db][(int)i] -= INFINITY;
                    });
                });
            }
            advance();
        }
        __syncthreads();
    }

    // ---- results
    l += __shfl_xor(l, 32);
    const int64_t out_row = (node0 + node) * (a.Hkv * a.G) + g * a.G + (row & G1);
    const int64_t part_row = ((int64_t)slot * a.T + node) * (a.Hkv * a.G) + g * a.G + (row & G1);
    if constexpr (KW > 1) {
        // the waves of a row through LDS (every wave is done with the tiles)
        constexpr int DP = D / X::PARTS;               // values of a row at once
        float *s_o = reinterpret_cast<float *>(lds);   // [KW][32 RW][DP], chunks of four swizzled by the row
        const int wrow = 32 * rw + r;
        float top = 0.f;   // the joined row's values are between the waves': none is larger
        static_for<0, ND>([&](auto db) { static_for<0, 16>([&](auto i) { top = fmaxf(top, finite_size(o[db][(int)i])); }); });
        top = fmaxf(top, __shfl_xor(top, 32));
        if (h == 0) {
            s_ml[kw][wrow][0] = m;
            s_ml[kw][wrow][1] = l;
            s_ml[kw][wrow][2] = l == 0.f ? 0.f : finite_size(top / l);
        }
        static_for<0, X::PARTS>([&](auto part) {
            if (part > 0) __syncthreads();
            static_for<0, ND / X::PARTS>([&](auto e) {
                constexpr int db = part * (ND / X::PARTS) + e;
                static_for<0, 4>([&](auto i) {
                    const int d4 = 8 * (int)e + 2 * (int)i + h;
                    *reinterpret_cast<f32x4_t *>(s_o + ((kw * 32 * RW + wrow) * DP + 4 * (d4 ^ (wrow & 15)))) =
                        f32x4_t{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
                });
            });
            __syncthreads();
            for (int e = tid; e < 32 * RW * (DP / 4); e += 256) {
                const int w = e / (DP / 4), d4 = e % (DP / 4), rr = row0 + w, d = (int)part * DP + 4 * d4;
                if (rr >= rows) break;
                const int nd = rr >> a.lgG, hd = g * a.G + (rr & G1);
                if (!((alive >> nd) & 1)) continue;
                float M = -INFINITY, Lsum = 0.f, size = 0.f;
                static_for<0, KW>([&](auto k) {
                    M = fmaxf(M, s_ml[k][w][0]);
                    size = fmaxf(size, s_ml[k][w][2]);
                });
                const float Ms = M == -INFINITY ? 0.f : M;
                f32x4_t O = {0.f, 0.f, 0.f, 0.f};
                static_for<0, KW>([&](auto k) {
                    const float f = fast_exp2(s_ml[k][w][0] - Ms);
                    Lsum = fmaf(f, s_ml[k][w][1], Lsum);
                    if (f != 0.f)
                        O += f * *reinterpret_cast<const f32x4_t *>(s_o + (((int)k * 32 * RW + w) * DP + 4 * (d4 ^ (w & 15))));
                });
                const float f = Lsum == 0.f ? 0.f : 1.f / Lsum;
                O *= f;
                if (a.split) {
                    const int64_t at = ((int64_t)slot * a.T + nd) * (a.Hkv * a.G) + hd;
                    const float sc = half_scale(size);
                    *reinterpret_cast<f16x4_t *>(a.part + at * D + d) = __builtin_convertvector(O * sc, f16x4_t);
                    if (d == 0) a.record[at] = make_float4(M, Lsum, 1.f / sc, 0.f);
                } else {
                    const int64_t at = (node0 + nd) * (a.Hkv * a.G) + hd;
                    *reinterpret_cast<bf16x4_t *>(a.out + at * D + d) = __builtin_convertvector(O, bf16x4_t);
                    if (d == 0) a.lse[at] = kLn2 * (M + log2f(Lsum));
                }
            }
        });
    } else {
        const float f = l == 0.f ? 0.f : 1.f / l;
        float top = 0.f;
        static_for<0, ND>([&](auto db) {
            static_for<0, 16>([&](auto i) {
                o[db][(int)i] *= f;
                top = fmaxf(top, finite_size(o[db][(int)i]));
            });
        });
        const float sc = half_scale(fmaxf(top, __shfl_xor(top, 32)));
        if (!valid) return;
        static_for<0, ND>([&](auto db) {
            static_for<0, 4>([&](auto i) {
                const f32x4_t v = {o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
                const int d = 32 * (int)db + 8 * (int)i + 4 * h;
                if (PACKED || a.split) *reinterpret_cast<f16x4_t *>(a.part + part_row * D + d) = __builtin_convertvector(v * sc, f16x4_t);
                else *reinterpret_cast<bf16x4_t *>(a.out + out_row * D + d) = __builtin_convertvector(v, bf16x4_t);
            });
        });
        if (h == 0) {
            if (PACKED || a.split) a.record[part_row] = make_float4(m, l, 1.f / sc, 0.f);
            else a.lse[out_row] = kLn2 * (m + log2f(l));
        }
    }
}

template <int D, int RW, bool F8>
__global__ __launch_bounds__(256, splice::tree_resident(D, F8)) void tree_kernel(TreeArgs args) {
    tree_item<D, RW, F8, false>(args, (int)blockIdx.y);
}

// Items of the prompt, then items of the generated rows.
template <int D, int RW, bool F8>
__global__ __launch_bounds__(256, splice::tree_resident(D, F8)) void tree_packed_kernel(TreeArgs args) {
    const int n = args.call.p_tiles * args.call.n_p;
    if ((int)blockIdx.y < n) tree_item<D, 4, false, true>(args, (int)blockIdx.y);
    else tree_item<D, RW, F8, false>(args, (int)blockIdx.y - n);
}

// Joins the chunks of every row (blockIdx.x the active cell and node).  D / 8
// lanes read a chunk's values.  MANY: a wave a row, whose lanes read a chunk's
// record each, and 64 / (D / 8) chunks at once; otherwise, with at most D / 8
// and at most 8 chunks, 64 / (D / 8) rows a wave (64 cells of 16 nodes, 2 chunks:
// a call of 131 us; with a wave a row 138).  Bound by the chunks' bytes: 10 us for
// 48 cells of 16 nodes, 32 heads, 7 chunks (4.5 TB/s), else by launch and one round of loads, 4.5.
template <int D, bool MANY>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs args) {
    constexpr int LPR = D / 8, SP = 64 / LPR, GROUP = MANY ? 64 : LPR;
    static_assert(splice::kTreeMaxChunks == 64 && LPR >= 8, "a chunk a lane");
    const TreeCall a = args.call;
    const int Hq = a.Hkv * a.G, ci = blockIdx.x / a.T, node = blockIdx.x % a.T;
    const uint32_t info = args.slots.info[ci];
    const int64_t at_node = (int64_t)(info & 255) * a.T + node;
    const int lane = threadIdx.x & 63, wave = blockIdx.y * 4 + (threadIdx.x >> 6), sp = lane / LPR, l = lane % LPR;
    const int hd = MANY ? wave : wave * SP + sp, head = min(hd, Hq - 1);   // rows behind the last are the last again
    const int first = (int)(info >> 16), n = (int)(args.slots.info[ci + 1] >> 16) - first;
    if (a.depth[at_node] < 0) return;
    const int64_t stride = (int64_t)a.T * Hq, row = (int64_t)first * stride + (int64_t)node * Hq + head;
    const int mine = MANY ? lane : l;
    float4 x = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if (mine < n) x = a.record[row + mine * stride];
    float M = x.x;
    for (int o = 1; o < GROUP; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
    const float share = fast_exp2(x.x - (M == -INFINITY ? 0.f : M)) * x.y;
    float L = share;
    for (int o = 1; o < GROUP; o <<= 1) L += __shfl_xor(L, o);
    const float weight = share == 0.f ? 0.f : share / L * x.z;
    const _Float16 *src = a.part + row * D + 8 * l;
    f32x8_t O = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    constexpr int U = MANY ? 4 : 8, STEP = MANY ? SP : 1;
    for (int s0 = 0; s0 < n; s0 += U * STEP) {
        static_for<0, U>([&](auto u) {
            const int s = s0 + (int)u * STEP + (MANY ? sp : 0), from = min(s, n - 1);
            float w = __shfl(weight, MANY ? from : sp * LPR + from);
            if (s >= n) w = 0.f;
            const f32x8_t v = __builtin_convertvector(*reinterpret_cast<const f16x8_t *>(src + from * stride * D), f32x8_t);
            static_for<0, 8>([&](auto i) { O[(int)i] = w == 0.f ? O[(int)i] : fmaf(w, v[(int)i], O[(int)i]); });   // 0 * inf
        });
    }
    if constexpr (MANY)
        for (int o = LPR; o < 64; o <<= 1) static_for<0, 8>([&](auto i) { O[(int)i] += __shfl_xor(O[(int)i], o); });
    if (hd >= Hq || (MANY && sp != 0)) return;
    const int64_t at = at_node * Hq + hd;
    *reinterpret_cast<bf16x8_t *>(a.out + at * D + 8 * l) = __builtin_convertvector(O, bf16x8_t);
    if (l == 0) a.lse[at] = kLn2 * (M + log2f(L));
}

template <int D, int RW, bool F8, bool PACKED>
bool launch_tree_kernel(const TreeArgs &args, int blocks, hipStream_t stream) {
    constexpr int OWN_LDS = TreeTile<D, RW, F8>::LDS, PROMPT_LDS = PACKED ? TreeTile<D, 4, false>::LDS : 0;
    constexpr int LDS = PROMPT_LDS > OWN_LDS ? PROMPT_LDS : OWN_LDS;
    void (*kernel)(TreeArgs);
    if constexpr (PACKED) kernel = tree_packed_kernel<D, RW, F8>;
    else kernel = tree_kernel<D, RW, F8>;
    // more LDS than a kernel may take unasked; asked once a device
    static std::atomic<uint64_t> raised{0};
    int dev = 0;
    if (LDS > 64 << 10) {
        if (hipGetDevice(&dev) != hipSuccess) return false;
        const uint64_t bit = 1ull << (dev & 63);
        if (!(raised.load() & bit)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS) !=
                hipSuccess)
                return false;
            raised.fetch_or(bit);
        }
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)args.call.Hkv, (unsigned)blocks), dim3(256), LDS, stream, args);
    return hipGetLastError() == hipSuccess;
}

template <int D>
bool launch_tree(const TreeArgs &a, const splice::TreePlan &p, int kv_format, hipStream_t stream) {
    const bool f8 = kv_format == SPLICE_KV_E4M3;
    bool ok = false;
    auto go = [&](auto rw) {
        constexpr int RW = decltype(rw)::value;
        if (p.row_waves != RW) return;
        if constexpr (RW < 4) {
            if (p.n_p > 0) {
                ok = f8 ? launch_tree_kernel<D, RW, true, true>(a, p.blocks, stream)
                        : launch_tree_kernel<D, RW, false, true>(a, p.blocks, stream);
                return;
            }
        }
        if (p.n_p > 0) return;   // no kernel: the plan has none such
        ok = f8 ? launch_tree_kernel<D, RW, true, false>(a, p.blocks, stream)
                : launch_tree_kernel<D, RW, false, false>(a, p.blocks, stream);
    };
    if constexpr (D <= 128) go(std::integral_constant<int, 1>{});
    go(std::integral_constant<int, 2>{});
    go(std::integral_constant<int, 4>{});
    const TreeCall &c = a.call;
    if (!ok || !c.split) return ok;
    const int Hq = c.Hkv * c.G, rows = p.most_chunks > 8 ? 4 : 4 * 64 / (D / 8);   // a work group's
    const dim3 grid((unsigned)(c.n_active * c.T), (unsigned)((Hq + rows - 1) / rows));
    if (p.most_chunks > 8) hipLaunchKernelGGL((tree_join_kernel<D, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((tree_join_kernel<D, false>), grid, dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess;
}

bool launch_tree_d64(const TreeArgs &, const splice::TreePlan &, int, hipStream_t);
bool launch_tree_d128(const TreeArgs &, const splice::TreePlan &, int, hipStream_t);
bool launch_tree_d256(const TreeArgs &, const splice::TreePlan &, int, hipStream_t);

}  // namespace splice_dev
