// tree_plan.hpp -- host-side checks and launch planning of the tree entries
// (splice_tree.h).  Everything here runs on the CPU before any launch.
#pragma once

#include <stdint.h>

#include <type_traits>

#include "plan.hpp"
#include "splice_tree.h"

namespace splice {

// Up to N cells that are not finished, in order: their steps and indexes.  Words
// throughout, as kernels read these at a computed place: a byte array beside a
// word array under one index has been compiled into a scalar load whose base
// is no multiple of four, and the hardware drops those bits.
template <int N>
struct TreeCells {
    int32_t step[N];
    uint32_t cell[N];
};

inline int active_cells(const splice_shape &sh, const int32_t *cell_step) {
    int n = 0;
    for (int c = 0; c < sh.n_cells; ++c) n += cell_step[c] >= 0;
    return n;
}

template <int N>
void list_cells(const splice_shape &sh, const int32_t *cell_step, TreeCells<N> &out) {
    int n = 0;
    for (int c = 0; c < sh.n_cells && n < N; ++c)
        if (cell_step[c] >= 0) {
            out.step[n] = cell_step[c];
            out.cell[n++] = (uint32_t)c;
        }
}

inline int32_t validate_tree_shape(const splice_shape *shape, const splice_tree *tree) {
    const int32_t rc = validate_shape(shape);
    if (rc != SPLICE_OK) return rc;
    if (!tree || (tree->kv_format != SPLICE_KV_BF16 && tree->kv_format != SPLICE_KV_E4M3)) return SPLICE_EINVAL;
    if (tree->n_nodes < 1) return SPLICE_ESHAPE;
    if (tree->n_nodes > SPLICE_MAX_NODES || shape->dtype != SPLICE_BF16) return SPLICE_EUNSUPPORTED;
    // a launch has fewer than 2^32 threads along x (256 cells, a work group a KV head each) and 2^16 work groups along y
    if (shape->n_q_heads >= 1 << 16) return SPLICE_EUNSUPPORTED;
    if (tree->n_nodes > shape->gen_capacity) return SPLICE_ESHAPE;
    return SPLICE_OK;
}

inline int32_t validate_tree(const splice_shape *shape, const splice_tree *tree, const int32_t *cell_step) {
    const int32_t rc = validate_tree_shape(shape, tree);
    if (rc != SPLICE_OK) return rc;
    if (shape->n_cells == 0) return SPLICE_OK;
    if (!cell_step) return SPLICE_EINVAL;
    for (int c = 0; c < shape->n_cells; ++c)
        if (cell_step[c] > shape->gen_capacity - tree->n_nodes) return SPLICE_ESHAPE;
    return SPLICE_OK;
}

// Calls f with (head_dim, 8-bit cache, room for the n active cells) as
// compile-time constants.  Up to 32 cells have arguments of their own size: a launch copies them, and
// 2 KB of cells more took 0.4 us of the host's 6.7 for a call that moves a few rows.
constexpr int kTreeFewCells = 32;
template <class F>
void with_format(int D, int kv_format, int n, F f) {
    auto room = [&](auto d, auto f8) {
        if (n <= kTreeFewCells) f(d, f8, std::integral_constant<int, kTreeFewCells>{});
        else f(d, f8, std::integral_constant<int, SPLICE_MAX_CELLS>{});
    };
    auto pick = [&](auto d) {
        if (kv_format == SPLICE_KV_E4M3) room(d, std::true_type{});
        else room(d, std::false_type{});
    };
    if (D == 64) pick(std::integral_constant<int, 64>{});
    else if (D == 128) pick(std::integral_constant<int, 128>{});
    else pick(std::integral_constant<int, 256>{});
}

// ---------------------------------------------------------------- attention

// Waves of a work group that take different rows (32 each); the other of its
// four waves take different keys of the same rows.  One up to 32 rows: waves of
// bytes in flight that do not wait for each other (us, one / two row waves: 64
// cells of 5 nodes, D = 128, 2k 8-bit rows each 82 / 96, bf16 rows 115 / 117; 3 cells of
// 5 nodes, D = 64, 16 / 21; but one cell of one node over 8k slots 20 / 19).  Two up
// to 64 rows, where two more would have none; four above, as a tile then serves
// 128 rows (four / two: 8 cells of 32 nodes over 8k slots 58 / 64).
constexpr int tree_row_waves(int D, int rows) { return rows <= 32 && D <= 128 ? 1 : (rows <= 64 ? 2 : 4); }
// 32-key blocks a wave takes of a tile.
constexpr int tree_key_blocks(int D, int row_waves) { return row_waves == 4 && D <= 128 ? 2 : 1; }
// With one wave a row every wave has tiles of its own.
constexpr int tree_tile_keys(int D, int row_waves) {
    return row_waves == 1 ? 32 : 32 * tree_key_blocks(D, row_waves) * (4 / row_waves);
}
constexpr int tree_resident(int D, bool f8) { return D > 128 && f8 ? 1 : 2; }   // work groups a compute unit holds

// A cell's list of keys is cut into chunks of `per` tiles, one work group
// each (per KV head and row tile); a slot is one chunk of one cell.
constexpr int kTreeMaxSlots = 640;
// Rounds of resident work groups a plan may take to balance its chunks, and what a
// work group costs beside its tiles, in tiles (us: 48 cells of 16 nodes over 8k
// slots, some on both sides of their onset, 6 rounds 152, 1 round 198, and 8 tiles 152, 2 165, 16 198;
// half of the cells spliced and none so, 148, 140, and 148, 166, 136; 64 cells of 16
// nodes, 2k bf16 rows each, 118, 119, and 118 with any).
constexpr int kTreeRounds = 6;
constexpr int kTreeStart = 8;
// What the join of chunks costs, in tiles: a launch and the partial results' way (two sets
// of 79 shapes, geometric means in us, 0 tiles 23.1 and 24.6, 3 22.1 and 23.7, 6 21.8 and 22.1, 8 21.8 and 22.0,
// where some lists of 100 tiles are no longer cut and take 19 rather than 15).
constexpr int kTreeJoin = 6;
constexpr int kTreeMaxChunks = 64;

struct TreePlan {
    int row_waves, row_tiles, per;
    int n_p, p_tiles;      // packed: chunks of the prompt, tiles of 128 rows; else 0
    int p_heavy0, p_heavy; // ... of them, first and number, with unspliced and spliced nodes
    int n_slots, blocks;   // partial results a (node, q head) may have, over all cells; work groups a KV head
    int most_chunks;       // of a cell
    bool split;            // some cell has more than one chunk
    size_t bytes;          // partial results: [slot][node][q head] of D fp16 and four floats
};

// An active cell: its index, the depth from which its nodes are spliced (64:
// none) and its first slot (there is one more, for the end).  An item of the
// grid: its active cell and chunk, two items a word; chunks of one number
// stand together, so that work groups that run together read the same part of
// the prompt, and the active cells are in the order of their class (unspliced,
// on both sides of the onset, spliced), so that they read the same span.
struct TreeSlots {
    uint32_t info[SPLICE_MAX_CELLS + 1];   // cell | onset << 8 | first slot << 16
    uint32_t order[kTreeMaxSlots / 2];     // active cell | chunk << 8, in 16 bits
};

inline void tree_slots(const TreeCells<SPLICE_MAX_CELLS> &cells, const uint8_t *onset, const int *tiles, int n, const TreePlan &p, TreeSlots &out) {
    uint32_t first = 0;
    int most = 0;
    for (int i = 0; i < n; ++i) {
        out.info[i] = cells.cell[i] | (uint32_t)onset[i] << 8 | first << 16;
        first += (uint32_t)(p.n_p + ceil_div(tiles[i], p.per));
        most = tiles[i] > most ? tiles[i] : most;
    }
    out.info[n] = first << 16;
    int at = 0;
    for (int chunk = 0; chunk * p.per < most; ++chunk)
        for (int i = 0; i < n; ++i)
            if (chunk * p.per < tiles[i]) {
                const uint32_t x = (uint32_t)i | (uint32_t)chunk << 8;
                out.order[at / 2] = at % 2 ? out.order[at / 2] | x << 16 : x;
                ++at;
            }
}

inline size_t tree_slot_bytes(const splice_shape &sh, int T) { return (size_t)T * sh.n_q_heads * (2 * sh.head_dim + 16); }

// The most tiles that a cell at `step` walks: prompt slots (a replaced span
// twice when nodes on both sides of the onset may share a row tile) and
// generated rows; every segment may end in a tile of its own.
// prompt, gen: whether the parts count.
inline int tree_tiles(const splice_shape &sh, const splice_call &call, int T, int tile, int64_t step, bool spliced, bool mixed,
                      bool prompt, bool gen) {
    int64_t low = call.window > 0 ? sh.prompt_len + step - call.window + 1 : 0;   // the first position that the root sees
    if (low < 0) low = 0;
    const int64_t Tp = sh.prompt_len, b0 = low < Tp ? low : Tp, g0 = low > Tp ? (low - Tp < step ? low - Tp : step) : 0;
    const int64_t sa = sh.span_lo > b0 ? sh.span_lo : b0, sb = sh.span_hi > sa ? sh.span_hi : sa;
    int64_t n = gen ? ceil_div(step + T - g0, tile) : 0;
    if (!prompt) return (int)n;
    if (!spliced) return (int)(n + ceil_div(Tp - b0, tile));
    n += ceil_div(sa - b0, tile) + ceil_div(Tp - sb, tile);
    const int span = ceil_div(sb - sa, tile);
    return (int)(n + (mixed ? span : 0) + (sh.donor_kind == SPLICE_DONOR_ZERO ? 0 : span));
}

inline int64_t tree_chunks(const int *tiles, int n, int per) {
    int64_t slots = 0;
    for (int i = 0; i < n; ++i) slots += ceil_div(tiles[i], per);
    return slots;
}

// A packed call: the cells' rows of a KV head, 128 a work group, share the
// prompt's tiles, and each cell's generated rows have items of their own.
// That takes another partial result a row, and pays where the cells together
// walk much prompt: n cells times its keys times head_dim from 5 * 2^20 on
// (us, apart / packed, half of the cells spliced: 64 cells of 5 nodes, D = 128, 512 keys
// 20 / 30, 1024 27 / 34, 2048 40 / 38; 40 cells of 12 nodes 512 keys 24 / 33, 2048 46 / 44;
// 8 cells of 5 nodes 2048 keys 21 / 21; 48 cells of 16 nodes 8192 keys 171 / 148; D = 256, 64
// cells of one node 256 keys 27 / 22, 1024 38 / 26; D = 64, 64 cells of 5 nodes 1024 keys
// 16 / 17; the border itself is coarse: near it either side may be the faster one). A call that sets
// split_keys packs whenever it can.
constexpr int kTreeMaxPrompt = 16;                 // chunks of the prompt
constexpr int kTreePackedRows = 64;                // rows of a cell (more fill the waves of a work group by themselves)
static_assert(tree_row_waves(64, kTreePackedRows) < 4 && tree_row_waves(128, kTreePackedRows) < 4 &&
              tree_row_waves(256, kTreePackedRows) < 4, "the packed kernels take up to two row waves for the generated rows");
constexpr int64_t kTreePackedWork = 5 << 20;

inline bool tree_packed(const splice_shape &sh, const splice_call &call, int T, int n, int64_t prompt_keys) {
    if (T * group_of(sh) > kTreePackedRows || n < 2 || prompt_keys < 1) return false;
    return call.split_keys > 0 || n * prompt_keys * sh.head_dim >= kTreePackedWork;
}

// Chunks of equal length, so that the work groups of all cells fill k rounds
// of what the GPU holds at once; k is the one that takes least by
// k * (per + kTreeStart), and kTreeJoin where lists are cut; of a packed call's prompt one more kTreeStart where the
// generated rows' items do not fit beside its last round (40 cells of 12 nodes,
// D = 256, 1024 keys in view: 16 chunks of two tiles 44 us, 8 of four, beside
// which they fit, 32).  tiles: of the cells' lists, in a packed call without
// the prompt, whose list is prompt_tiles long.
// n_of: cells of each class.
inline TreePlan tree_plan(const splice_shape &sh, const splice_call &call, int T, const int *tiles, int n, const int *n_of,
                          int n_cu, bool f8, bool packed, int prompt_tiles) {
    TreePlan p;
    const int rows = T * group_of(sh);
    p.row_waves = tree_row_waves(sh.head_dim, rows);
    p.row_tiles = ceil_div(rows, 32 * p.row_waves);
    p.n_p = p.p_tiles = p.p_heavy0 = p.p_heavy = 0;
    const int tile = tree_tile_keys(sh.head_dim, p.row_waves), step = p.row_waves == 1 ? 4 : 1;   // four waves, four tiles
    const int64_t items = (int64_t)sh.n_kv_heads * p.row_tiles, room = (int64_t)n_cu * tree_resident(sh.head_dim, f8);
    int64_t sum = 0;
    int most = 1;
    for (int i = 0; i < n; ++i) {
        sum += tiles[i];
        most = tiles[i] > most ? tiles[i] : most;
    }
    const int most_chunks = kTreeMaxChunks - (packed ? kTreeMaxPrompt : 0);
    const int least = step * ceil_div(most, (int64_t)step * most_chunks);   // no cell in more than kTreeMaxChunks
    auto fits = [&](int per, int64_t limit) { return tree_chunks(tiles, n, per) <= limit; };
    if (call.split_keys > 0) {
        p.per = step * ceil_div(call.split_keys, tile * step);
        if (p.per < least) p.per = least;
        while (!fits(p.per, kTreeMaxSlots)) p.per *= 2;
    } else {
        p.per = step * ceil_div(most, step);   // whole lists
        int64_t best = packed ? INT64_MAX : ceil_div(n * items, room) * ((int64_t)p.per / step + kTreeStart);
        for (int k = 1; k <= (packed ? 1 : kTreeRounds); ++k) {   // the prompt's items fill the further rounds
            int64_t limit = k * room / items;
            limit = limit < kTreeMaxSlots ? limit : kTreeMaxSlots;
            if (limit < n) continue;   // not even whole lists fit
            int per = step * ceil_div(sum, limit * step);
            if (per < least) per = least;
            while (per < most && !fits(per, limit)) per += step * (1 + per / (16 * step));
            const bool cut = !packed && tree_chunks(tiles, n, per) > n;   // (packed results are joined anyhow)
            const int64_t cost = k * ((int64_t)per / step + kTreeStart) + (cut ? kTreeJoin : 0);
            if (cost < best) {
                best = cost;
                p.per = per;
            }
        }
    }
    p.n_slots = (int)tree_chunks(tiles, n, p.per);
    p.blocks = p.row_tiles * p.n_slots;
    p.split = p.n_slots > n;
    if (packed) {
        p.p_tiles = ceil_div((int64_t)n * rows, 128);
        if (n_of[0] < n) {
            p.p_heavy0 = (int)((int64_t)n_of[0] * rows / 128);
            p.p_heavy = n_of[0] + n_of[1] > 0 ? ceil_div((int64_t)(n_of[0] + n_of[1]) * rows, 128) - p.p_heavy0 : 0;
        }
        const int64_t row_items = (int64_t)sh.n_kv_heads * p.p_tiles;
        const int64_t gen_items = (int64_t)sh.n_kv_heads * p.blocks;
        int64_t best = INT64_MAX;
        for (int np = 1; np <= kTreeMaxPrompt && np <= prompt_tiles; ++np) {
            if (np > 1 && call.split_keys == 0 && row_items * np > kTreeRounds * room) break;
            const int64_t per = ceil_div(prompt_tiles, np);
            const int64_t rounds = ceil_div(row_items * np, room), spare = rounds * room - row_items * np;
            const int64_t cost = call.split_keys > 0 ? (per * 64 >= call.split_keys ? -np : np)
                                                     : rounds * (per + kTreeStart) + (spare < gen_items ? kTreeStart : 0);
            if (cost < best) {
                best = cost;
                p.n_p = np;
            }
        }
        p.blocks += p.p_tiles * p.n_p;
        p.n_slots += n * p.n_p;
        p.split = true;
    }
    p.most_chunks = p.n_p + ceil_div(most, p.per);
    p.bytes = p.split ? p.n_slots * tree_slot_bytes(sh, T) : 0;
    return p;
}

// A call's plan, and what its kernels read: n active cells in the order of
// their class, their steps, and the grid's items.
inline TreePlan tree_prepare(const splice_shape &sh, const splice_call &call, const splice_tree &tree, const int32_t *cell_LW,
                             const int32_t *cell_step, int n_cu, int &n, int32_t *step, TreeSlots &slots) {
    const int T = tree.n_nodes;
    const bool f8 = tree.kv_format == SPLICE_KV_E4M3;
    TreeCells<SPLICE_MAX_CELLS> cells, sorted;
    n = active_cells(sh, cell_step);
    if (n == 0) return TreePlan{};
    list_cells(sh, cell_step, cells);
    uint8_t onset[SPLICE_MAX_CELLS], sorted_onset[SPLICE_MAX_CELLS], cls[SPLICE_MAX_CELLS];
    int n_of[3] = {0, 0, 0};
    for (int i = 0; i < n; ++i) {
        const int32_t *lw = cell_LW + 2 * cells.cell[i];
        const int64_t ahead = (int64_t)lw[1] - cells.step[i];   // depth of the onset
        const bool never = call.layer < lw[0] || ahead >= T;
        onset[i] = (uint8_t)(never ? SPLICE_MAX_NODES : (ahead > 0 ? ahead : 0));
        cls[i] = never ? 0 : (ahead > 0 ? 1 : 2);
        ++n_of[cls[i]];
    }
    int at[3] = {0, n_of[0], n_of[0] + n_of[1]}, min_step = cells.step[0];
    for (int i = 0; i < n; ++i) {
        const int to = at[cls[i]]++;
        sorted.cell[to] = cells.cell[i];
        sorted.step[to] = step[to] = cells.step[i];
        sorted_onset[to] = onset[i];
        min_step = cells.step[i] < min_step ? cells.step[i] : min_step;
    }
    // a packed call's list of the prompt: the longest of the classes', for the widest view.  Row tiles with
    // nodes on both sides of the onset walk both forms of a buffer donor's span; they are few, begin
    // first, and count only where there are no others.  Of the ZERO donor spliced nodes walk no span, so unspliced
    // ones set the chunks (half of 48 cells of 16 nodes spliced over all of 8k slots: 95 us, by the spliced cells' list 148).
    const bool zero = sh.donor_kind == SPLICE_DONOR_ZERO, some_spliced = n_of[1] + n_of[2] > 0;
    const bool mixed_view = zero ? n_of[1] > 0 : n_of[1] == n;
    auto view = [&](bool spliced, bool mixed) {
        return tree_tiles(sh, call, T, tree_tile_keys(sh.head_dim, 4), min_step, spliced, mixed, true, false);
    };
    int prompt_tiles = some_spliced ? view(true, mixed_view) : 0;
    if (n_of[0] > 0 && view(false, false) > prompt_tiles) prompt_tiles = view(false, false);
    int64_t prompt_keys = sh.prompt_len;
    if (call.window > 0 && (int64_t)call.window - min_step - 1 < prompt_keys) prompt_keys = (int64_t)call.window - min_step - 1;
    if (zero && n_of[2] == n) {   // nobody walks the span
        const int64_t low = sh.prompt_len - prompt_keys;
        if (sh.span_hi > low) prompt_keys -= sh.span_hi - (sh.span_lo > low ? sh.span_lo : low);
    }
    const bool packed = tree_packed(sh, call, T, n, prompt_keys);
    int tiles[SPLICE_MAX_CELLS];
    const int tile = tree_tile_keys(sh.head_dim, tree_row_waves(sh.head_dim, T * group_of(sh)));
    for (int i = 0; i < n; ++i) {
        const bool spliced = i >= n_of[0], mixed = spliced && i < n_of[0] + n_of[1];
        tiles[i] = tree_tiles(sh, call, T, tile, sorted.step[i], spliced, mixed, !packed, true);
    }
    const TreePlan p = tree_plan(sh, call, T, tiles, n, n_of, n_cu, f8, packed, prompt_tiles);
    tree_slots(sorted, sorted_onset, tiles, n, p, slots);
    return p;
}

// Bytes that no plan of this shape passes, whatever the steps.
inline size_t tree_most_bytes(const splice_shape &sh, const splice_call &call, int T, int n_cu) {
    const int rows = T * group_of(sh), rw = tree_row_waves(sh.head_dim, rows);
    const int64_t items = (int64_t)sh.n_kv_heads * ceil_div(rows, 32 * rw), room = (int64_t)kTreeRounds * n_cu * 2;
    int64_t most = 0;
    for (int n = 1; n <= sh.n_cells; ++n) {
        int64_t slots = call.split_keys == 0 && room / items < kTreeMaxSlots ? room / items : kTreeMaxSlots;
        slots = slots < (int64_t)n * kTreeMaxChunks ? slots : (int64_t)n * kTreeMaxChunks;
        slots = slots > n ? slots : n;
        if (tree_packed(sh, call, T, n, sh.prompt_len)) {
            int64_t np = room / ((int64_t)sh.n_kv_heads * ceil_div((int64_t)n * rows, 128));
            np = call.split_keys > 0 || np > kTreeMaxPrompt ? kTreeMaxPrompt : (np > 1 ? np : 1);
            slots += n * np;
        }
        most = slots > most ? slots : most;
    }
    return most * tree_slot_bytes(sh, T);
}

}  // namespace splice
