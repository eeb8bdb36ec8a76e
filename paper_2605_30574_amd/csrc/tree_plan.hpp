// tree_plan.hpp -- host-side checks and launch planning of the tree entries
// (splice_tree.h).  Everything here runs on the CPU before any launch.
#pragma once

#include <stdint.h>

#include <type_traits>

#include "plan.hpp"
#include "splice_tree.h"

namespace splice {

// The cells that are not finished, in order: their index and step.
struct TreeCells {
    int32_t step[SPLICE_MAX_CELLS];
    uint8_t cell[SPLICE_MAX_CELLS];
};

inline int active_cells(const splice_shape &sh, const int32_t *cell_step, TreeCells &out) {
    int n = 0;
    for (int c = 0; c < sh.n_cells; ++c)
        if (cell_step[c] >= 0) {
            out.step[n] = cell_step[c];
            out.cell[n++] = (uint8_t)c;
        }
    return n;
}

inline int32_t validate_tree_shape(const splice_shape *shape, const splice_tree *tree) {
    const int32_t rc = validate_shape(shape);
    if (rc != SPLICE_OK) return rc;
    if (!tree || (tree->kv_format != SPLICE_KV_BF16 && tree->kv_format != SPLICE_KV_E4M3)) return SPLICE_EINVAL;
    if (tree->n_nodes < 1) return SPLICE_ESHAPE;
    if (tree->n_nodes > SPLICE_MAX_NODES || shape->dtype != SPLICE_BF16) return SPLICE_EUNSUPPORTED;
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

// Calls f with (head_dim, 8-bit cache) as compile-time constants.
template <class F>
void with_format(int D, int kv_format, F f) {
    auto pick = [&](auto d) {
        if (kv_format == SPLICE_KV_E4M3) f(d, std::true_type{});
        else f(d, std::false_type{});
    };
    if (D == 64) pick(std::integral_constant<int, 64>{});
    else if (D == 128) pick(std::integral_constant<int, 128>{});
    else pick(std::integral_constant<int, 256>{});
}

// ---------------------------------------------------------------- attention

// Waves of a work group that take different rows (32 each); the other of its
// four waves take different keys of the same rows.
constexpr int tree_row_waves(int D, int rows) { return rows <= 32 && D <= 128 ? 1 : (rows <= 64 ? 2 : 4); }
// 32-key blocks a wave takes of a tile.
constexpr int tree_key_blocks(int D, int row_waves) { return row_waves == 4 && D <= 128 ? 2 : 1; }
constexpr int tree_tile_keys(int D, int row_waves) { return 32 * tree_key_blocks(D, row_waves) * (4 / row_waves); }

constexpr int kTreeMaxSplits = 64;
constexpr int kTreeItemsTarget = 1024;   // work groups a split aims for
constexpr int kTreeMinTiles = 2;         // tiles of keys a split takes at least

struct TreePlan {
    int row_waves, row_tiles, n_split;
    size_t bytes;   // partial results: [split][active cell][node][q head] of D + 2 floats
};

// keys: the most any cell of the call sees.
inline TreePlan tree_plan(const splice_shape &sh, const splice_call &call, int T, int n_active, int64_t keys) {
    TreePlan p;
    const int rows = T * group_of(sh);
    p.row_waves = tree_row_waves(sh.head_dim, rows);
    p.row_tiles = ceil_div(rows, 32 * p.row_waves);
    const int64_t items = (int64_t)n_active * sh.n_kv_heads * p.row_tiles;
    const int tile = tree_tile_keys(sh.head_dim, p.row_waves);
    int64_t n = call.split_keys > 0 ? ceil_div(keys, call.split_keys) : ceil_div(kTreeItemsTarget, items);
    const int64_t most = ceil_div(keys, (call.split_keys > 0 ? 1 : kTreeMinTiles) * tile);
    n = n < most ? n : most;
    n = n < kTreeMaxSplits ? n : kTreeMaxSplits;
    p.n_split = n > 1 ? (int)n : 1;
    p.bytes = p.n_split > 1 ? (size_t)p.n_split * n_active * T * sh.n_q_heads * (sh.head_dim + 2) * 4 : 0;
    return p;
}

// Keys a cell at `step` may see: prompt slots (both of a replaced span's if
// nodes on either side of the onset share a tile) and generated rows.
inline int64_t tree_keys(const splice_shape &sh, const splice_call &call, int T, int64_t step) {
    int64_t prompt = sh.prompt_len, gen = step;
    if (call.window > 0) {
        const int64_t low = sh.prompt_len + step - call.window + 1;   // of the root
        if (low > 0) prompt -= low < prompt ? low : prompt;
        if (low > sh.prompt_len) gen -= low - sh.prompt_len < gen ? low - sh.prompt_len : gen;
    }
    return prompt + gen + T;
}

}  // namespace splice
