// page_plan.hpp -- launch planning of splice_page_attn (splice_pages.h), on the
// host before any launch.
//
// A KV head's rows are (cell, token, q head) triples.  A row tile is a work group's
// rows; its list of keys is walked page by page, cut into parts of `per` pages,
// one work group each.  Own tiles hold rows of one cell, and walk
//   - the prompt (unspliced or spliced: their tokens are in different tiles) and
//     the cell's rows, or
//   - the cell's rows alone, where the prompt is shared: then tiles of any cells'
//     unspliced or spliced rows walk the prompt.
// A (row, part) leaves a partial result; where a row has more than one, a second
// launch joins them.
#pragma once

#include <algorithm>

#include "page_format.hpp"

namespace splice {

constexpr int kPageMaxParts = 64;    // partial results a row may have (a lane each in the join)
constexpr int64_t kPageWorkspace = (int64_t)64 << 20;   // what they may take, where two of them take less

// Rows of an own tile whose waves take different keys, and of one whose waves take different rows.
constexpr int page_narrow_rows(int D, int r) { return 16 * (D <= 128 ? r : 1); }
constexpr int page_wide_rows(int D) { return D <= 128 ? 128 : 64; }

struct PagePlan {
    int own;                 // row sets of 16 a wave of an own tile holds with its waves on different keys (1, 2); 0: wide tiles
    bool shared;             // the prompt's tiles hold rows of any cells
    int own_rows;            // rows of an own tile
    int own_tiles, own_each; // own tiles in all; of every cell, where they have equally many, else 0
    int own_per, own_parts;
    int rows_u, rows_s;      // shared: unspliced and spliced rows of a KV head, their tiles
    int tiles_u, tiles_s;
    int prompt_per, prompt_parts;
    int parts;
    int64_t blocks, bytes;
};

// Partial results that a call of this shape may leave: the workspace holds that many.
inline int page_most_parts(const splice_shape &sh, const splice_pages &pg) {
    const int64_t one = (int64_t)sh.n_cells * pg.n_tokens * sh.n_q_heads * (sh.head_dim + 2) * 4;
    return (int)std::min<int64_t>(kPageMaxParts, std::max<int64_t>(2, kPageWorkspace / std::max<int64_t>(one, 1)));
}
inline int64_t page_part_bytes(const splice_shape &sh, const splice_pages &pg) {
    return ((int64_t)sh.n_cells * pg.n_tokens * sh.n_q_heads * (sh.head_dim + 2) * 4 + 255) / 256 * 256;
}

// A cell of a call: rows it has, tokens it adds, how many of them come before its onset.
struct PageCell {
    int cell, step, count, split;
};

inline int page_pages(int lo, int hi) { return hi > lo ? (hi - 1) / kPageRows - lo / kPageRows + 1 : 0; }

// Pages that a tile with tokens [t0, t1) of a cell walks.
inline int own_list(const splice_shape &sh, int window, const PageCell &c, int t0, int t1, bool spliced, bool shared) {
    const int64_t low = window > 0 ? (int64_t)sh.prompt_len + c.step + t0 - window + 1 : 0;
    const int g0 = (int)std::max<int64_t>(0, low - sh.prompt_len), v0 = (int)std::min<int64_t>(sh.prompt_len, std::max<int64_t>(0, low));
    int n = page_pages(g0, c.step + t1);
    if (shared) return n;
    if (!spliced) return n + page_pages(v0, sh.prompt_len);
    n += page_pages(v0, sh.span_lo) + page_pages(std::max(v0, sh.span_hi), sh.prompt_len);
    return sh.donor_kind == SPLICE_DONOR_ZERO ? n : n + page_pages(std::max(v0, sh.span_lo), sh.span_hi);
}

inline PagePlan page_plan(const splice_shape &sh, const splice_call &call, const splice_pages &pg, const PageCell *cells, int n,
                          int units) {
    PagePlan p{};
    const int G = group_of(sh), D = sh.head_dim, Hkv = sh.n_kv_heads;
    int most_rows = 0;
    for (int i = 0; i < n; ++i) most_rows = std::max(most_rows, cells[i].count * G);
    const int seen = call.window > 0 ? std::min(sh.prompt_len, call.window) : sh.prompt_len;
    p.own = most_rows <= 16 ? 1 : (most_rows <= 64 ? (D <= 128 ? 2 : 1) : 0);
    p.own_rows = p.own ? page_narrow_rows(D, p.own) : page_wide_rows(D);
    // tiles of several cells' rows save walks over the prompt only where a cell's own rows do not fill them
    p.shared = n > 1 && most_rows <= 64 && (int64_t)(n - 1) * seen * D >= (int64_t)5 << 18;
    // own tiles, their number and pages
    int64_t pages = 0;
    int longest = 0;
    p.own_each = -1;
    for (int i = 0; i < n; ++i) {
        const PageCell &c = cells[i];
        int tiles = 0;
        auto add = [&](int t0, int t1, bool spliced) {
            const int rows = (t1 - t0) * G, of = ceil_div(rows, p.own_rows), per_tile = p.own_rows / G;
            tiles += of;
            // the last and the first tile's lists bound the others'
            const int hi = own_list(sh, call.window, c, std::max(t0, t1 - per_tile), t1, spliced, p.shared);
            const int lo = own_list(sh, call.window, c, t0, std::min(t1, t0 + per_tile), spliced, p.shared);
            longest = std::max(longest, std::max(lo, hi));
            pages += (int64_t)of * (lo + hi) / 2;
        };
        if (p.shared) add(0, c.count, false);
        else {
            if (c.split > 0) add(0, c.split, false);
            if (c.split < c.count) add(c.split, c.count, true);
        }
        p.own_each = p.own_each == -1 || p.own_each == tiles ? tiles : 0;
        p.own_tiles += tiles;
    }
    int cap = page_most_parts(sh, pg);
    // the prompt's tiles
    if (p.shared) {
        for (int i = 0; i < n; ++i) {
            p.rows_u += cells[i].split * G;
            p.rows_s += (cells[i].count - cells[i].split) * G;
        }
        const int RT = page_wide_rows(D), list = page_pages(0, seen) + 2;
        p.tiles_u = ceil_div(p.rows_u, RT);
        p.tiles_s = ceil_div(p.rows_s, RT);
        const int64_t tiles = (int64_t)(p.tiles_u + p.tiles_s) * Hkv;
        int parts = (int)std::min<int64_t>(std::max(1, cap / 2), std::max<int64_t>(1, 2 * units / tiles));
        p.prompt_per = call.split_keys ? call.split_keys / kPageRows : std::max(4, ceil_div(list, parts));
        p.prompt_parts = std::min(ceil_div(list, p.prompt_per), std::max(1, cap - 1));
        p.prompt_per = ceil_div(list, p.prompt_parts);
        cap = std::max(1, cap - p.prompt_parts);
    }
    const int64_t target = (int64_t)units * (p.own ? 3 : 2);
    const int64_t blocks = (int64_t)p.own_tiles * Hkv;
    int per = (int)std::max<int64_t>(p.own ? 4 : 8, (pages * Hkv + target - 1) / target);
    if (blocks >= 2 * target) per = std::max(1, longest);   // enough work groups without a cut
    if (call.split_keys) per = call.split_keys / kPageRows;
    p.own_parts = std::min(std::max(1, ceil_div(longest, per)), cap);
    p.own_per = std::max(1, ceil_div(longest, p.own_parts));
    p.parts = p.own_parts + p.prompt_parts;
    p.blocks = blocks * p.own_parts + (int64_t)(p.tiles_u + p.tiles_s) * Hkv * p.prompt_parts;
    p.bytes = p.parts > 1 ? p.parts * page_part_bytes(sh, pg) : 0;
    return p;
}

}  // namespace splice
