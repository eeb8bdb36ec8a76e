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

// What a walk is taken to cost, in us, fitted to sweeps of the part lengths of ten shapes (D = 128; pages of other
// heads by their bytes): a page takes a work group `alone` where the GPU has room for all of them, and all of
// them take `rate` pages a us where it has not.  A narrow work group's four waves take a page each, a wide one's all the
// same page for eight times the rows.
struct PageCost {
    double alone, rate;
};
inline PageCost page_cost(int D, int own) {
    const double size = D / 128.0;
    if (own == 1) return {D == 256 ? 0.45 : 0.24 * size, 588 / size};
    if (own == 2) return {0.35 * size, 400 / size};
    return {1.55 * size, 216 / size};
}
constexpr double kPageStart = 4;       // a launch and a work group's first bytes
constexpr double kPageNext = 2;        // what a work group costs that follows another
constexpr double kPageJoin = 4;        // a second launch, and the partial results' way there and back:
constexpr double kPageJoinPart = 0.2;  // each
constexpr double kPageJoinRate = 4e6;  // bytes a us
constexpr double kPageAgain = 1000;    // pages (D = 128) a us that several cells' narrow tiles take of one prompt, from the caches

struct PageWork {
    int tiles, each, longest;
    int64_t pages;   // of all tiles of a KV head
};

inline PageWork own_work(const splice_shape &sh, const splice_call &call, const PageCell *cells, int n, int own_rows, bool shared) {
    PageWork w{0, -1, 0, 0};
    const int G = group_of(sh), per_tile = own_rows / G;
    for (int i = 0; i < n; ++i) {
        const PageCell &c = cells[i];
        int tiles = 0;
        auto add = [&](int t0, int t1, bool spliced) {
            const int of = ceil_div((int64_t)(t1 - t0) * G, own_rows);
            tiles += of;
            const int hi = own_list(sh, call.window, c, std::max(t0, t1 - per_tile), t1, spliced, shared);
            const int lo = of == 1 ? hi : own_list(sh, call.window, c, t0, std::min(t1, t0 + per_tile), spliced, shared);
            w.longest = std::max(w.longest, std::max(lo, hi));
            w.pages += (int64_t)of * (lo + hi) / 2;
        };
        const int split = shared ? c.count : c.split;
        if (split > 0) add(0, split, false);
        if (split < c.count) add(split, c.count, true);
        w.each = w.each == -1 || w.each == tiles ? tiles : 0;
        w.tiles += tiles;
    }
    return w;
}

inline PagePlan page_plan(const splice_shape &sh, const splice_call &call, const splice_pages &pg, const PageCell *cells, int n,
                          int units) {
    static const int counts[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64};
    const int G = group_of(sh), D = sh.head_dim, Hkv = sh.n_kv_heads, cap = page_most_parts(sh, pg);
    int most_rows = 0, rows_u = 0, rows_s = 0;
    for (int i = 0; i < n; ++i) {
        most_rows = std::max(most_rows, cells[i].count * G);
        rows_u += cells[i].split * G;
        rows_s += (cells[i].count - cells[i].split) * G;
    }
    const int own = most_rows <= 16 ? 1 : (most_rows <= 64 ? (D <= 128 ? 2 : 1) : 0);
    const int own_rows = own ? page_narrow_rows(D, own) : page_wide_rows(D);
    const PageCost cost = page_cost(D, own);
    PageCost wide = page_cost(D, 0);
    const double slots = 2.0 * units, result = (double)(rows_u + rows_s) * Hkv * D * 4 * 2 / kPageJoinRate;
    const int seen = call.window > 0 ? std::min(sh.prompt_len, call.window) : sh.prompt_len, list = page_pages(0, seen) + 2;
    const int tiles_u = ceil_div(rows_u, page_wide_rows(D)), tiles_s = ceil_div(rows_s, page_wide_rows(D));
    if (tiles_u + tiles_s > 0)   // waves without rows leave the others room
        wide.alone *= 0.4 + 0.6 * (rows_u + rows_s) / ((tiles_u + tiles_s) * page_wide_rows(D));
    const int forced = call.split_keys / kPageRows;
    PagePlan best{};
    double least = 0;
    bool any = false;
    // tiles of several cells' rows save walks over the prompt where a cell's own rows do not fill them
    double again = 0;   // pages of the prompt walked by tiles of their own
    for (int shared = 0; shared <= (n > 1 && own && seen > 0 ? 1 : 0); ++shared) {
        const PageWork w = own_work(sh, call, cells, n, own_rows, shared != 0);
        if (shared == 0 && n > 1 && own == 1 && seen > 0)
            again = std::max<int64_t>(0, w.pages - own_work(sh, call, cells, n, own_rows, true).pages) * (double)Hkv;
        const double own_pages = (double)w.pages * Hkv, prompt_tiles = shared ? (double)(tiles_u + tiles_s) * Hkv : 0;
        int last_prompt = 0;
        for (int pc : counts) {
            int per_prompt = shared ? (forced ? forced : ceil_div(list, pc)) : 0;
            const int prompt_parts = shared ? std::min(ceil_div(list, per_prompt), cap - 1) : 0;
            if (shared) per_prompt = ceil_div(list, prompt_parts);
            if (pc > 1 && prompt_parts == last_prompt) break;   // as before: no more parts than pages, or than there is room for
            last_prompt = prompt_parts;
            int last_own = 0;
            for (int oc : counts) {
                int per = forced ? forced : std::max(1, ceil_div(w.longest, oc));
                const int parts = std::min(std::max(1, ceil_div(w.longest, per)), cap - prompt_parts);
                per = std::max(1, ceil_div(w.longest, parts));
                if (own && per > 8) per = (per + 7) / 8 * 8;   // the four waves' two pages each
                if (oc > 1 && parts == last_own) break;
                last_own = parts;
                // work groups with pages: every tile's list is cut after `per`
                const double groups = std::max((double)w.tiles * Hkv, std::min((double)w.tiles * Hkv * parts, own_pages / per + 0.5 * w.tiles * Hkv));
                const double prompts = prompt_tiles * prompt_parts, all = groups + prompts;
                const double most = groups / cost.alone;
                double t = (shared ? own_pages : own_pages - again) / std::min(most, cost.rate) + 0.5 * per * cost.alone;
                if (!shared) t += again / std::min(most, kPageAgain * 128 / D);
                if (shared) {
                    t += prompt_tiles * list / std::min(prompts / wide.alone, wide.rate);
                    t = std::max(t, per_prompt * wide.alone * 1.3);
                }
                t += kPageStart + kPageNext * std::max(0.0, all - slots) / slots;
                if (parts + prompt_parts > 1) t += kPageJoin + (kPageJoinPart + result) * (parts + prompt_parts);
                if (!any || t < least) {
                    any = true;
                    least = t;
                    best = PagePlan{own, shared != 0, own_rows, w.tiles, w.each, per, parts, shared ? rows_u : 0, shared ? rows_s : 0,
                                    shared ? tiles_u : 0, shared ? tiles_s : 0, per_prompt, prompt_parts, parts + prompt_parts, 0, 0};
                }
            }
        }
    }
    best.blocks = (int64_t)best.own_tiles * Hkv * best.own_parts + (int64_t)(best.tiles_u + best.tiles_s) * Hkv * best.prompt_parts;
    best.bytes = best.parts > 1 ? best.parts * page_part_bytes(sh, pg) : 0;
    return best;
}

}  // namespace splice
