// page_format.hpp -- the bytes of a page of 4-bit rows (splice_pages.h), the
// checks that its entries share, and what a call's kernels are told of its cells.
//
// The order of a page's bytes is that in which the attention's matrix
// instructions take their operands, so that a lane's share of a tile is one
// 16-byte load and nothing is transposed on the way:
//   K: v_mfma_f32_16x16x32_bf16 takes 16 tokens x 32 values, lane (token r mod 16, c) eight
//      values.  q's and k's values may stand in any order that is the same for both: a
//      lane's 16 bytes are its token's block c of 32 values, eight for each of four products,
//      under one scale byte, of which a dword has those of tiles 0..3;
//   V: v_mfma_f32_16x16x32_bf16 takes 16 values x 32 tokens, lane (value,
//      c) the tokens whose scores lane (query, c) holds, 4 c + f of either 16-token tile e:
//      16 bytes are 8 tokens of 4 values each.
#pragma once

#include <stdint.h>

#include <type_traits>

#include "plan.hpp"
#include "splice_pages.h"

namespace splice {

constexpr int kPageRows = SPLICE_PAGE_ROWS;

// Places within a head's bytes of a page.
template <int D>
struct PageLayout {
    static constexpr int kBlocks = D / 32;                      // scales a row
    static constexpr int kChunkBlocks = kBlocks < 4 ? kBlocks : 4;
    static constexpr int kV = 32 * D, kKScale = 64 * D, kVScale = 66 * D, kBytes = 68 * D;
    // the 4 bytes (8 values) i of token r's K codes
    static constexpr int k_code(int r, int i) { return r * (D / 2) + 4 * i; }
    // the 2 bytes of V's values 4 u .. 4 u + 3 of token r
    static constexpr int v_code(int r, int u) {
        return kV + ((((r >> 5) * (D / 64) + (u >> 4)) * 4 + ((r >> 2) & 3)) * 16 + (u & 15)) * 16 + ((r >> 4) & 1) * 8 + (r & 3) * 2;
    }
    static constexpr int k_scale(int r, int block) {
        return kKScale + (((block / kChunkBlocks) * 16 + (r & 15)) * kChunkBlocks + block % kChunkBlocks) * 4 + (r >> 4);
    }
    static constexpr int v_scale(int r, int block) {
        return kVScale + ((((r >> 5) * 4 + ((r >> 2) & 3)) * 2 + (block & 1)) * (D / 64) + (block >> 1)) * 8 + ((r >> 4) & 1) * 4 + (r & 3);
    }
};

inline int64_t page_bytes(const splice_shape &sh) { return (int64_t)sh.n_kv_heads * 68 * sh.head_dim; }

inline int32_t validate_pages(const splice_shape *shape, const splice_pages *pages) {
    const int32_t rc = validate_shape(shape);
    if (rc != SPLICE_OK) return rc;
    if (!pages) return SPLICE_EINVAL;
    if (pages->n_pages < 1 || pages->table_len < 1 || pages->n_tokens < 1) return SPLICE_ESHAPE;
    if (pages->n_pages > 1 << 24 || pages->table_len > 1 << 22 || pages->n_tokens > SPLICE_MAX_PAGE_TOKENS ||
        shape->dtype != SPLICE_BF16 || shape->n_q_heads >= 1 << 16 || shape->n_layers >= 1 << 16)
        return SPLICE_EUNSUPPORTED;
    if (shape->gen_capacity > (int64_t)pages->table_len * kPageRows) return SPLICE_ESHAPE;
    return SPLICE_OK;
}

inline int new_of(const splice_pages &pg, const int32_t *cell_new, int c) { return cell_new ? cell_new[c] : pg.n_tokens; }

// The steps and numbers of new tokens of a call's cells.
inline int32_t validate_page_cells(const splice_shape &sh, const splice_pages &pg, const int32_t *cell_step, const int32_t *cell_new) {
    if (sh.n_cells == 0) return SPLICE_OK;
    if (!cell_step) return SPLICE_EINVAL;
    for (int c = 0; c < sh.n_cells; ++c) {
        if (cell_step[c] < 0) continue;
        const int n = new_of(pg, cell_new, c);
        if (n < 0 || n > pg.n_tokens || cell_step[c] > sh.gen_capacity - n) return SPLICE_ESHAPE;
    }
    return SPLICE_OK;
}

// The cells of a call that have tokens, in order.  Words throughout, as in tree_plan.hpp.
template <int N>
struct PageCells {
    int32_t step[N], count[N];
    uint32_t cell[N];
};

inline int cells_with_tokens(const splice_shape &sh, const splice_pages &pg, const int32_t *cell_step, const int32_t *cell_new) {
    int n = 0;
    for (int c = 0; c < sh.n_cells; ++c) n += cell_step[c] >= 0 && new_of(pg, cell_new, c) > 0;
    return n;
}

template <int N>
void list_page_cells(const splice_shape &sh, const splice_pages &pg, const int32_t *cell_step, const int32_t *cell_new,
                     PageCells<N> &out) {
    int n = 0;
    for (int c = 0; c < sh.n_cells && n < N; ++c)
        if (cell_step[c] >= 0 && new_of(pg, cell_new, c) > 0) {
            out.step[n] = cell_step[c];
            out.count[n] = new_of(pg, cell_new, c);
            out.cell[n++] = (uint32_t)c;
        }
}

// Calls f with (head_dim, room for n cells) as compile-time constants.
constexpr int kPageFewCells = 32;
template <class F>
void with_head_dim(int D, int n, F f) {
    auto room = [&](auto d) {
        if (n <= kPageFewCells) f(d, std::integral_constant<int, kPageFewCells>{});
        else f(d, std::integral_constant<int, SPLICE_MAX_CELLS>{});
    };
    if (D == 64) room(std::integral_constant<int, 64>{});
    else if (D == 128) room(std::integral_constant<int, 128>{});
    else room(std::integral_constant<int, 256>{});
}

}  // namespace splice
