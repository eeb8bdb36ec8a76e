// page_attn.hip -- host side of splice_page_attn (splice_pages.h): checks, plan,
// launch.  The kernels are in page_attn.hpp, one unit per head_dim.

#include "page_attn.hpp"

using splice_dev::PageArgs;

namespace {

// Compute units of the current device (256 when HIP cannot tell: the plan then still holds, it only
// balances for that many).
int compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) {
        (void)hipGetLastError();
        return 256;
    }
    if (dev < 64 && (n = known[dev].load()) > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) {
        (void)hipGetLastError();
        return 256;
    }
    if (dev < 64) known[dev].store(n);
    return n;
}

int32_t check_call(const splice_shape &sh, const splice_call *call) {
    if (!call) return SPLICE_EINVAL;
    splice_call checked = *call;
    checked.step = 0;   // every token takes its own step
    const int32_t rc = splice::validate_call(sh, &checked);
    if (rc != SPLICE_OK) return rc;
    return isfinite(call->scale * splice_dev::kLog2e) ? SPLICE_OK : SPLICE_EINVAL;
}

}  // namespace

extern "C" {

int64_t splice_page_attn_workspace_bytes(const splice_shape *shape, const splice_call *call, const splice_pages *pages) {
    int32_t rc = splice::validate_pages(shape, pages);
    if (rc != SPLICE_OK) return rc;
    rc = check_call(*shape, call);
    if (rc != SPLICE_OK) return rc;
    return splice::page_most_parts(*shape, *pages) * splice::page_part_bytes(*shape, *pages);
}

int32_t splice_page_attn(const splice_shape *shape, const splice_call *call, const splice_pages *pages,
                         const int32_t *cell_LW, const int32_t *cell_step, const int32_t *cell_new, const int32_t *tables,
                         const int32_t *clean_table, const int32_t *donor_table, const void *q, const void *pool, void *out,
                         float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    int32_t rc = splice::validate_pages(shape, pages);
    if (rc != SPLICE_OK) return rc;
    const splice_shape &sh = *shape;
    rc = check_call(sh, call);
    if (rc != SPLICE_OK) return rc;
    rc = splice::validate_page_cells(sh, *pages, cell_step, cell_new);
    if (rc != SPLICE_OK) return rc;
    rc = splice::validate_cells(sh, cell_LW);
    if (rc != SPLICE_OK) return rc;
    if (sh.n_cells == 0) return SPLICE_OK;
    const bool zero = sh.donor_kind == SPLICE_DONOR_ZERO, has_prompt = sh.prompt_len > 0;
    if (!tables || !q || !pool || !out || !lse || (has_prompt && !clean_table)) return SPLICE_EINVAL;
    if (zero ? donor_table != nullptr : has_prompt && !donor_table) return SPLICE_EINVAL;
    const void *wide[] = {q, pool, out}, *words[] = {tables, clean_table, donor_table, lse};
    for (const void *p : wide)
        if (!splice::aligned(p, 16)) return SPLICE_EINVAL;
    for (const void *p : words)
        if (!splice::aligned(p, 4)) return SPLICE_EINVAL;

    splice::PageCell cells[SPLICE_MAX_CELLS];
    int n = 0, most_count = 0;
    for (int c = 0; c < sh.n_cells; ++c) {
        const int count = cell_step[c] >= 0 ? splice::new_of(*pages, cell_new, c) : 0;
        if (count == 0) continue;
        // tokens before the onset are not spliced
        const int64_t before = call->layer >= cell_LW[2 * c] ? (int64_t)cell_LW[2 * c + 1] - cell_step[c] : count;
        cells[n++] = {c, cell_step[c], count, (int)std::min<int64_t>(count, std::max<int64_t>(0, before))};
        most_count = std::max(most_count, count);
    }
    if (n == 0) return SPLICE_OK;
    const splice::PagePlan p = splice::page_plan(sh, *call, *pages, cells, n, compute_units());
    // a launch has fewer than 2^32 threads along x, the join a wave a row
    if (p.blocks >= (int64_t)1 << 24 || p.own_tiles >= 1 << 24 || (p.parts > 1 && (int64_t)most_count * sh.n_q_heads >= (int64_t)1 << 26))
        return SPLICE_EUNSUPPORTED;
    if (p.bytes > 0 && (!workspace || !splice::aligned(workspace, 256) || workspace_bytes < (size_t)p.bytes)) return SPLICE_EWORKSPACE;
    PageArgs args;
    int tile = 0;
    const int G = splice::group_of(sh);
    for (int i = 0; i < n; ++i) {
        const splice::PageCell &c = cells[i];
        args.step[i] = (uint32_t)c.step;
        args.count_split[i] = (uint32_t)c.count | (uint32_t)c.split << 16;
        args.cell_tile[i] = (uint32_t)c.cell << 24 | (uint32_t)tile;
        const int split = p.shared ? c.count : c.split;
        tile += splice::ceil_div(split * G, p.own_rows) + splice::ceil_div((c.count - split) * G, p.own_rows);
    }
    splice_dev::PageCall &a = args.call;
    a.q = (const char *)q;
    a.pool = (const uint8_t *)pool;
    a.tables = tables;
    a.clean = clean_table;
    a.donor = donor_table;
    a.out = (__bf16 *)out;
    a.lse = lse;
    a.part = (float *)workspace;
    a.part_stride = splice::page_part_bytes(sh, *pages) / 4;
    a.C = sh.n_cells;
    a.T = pages->n_tokens;
    a.G = G;
    a.Hkv = sh.n_kv_heads;
    a.Tp = sh.prompt_len;
    a.span_lo = sh.span_lo;
    a.span_hi = sh.span_hi;
    a.window = call->window;
    a.zero_donor = zero ? 1 : 0;
    a.n_pages = pages->n_pages;
    a.table_len = pages->table_len;
    a.n_active = n;
    a.shared = p.shared ? 1 : 0;
    a.own_rows = p.own_rows;
    a.own_each = p.own_each;
    a.own_per = p.own_per;
    a.own_parts = p.own_parts;
    a.rows_u = p.rows_u;
    a.tiles_u = p.tiles_u;
    a.tiles_s = p.tiles_s;
    a.prompt_per = p.prompt_per;
    a.prompt_parts = p.prompt_parts;
    a.parts = p.parts;
    a.qk_scale = call->scale * splice_dev::kLog2e;
    hipStream_t st = (hipStream_t)stream;
    const bool ok = sh.head_dim == 64    ? splice_dev::launch_page_attn_d64(args, p, most_count, st)
                    : sh.head_dim == 128 ? splice_dev::launch_page_attn_d128(args, p, most_count, st)
                                         : splice_dev::launch_page_attn_d256(args, p, most_count, st);
    return ok ? SPLICE_OK : SPLICE_EHIP;
}

}  // extern "C"
