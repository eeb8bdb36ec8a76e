// page_tables.hip -- which pages the cells hold (splice_page_fork) and which of
// their rows stay (splice_page_compact), see splice_pages.h.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.hpp"
#include "page_format.hpp"

namespace {

using namespace splice_dev;
using splice::kPageRows;
using splice::PageCells;
using splice::PageLayout;

constexpr int kTableThreads = 1024;
constexpr int kCopyThreads = 256, kCopyUnits = 8;   // 16-byte units a thread of the copy moves
constexpr int kCompactThreads = 256;

struct ForkArgs {
    const int32_t *tables, *refs;
    int32_t *new_tables, *new_refs, *missing, *copied;
    int C, L, n_pages;
    int32_t parent[SPLICE_MAX_CELLS], rows[SPLICE_MAX_CELLS], want[SPLICE_MAX_CELLS];
};

// Counts are added to and read past the first-level cache: other waves change them.
__device__ __forceinline__ void count(int32_t *refs, int page, int by) {
    __hip_atomic_fetch_add(refs + page, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ int counted(const int32_t *refs, int page) {
    return __hip_atomic_load(refs + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void phase() {
    __threadfence();
    __syncthreads();
}

// One work group: counts change with every entry that is another after the
// call, then every cell decides on its last page, then the pages are
// walked from the lowest on and the free ones handed out by their ordinal.
// Whole numbers are added in any order, so the result is one.
__global__ __launch_bounds__(kTableThreads) void fork_kernel(ForkArgs a) {
    __shared__ int s_last[SPLICE_MAX_CELLS], s_start[SPLICE_MAX_CELLS + 1], s_wave[kTableThreads / 64];
    __shared__ uint8_t s_copies[SPLICE_MAX_CELLS];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    auto valid = [&](int page) { return page >= 0 && page < a.n_pages; };
    for (int p = tid; p < a.n_pages; p += kTableThreads) a.new_refs[p] = a.refs[p];
    phase();
    for (int i = tid; i < a.C * a.L; i += kTableThreads) {
        const int c = i / a.L, j = i - c * a.L, from = a.parent[c];
        const bool held = from >= 0 && j < (a.rows[c] + kPageRows - 1) / kPageRows;
        const int old = a.tables[i];
        int now = held ? a.tables[(int64_t)from * a.L + j] : -1;
        if (!valid(now)) now = -1;
        if (!(held && from == c)) {
            if (valid(old)) count(a.new_refs, old, -1);
            if (now >= 0) count(a.new_refs, now, 1);
        }
        a.new_tables[i] = now;
    }
    int held = 0, last = -1;
    if (tid < a.C) {
        held = (a.rows[tid] + kPageRows - 1) / kPageRows;
        if (a.parent[tid] >= 0 && a.rows[tid] % kPageRows) {
            last = a.tables[(int64_t)a.parent[tid] * a.L + held - 1];
            if (!valid(last)) last = -1;
        }
        s_last[tid] = last;
    }
    phase();
    int asks = 0;
    bool copies = false;
    if (tid < a.C) {
        if (last >= 0) {
            int number = 0, first = a.C;
            for (int c = a.C - 1; c >= 0; --c)
                if (s_last[c] == last) {
                    ++number;
                    first = c;
                }
            copies = !(counted(a.new_refs, last) == number && first == tid);
        }
        asks = (copies ? 1 : 0) + max((a.want[tid] + kPageRows - 1) / kPageRows - held, 0);
        s_copies[tid] = copies;
        a.copied[2 * tid] = a.copied[2 * tid + 1] = -1;
        if (copies) a.new_tables[(int64_t)tid * a.L + held - 1] = -1;
    }
    // where the pages that a cell asks for start among those of all
    int before = asks;
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(before, o);
        if (lane >= o) before += x;
    }
    if (lane == 63) s_wave[wave] = before;
    phase();   // ... and every cell has read the counts
    if (copies) count(a.new_refs, last, -1);   // never to zero: another holder is left
    if (tid < a.C) {
        int at = before - asks;
        for (int w = 0; w < wave; ++w) at += s_wave[w];
        s_start[tid] = at;
        if (tid == a.C - 1) s_start[a.C] = at + asks;
    }
    phase();
    const int total = s_start[a.C];
    int found = 0;
    for (int base = 0; base < a.n_pages && found < total; base += kTableThreads) {
        const int p = base + tid;
        const bool is_free = p < a.n_pages && counted(a.new_refs, p) == 0;
        const uint64_t mask = __ballot(is_free);
        __syncthreads();   // s_wave is another tile's until here
        if (lane == 0) s_wave[wave] = __popcll(mask);
        __syncthreads();
        int o = found + __popcll(mask & ((1ull << lane) - 1));
        for (int w = 0; w < kTableThreads / 64; ++w) {
            if (w < wave) o += s_wave[w];
            found += s_wave[w];
        }
        if (is_free && o < total) {
            int c = 0;   // the last cell whose first request is at or before o
            for (int step = SPLICE_MAX_CELLS / 2; step > 0; step >>= 1)
                if (c + step < a.C && s_start[c + step] <= o) c += step;
            const int at = o - s_start[c], h = (a.rows[c] + kPageRows - 1) / kPageRows, slot = h + at - (s_copies[c] ? 1 : 0);
            a.new_tables[(int64_t)c * a.L + slot] = p;
            a.new_refs[p] = 1;
            if (s_copies[c] && at == 0) {
                a.copied[2 * c] = s_last[c];
                a.copied[2 * c + 1] = p;
            }
        }
    }
    if (tid == 0) *a.missing = max(total - found, 0);
}

// Pages copied: blockIdx.x the cell, y a part of the page, z the layer.  None is
// both read and written: a page that is read has a holder, one that is written was free.
__global__ __launch_bounds__(kCopyThreads) void copy_pages_kernel(const int32_t *copied, uint8_t *pool, int64_t layer_stride,
                                                                  int64_t page_bytes) {
    const int from = copied[2 * blockIdx.x], to = copied[2 * blockIdx.x + 1];
    if (from < 0) return;
    uint8_t *layer = pool + (int64_t)blockIdx.z * layer_stride;
    const u32x4_t *src = reinterpret_cast<const u32x4_t *>(layer + from * page_bytes);
    u32x4_t *dst = reinterpret_cast<u32x4_t *>(layer + to * page_bytes);
    const int64_t units = page_bytes / 16, base = (int64_t)blockIdx.y * (kCopyThreads * kCopyUnits) + threadIdx.x;
    u32x4_t w[kCopyUnits];
    static_for<0, kCopyUnits>([&](auto i) {
        if (base + i * kCopyThreads < units) w[i] = src[base + i * kCopyThreads];
    });
    static_for<0, kCopyUnits>([&](auto i) {
        if (base + i * kCopyThreads < units) dst[base + i * kCopyThreads] = w[i];
    });
}

struct CompactArgs {
    uint8_t *pool;
    const int32_t *tables, *keep;
    int64_t layer_stride;
    int T, Hkv, cap, n_pages, table_len;
    PageCells<SPLICE_MAX_CELLS> cells;
};

// A work group moves the rows of one (cell, KV head, layer).  Pages that hold
// kept rows pass through LDS in ascending order, their rows are put where they go in a second page
// there, which is written out when it is full.  A row never moves up and every page is
// in LDS or registers before any page from it on is written, so rows may overlap.
template <int D>
__global__ __launch_bounds__(kCompactThreads) void compact_kernel(CompactArgs a) {
    using Lay = PageLayout<D>;
    constexpr int UNITS = Lay::kBytes / 16, U = (UNITS + kCompactThreads - 1) / kCompactThreads;
    __shared__ __attribute__((aligned(16))) uint8_t s_src[Lay::kBytes], s_dst[Lay::kBytes];
    __shared__ int s_row[kPageRows];
    const int ci = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, tid = threadIdx.x, lane = tid % 64;
    const int c = (int)a.cells.cell[ci], base = a.cells.step[ci];
    const int32_t *keep = a.keep + (int64_t)c * a.T, *table = a.tables + (int64_t)c * a.table_len;
    uint8_t *pool = a.pool + (int64_t)blockIdx.y * a.layer_stride + (int64_t)g * Lay::kBytes;
    const int64_t page_bytes = (int64_t)a.Hkv * Lay::kBytes;
    auto entry = [&](int i) { return i < a.T ? keep[i] : -1; };
    auto page_at = [&](int p) -> uint8_t * {   // of the cell's page p; null where there is none
        const int id = table[p];
        return id >= 0 && id < a.n_pages ? pool + id * page_bytes : nullptr;
    };
    u32x4_t w[U];
    auto load = [&](const uint8_t *at) {
        static_for<0, U>([&](auto i) {
            const int u = tid + i * kCompactThreads;
            if (at && u < UNITS) w[i] = reinterpret_cast<const u32x4_t *>(at)[u];
        });
    };
    // Rows `rows` of the page in s_dst to the cell's page p.
    auto write = [&](int p, uint64_t rows) {
        uint8_t *to = page_at(p);
        if (!to) return;
        if (rows == ~0ull) {
            for (int u = tid; u < UNITS; u += kCompactThreads)
                reinterpret_cast<u32x4_t *>(to)[u] = reinterpret_cast<const u32x4_t *>(s_dst)[u];
            return;
        }
        auto has = [&](int r) { return (rows >> r) & 1; };
        for (int u = tid; u < kPageRows * D / 8; u += kCompactThreads)
            if (const int r = u / (D / 8), i = Lay::k_code(r, u % (D / 8)); has(r))
                *reinterpret_cast<uint32_t *>(to + i) = *reinterpret_cast<const uint32_t *>(s_dst + i);
        for (int u = tid; u < kPageRows * D / 4; u += kCompactThreads)
            if (const int r = u / (D / 4), i = Lay::v_code(r, u % (D / 4)); has(r))
                *reinterpret_cast<uint16_t *>(to + i) = *reinterpret_cast<const uint16_t *>(s_dst + i);
        for (int u = tid; u < kPageRows * Lay::kBlocks; u += kCompactThreads)
            if (const int r = u / Lay::kBlocks, b = u % Lay::kBlocks; has(r)) {
                to[Lay::k_scale(r, b)] = s_dst[Lay::k_scale(r, b)];
                to[Lay::v_scale(r, b)] = s_dst[Lay::v_scale(r, b)];
            }
    };
    int at = 0, before = -1;              // list index of the next row, and the entry before it
    int mine = entry(lane);               // entries at .. at + 63, one a lane of every wave
    uint64_t rows = 0;                    // of the page in s_dst
    const int first = __shfl(mine, 0);
    if (first < 0 || first >= a.cap - base) return;
    int page = (base + first) / kPageRows;
    const uint8_t *src = page_at(page);
    load(src);
    for (;;) {
        // the entries that lie in this page: they ascend, so the first n of the lanes'
        const int up = __shfl_up(mine, 1), prev = lane == 0 ? before : up;
        const bool good = mine >= 0 && mine < a.cap - base && mine > prev;
        const uint64_t in = __ballot(good && (base + mine) / kPageRows == page);
        const int n = ~in ? __builtin_ctzll(~in) : 64;
        const int done = base + at;
        __syncthreads();                  // s_src and s_row are read no more
        if (src) static_for<0, U>([&](auto i) {
            const int u = tid + i * kCompactThreads;
            if (u < UNITS) reinterpret_cast<u32x4_t *>(s_src)[u] = w[i];
        });
        if (tid < n) s_row[tid] = (base + mine) % kPageRows;
        const bool whole = src != nullptr;
        at += n;
        before = __shfl(mine, n - 1);
        mine = entry(at + lane);
        const int next = __shfl(mine, 0);
        const bool more = next > before && next < a.cap - base;
        if (more) {
            page = (base + next) / kPageRows;
            src = page_at(page);
            load(src);
        }
        __syncthreads();
        for (int k = 0; k < n;) {         // as far as the page in s_dst reaches
            const int r0 = (done + k) % kPageRows, m = min(n - k, kPageRows - r0);
            if (whole) {
                for (int u = tid; u < m * (D / 32); u += kCompactThreads) {
                    const int i = u / (D / 32), b = 4 * (u % (D / 32));
                    *reinterpret_cast<u32x4_t *>(s_dst + Lay::k_code(r0 + i, b)) =
                        *reinterpret_cast<const u32x4_t *>(s_src + Lay::k_code(s_row[k + i], b));
                }
                for (int u = tid; u < m * (D / 4); u += kCompactThreads) {
                    const int i = u / (D / 4), b = u % (D / 4);
                    *reinterpret_cast<uint16_t *>(s_dst + Lay::v_code(r0 + i, b)) =
                        *reinterpret_cast<const uint16_t *>(s_src + Lay::v_code(s_row[k + i], b));
                }
                for (int u = tid; u < m * Lay::kBlocks; u += kCompactThreads) {
                    const int i = u / Lay::kBlocks, b = u % Lay::kBlocks;
                    s_dst[Lay::k_scale(r0 + i, b)] = s_src[Lay::k_scale(s_row[k + i], b)];
                    s_dst[Lay::v_scale(r0 + i, b)] = s_src[Lay::v_scale(s_row[k + i], b)];
                }
                rows |= (m == 64 ? ~0ull : (1ull << m) - 1) << r0;
            }
            k += m;
            if (r0 + m == kPageRows || (k == n && !more)) {
                __syncthreads();
                write((done + k - 1) / kPageRows, rows);
                rows = 0;
                __syncthreads();
            }
        }
        if (!more) return;
    }
}

int32_t launched() { return hipGetLastError() == hipSuccess ? SPLICE_OK : SPLICE_EHIP; }

bool pool_ok(const splice_shape &sh, const splice_pages &pg, const void *pool, int64_t layer_stride) {
    return pool && splice::aligned(pool, 16) && layer_stride % 16 == 0 && layer_stride >= 0 &&
           (sh.n_layers == 1 || layer_stride >= (int64_t)pg.n_pages * splice::page_bytes(sh));
}

}  // namespace

extern "C" {

int32_t splice_page_fork(const splice_shape *shape, const splice_pages *pages, const int32_t *parent, const int32_t *rows,
                         const int32_t *want, const int32_t *tables, const int32_t *refs, int32_t *new_tables,
                         int32_t *new_refs, int32_t *missing, int32_t *copied, void *pool, int64_t layer_stride,
                         void *stream) {
    const int32_t rc = splice::validate_pages(shape, pages);
    if (rc != SPLICE_OK) return rc;
    const splice_shape &sh = *shape;
    const int C = sh.n_cells;
    if (C == 0) return SPLICE_OK;
    if (!parent || !rows || !want) return SPLICE_EINVAL;
    bool parts = false;
    for (int c = 0; c < C; ++c) {
        if (parent[c] >= C || rows[c] < 0 || want[c] < rows[c] || want[c] > (int64_t)pages->table_len * kPageRows ||
            (parent[c] < 0 && rows[c] > 0))
            return SPLICE_ESHAPE;
        parts |= rows[c] % kPageRows != 0;
    }
    if ((int64_t)C * pages->table_len > 1 << 30) return SPLICE_EUNSUPPORTED;
    int32_t *const ints[] = {const_cast<int32_t *>(tables), const_cast<int32_t *>(refs), new_tables, new_refs, missing, copied};
    for (const int32_t *p : ints)
        if (!p || !splice::aligned(p, 4)) return SPLICE_EINVAL;
    if (new_tables == tables || new_refs == refs) return SPLICE_EINVAL;
    if (!pool_ok(sh, *pages, pool, layer_stride)) return SPLICE_EINVAL;
    ForkArgs a{tables, refs, new_tables, new_refs, missing, copied, C, pages->table_len, pages->n_pages, {}, {}, {}};
    for (int c = 0; c < C; ++c) {
        a.parent[c] = parent[c];
        a.rows[c] = rows[c];
        a.want[c] = want[c];
    }
    hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kTableThreads), 0, (hipStream_t)stream, a);
    if (int32_t e = launched(); e != SPLICE_OK) return e;
    if (!parts) return SPLICE_OK;   // whole pages only: none is copied
    const int64_t bytes = splice::page_bytes(sh);
    const dim3 grid((unsigned)C, (unsigned)splice::ceil_div(bytes, 16 * kCopyThreads * kCopyUnits), (unsigned)sh.n_layers);
    hipLaunchKernelGGL(copy_pages_kernel, grid, dim3(kCopyThreads), 0, (hipStream_t)stream, copied, (uint8_t *)pool, layer_stride,
                       bytes);
    return launched();
}

int32_t splice_page_compact(const splice_shape *shape, const splice_pages *pages, const int32_t *cell_step,
                            const int32_t *keep, const int32_t *tables, void *pool, int64_t layer_stride, void *stream) {
    const int32_t rc = splice::validate_pages(shape, pages);
    if (rc != SPLICE_OK) return rc;
    const splice_shape &sh = *shape;
    if (sh.n_cells == 0) return SPLICE_OK;
    if (!cell_step) return SPLICE_EINVAL;
    CompactArgs a{(uint8_t *)pool, tables, keep, layer_stride, pages->n_tokens, sh.n_kv_heads, sh.gen_capacity,
                  pages->n_pages, pages->table_len, {}};
    int n = 0;
    for (int c = 0; c < sh.n_cells; ++c) {
        if (cell_step[c] > sh.gen_capacity) return SPLICE_ESHAPE;
        if (cell_step[c] < 0) continue;
        a.cells.step[n] = cell_step[c];
        a.cells.cell[n++] = (uint32_t)c;
    }
    if (!keep || !tables || !splice::aligned(keep, 4) || !splice::aligned(tables, 4) || !pool_ok(sh, *pages, pool, layer_stride))
        return SPLICE_EINVAL;
    if (n == 0) return SPLICE_OK;
    const dim3 grid((unsigned)(n * sh.n_kv_heads), (unsigned)sh.n_layers);
    hipStream_t st = (hipStream_t)stream;
    if (sh.head_dim == 64) hipLaunchKernelGGL(compact_kernel<64>, grid, dim3(kCompactThreads), 0, st, a);
    else if (sh.head_dim == 128) hipLaunchKernelGGL(compact_kernel<128>, grid, dim3(kCompactThreads), 0, st, a);
    else hipLaunchKernelGGL(compact_kernel<256>, grid, dim3(kCompactThreads), 0, st, a);
    return launched();
}

}  // extern "C"
