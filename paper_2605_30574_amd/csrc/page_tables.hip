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

// The pages' counts: in LDS where they have room there, else in new_refs, which other waves' additions
// reach past the first-level cache.
constexpr int kLdsPages = 12288;
template <bool LDS>
struct Counts {
    int32_t *refs;
    __device__ __forceinline__ void add(int page, int by) const {
        if constexpr (LDS) atomicAdd(refs + page, by);
        else __hip_atomic_fetch_add(refs + page, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __device__ __forceinline__ int of(int page) const {
        if constexpr (LDS) return refs[page];
        else return __hip_atomic_load(refs + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __device__ __forceinline__ void phase() const {
        if constexpr (!LDS) __threadfence();
        __syncthreads();
    }
};

// One work group: counts change with every entry that is another after the
// call, then every cell decides on its last page, then the pages are
// walked from the lowest on and the free ones handed out by their ordinal.
// Whole numbers are added in any order, so the result is one.  Its chain of memory round trips and
// barriers bounds it: 128 cells of 16 entries forked in the middle of a page, 4098 pages, 11.6 us.  Forked behind
// full pages, in a replayed graph, they take 7.0 us with 4098 pages and 8.0 with 12288, whose counts are in
// LDS; with the counts in memory 25 with 12289 pages and 40 with 131072.
template <bool LDS>
__global__ __launch_bounds__(kTableThreads) void fork_kernel(ForkArgs a) {
    extern __shared__ int32_t s_refs[];
    __shared__ int s_last[SPLICE_MAX_CELLS], s_start[SPLICE_MAX_CELLS + 1], s_wave[kTableThreads / 64];
    __shared__ int s_parent[SPLICE_MAX_CELLS], s_held[SPLICE_MAX_CELLS];
    __shared__ uint8_t s_copies[SPLICE_MAX_CELLS];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const Counts<LDS> counts{LDS ? s_refs : a.new_refs};
    auto valid = [&](int page) { return page >= 0 && page < a.n_pages; };
    for (int p = tid; p < a.n_pages; p += kTableThreads) counts.refs[p] = a.refs[p];
    int held = 0, last = -1, asks = 0;
    if (tid < a.C) {
        const int rows = a.rows[tid], parent = a.parent[tid];
        held = (rows + kPageRows - 1) / kPageRows;
        asks = max((a.want[tid] + kPageRows - 1) / kPageRows - held, 0);
        if (parent >= 0 && rows % kPageRows) {
            last = a.tables[(int64_t)parent * a.L + held - 1];
            if (!valid(last)) last = -1;
        }
        s_parent[tid] = parent;
        s_held[tid] = held;
        s_last[tid] = last;
        a.copied[2 * tid] = a.copied[2 * tid + 1] = -1;
    }
    counts.phase();
    for (int i = tid; i < a.C * a.L; i += kTableThreads) {
        const int c = i / a.L, j = i - c * a.L, from = s_parent[c];
        const bool in = from >= 0 && j < s_held[c];
        const int old = a.tables[i];
        int now = in ? a.tables[(int64_t)from * a.L + j] : -1;
        if (!valid(now)) now = -1;
        if (!(in && from == c)) {
            if (valid(old)) counts.add(old, -1);
            if (now >= 0) counts.add(now, 1);
        }
        a.new_tables[i] = now;
    }
    counts.phase();
    bool copies = false;
    if (last >= 0) {
        int number = 0, first = a.C;
        for (int c = a.C - 1; c >= 0; --c)
            if (s_last[c] == last) {
                ++number;
                first = c;
            }
        copies = !(counts.of(last) == number && first == tid);
    }
    if (copies) {
        ++asks;
        a.new_tables[(int64_t)tid * a.L + held - 1] = -1;
    }
    if (tid < a.C) s_copies[tid] = copies;
    // where the pages that a cell asks for start among those of all
    int before = asks;
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(before, o);
        if (lane >= o) before += x;
    }
    if (lane == 63) s_wave[wave] = before;
    counts.phase();   // ... and every cell has read the counts
    if (copies) counts.add(last, -1);   // never to zero: another holder is left
    if (tid < a.C) {
        int at = before - asks;
        for (int w = 0; w < wave; ++w) at += s_wave[w];
        s_start[tid] = at;
        if (tid == a.C - 1) s_start[a.C] = at + asks;
    }
    counts.phase();
    const int total = s_start[a.C];
    int found = 0;
    constexpr int EACH = 4;   // consecutive pages a thread looks at
    for (int base = 0; base < a.n_pages && found < total; base += kTableThreads * EACH) {
        const int p0 = base + tid * EACH;
        int free = 0;   // a bit a page
        static_for<0, EACH>([&](auto i) {
            if (p0 + i < a.n_pages && counts.of(p0 + i) == 0) free |= 1 << i;
        });
        const int mine = __popc(free);
        int upto = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            if (lane >= o) upto += x;
        }
        __syncthreads();   // s_wave is another tile's until here
        if (lane == 63) s_wave[wave] = upto;
        __syncthreads();
        int o = found + upto - mine;
        for (int w = 0; w < kTableThreads / 64; ++w) {
            if (w < wave) o += s_wave[w];
            found += s_wave[w];
        }
        static_for<0, EACH>([&](auto i) {
            if ((free >> i & 1) && o < total) {
                const int p = p0 + i;
                int c = 0;   // the last cell whose first request is at or before o
                for (int step = SPLICE_MAX_CELLS / 2; step > 0; step >>= 1)
                    if (c + step < a.C && s_start[c + step] <= o) c += step;
                const int at = o - s_start[c], slot = s_held[c] + at - (s_copies[c] ? 1 : 0);
                a.new_tables[(int64_t)c * a.L + slot] = p;
                counts.refs[p] = 1;
                if (s_copies[c] && at == 0) {
                    a.copied[2 * c] = s_last[c];
                    a.copied[2 * c + 1] = p;
                }
                ++o;
            }
        });
    }
    if (tid == 0) *a.missing = max(total - found, 0);
    if constexpr (LDS) {
        __syncthreads();
        for (int p = tid; p < a.n_pages; p += kTableThreads) a.new_refs[p] = s_refs[p];
    }
}

// Pages copied: blockIdx.x the cell, y a part of the page, z the layer.  None is
// both read and written: a page that is read has a holder, one that is written was free.
// Bound by the bytes written: one page of 8 heads of 128 to 127 cells in 36 layers, 318 MB, 72 us
// (4.4 TB/s; the page that is read stays in the caches).
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

// A work group moves the rows of one (cell, KV head, layer).  Pages that hold kept rows pass through LDS in
// ascending order; every thread has its share of the page that is being put together in registers, in the order of
// the page's bytes, and takes what of it lies in the page in LDS, so that a full page goes out in whole lines.  A row
// never moves up and every page is in LDS or registers before any page from it on is written, so
// rows may overlap.  Bound by the bytes of the pages that it reads and writes: every second row of 15 cells' 4096,
// 8 heads of 128, 8 layers, 0.8 GB in 208 us (3.9 TB/s; with the page put together in LDS too 222).
template <int D>
__global__ __launch_bounds__(kCompactThreads) void compact_kernel(CompactArgs a) {
    using Lay = PageLayout<D>;
    constexpr int UNITS = Lay::kBytes / 16, U = (UNITS + kCompactThreads - 1) / kCompactThreads;
    constexpr int SHARES = 2 * D, S = (SHARES + kCompactThreads - 1) / kCompactThreads;   // of 16 bytes of K, of V; of one byte of their scales
    __shared__ __attribute__((aligned(16))) uint8_t s_page[Lay::kBytes];
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
    // the thread's share n: of K and of the scales row r and piece b, of V value piece u and rows r0 + 16 e + f
    auto row_of = [&](int n) { return (tid + n * kCompactThreads) / Lay::kBlocks; };
    auto piece_of = [&](int n) { return (tid + n * kCompactThreads) % Lay::kBlocks; };
    auto value_row = [&](int n) { const int x = tid + n * kCompactThreads; return x / (D) * 32 + x / 16 % 4 * 4; };
    auto value_unit = [&](int n) { const int x = tid + n * kCompactThreads; return x / 64 % (D / 64) * 16 + x % 16; };
    auto mine = [&](int n) { return SHARES % kCompactThreads == 0 || tid + n * kCompactThreads < SHARES; };
    u32x4_t kw[S], vw[S];
    uint8_t ks[S], vs[S];
    // Rows r0 .. r0 + m - 1 of the page that is put together are rows s_row[k], ... of the one in LDS.
    auto take = [&](int r0, int m, int k) {
        static_for<0, S>([&](auto n) {
            if (!mine(n)) return;
            const int r = row_of(n) - r0, b = piece_of(n);
            if (r >= 0 && r < m) {
                const int from = s_row[k + r];
                kw[n] = *reinterpret_cast<const u32x4_t *>(s_page + Lay::k_code(from, 4 * b));
                ks[n] = s_page[Lay::k_scale(from, b)];
                vs[n] = s_page[Lay::v_scale(from, b)];
            }
            const int first = value_row(n) - r0, u = value_unit(n);
            static_for<0, 8>([&](auto j) {
                const int i = first + 16 * (j / 4) + j % 4;
                if (i >= 0 && i < m) {
                    const uint32_t x = *reinterpret_cast<const uint16_t *>(s_page + Lay::v_code(s_row[k + i], u));
                    vw[n][(int)(j / 2)] = j % 2 ? (vw[n][(int)(j / 2)] & 0xffffu) | x << 16 : (vw[n][(int)(j / 2)] & 0xffff0000u) | x;
                }
            });
        });
    };
    // Rows `rows` of it to the cell's page p.
    auto write = [&](int p, uint64_t rows) {
        uint8_t *to = page_at(p);
        if (!to) return;
        static_for<0, S>([&](auto n) {
            if (!mine(n)) return;
            const int x = tid + n * kCompactThreads, r = row_of(n), b = piece_of(n);
            if (rows >> r & 1) {
                *reinterpret_cast<u32x4_t *>(to + 16 * x) = kw[n];
                to[Lay::k_scale(r, b)] = ks[n];
                to[Lay::v_scale(r, b)] = vs[n];
            }
            if (rows == ~0ull) {
                *reinterpret_cast<u32x4_t *>(to + Lay::kV + 16 * x) = vw[n];
                return;
            }
            static_for<0, 8>([&](auto j) {
                if (rows >> (value_row(n) + 16 * (j / 4) + j % 4) & 1)
                    *reinterpret_cast<uint16_t *>(to + Lay::kV + 16 * x + 2 * j) = (uint16_t)(vw[n][(int)(j / 2)] >> (16 * (j % 2)));
            });
        });
    };
    int at = 0, before = -1;              // list index of the next row, and the entry before it
    int kept = entry(lane);               // entries at .. at + 63, one a lane of every wave
    uint64_t rows = 0;                    // of the page that is put together
    const int first = __shfl(kept, 0);
    if (first < 0 || first >= a.cap - base) return;
    int page = (base + first) / kPageRows;
    const uint8_t *src = page_at(page);
    load(src);
    for (;;) {
        // the entries that lie in this page: they ascend, so the first n of the lanes'
        const int up = __shfl_up(kept, 1), prev = lane == 0 ? before : up;
        const bool good = kept >= 0 && kept < a.cap - base && kept > prev;
        const uint64_t in = __ballot(good && (base + kept) / kPageRows == page);
        const int n = ~in ? __builtin_ctzll(~in) : 64;
        const int done = base + at;
        __syncthreads();                  // s_page and s_row are read no more
        if (src) static_for<0, U>([&](auto i) {
            const int u = tid + i * kCompactThreads;
            if (u < UNITS) reinterpret_cast<u32x4_t *>(s_page)[u] = w[i];
        });
        if (tid < n) s_row[tid] = (base + kept) % kPageRows;
        const bool there = src != nullptr;
        at += n;
        before = __shfl(kept, n - 1);
        kept = entry(at + lane);
        const int next = __shfl(kept, 0);
        const bool more = next > before && next < a.cap - base;
        if (more) {
            page = (base + next) / kPageRows;
            src = page_at(page);
            load(src);
        }
        __syncthreads();
        for (int k = 0; k < n;) {         // as far as the page that is put together reaches
            const int r0 = (done + k) % kPageRows, m = min(n - k, kPageRows - r0);
            if (there) {
                take(r0, m, k);
                rows |= (m == 64 ? ~0ull : (1ull << m) - 1) << r0;
            }
            k += m;
            if (r0 + m == kPageRows || (k == n && !more)) {
                write((done + k - 1) / kPageRows, rows);
                rows = 0;
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
    if (pages->n_pages <= kLdsPages)
        hipLaunchKernelGGL(fork_kernel<true>, dim3(1), dim3(kTableThreads), pages->n_pages * sizeof(int32_t), (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(fork_kernel<false>, dim3(1), dim3(kTableThreads), 0, (hipStream_t)stream, a);
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
