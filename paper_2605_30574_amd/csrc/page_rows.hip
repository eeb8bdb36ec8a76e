// page_rows.hip -- rows of a cache in 4-bit pages (splice_pages.h): rotated,
// quantised and written (splice_page_append), read back (splice_page_read).

#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "device_common.hpp"
#include "page_format.hpp"
#include "rotary.hpp"

#pragma clang fp contract(off)

namespace {

using namespace splice_dev;
using splice::kPageRows;
using splice::PageCells;
using splice::PageLayout;

constexpr int kRowThreads = 256;
constexpr int kMinExp = -100;   // smallest exponent of a block

typedef __bf16 bf16x8v_t __attribute__((ext_vector_type(8)));
typedef float f32x8v_t __attribute__((ext_vector_type(8)));

template <int CELLS>
struct PageAppendArgs {
    const __bf16 *q, *k, *v;
    __bf16 *q_out;
    uint8_t *pool;
    const int32_t *tables;
    const int64_t *pos;
    const double *freq;
    int64_t q_stride, k_stride, v_stride;
    int T, Hq, Hkv, Tp, half_rotary, interleaved, n_pages, table_len;
    double mscale;
    PageCells<CELLS> cells;
};

// A lane's eight values of a block of 32 (four lanes) to 4-bit codes, the
// lower value of a byte in its low half.  With the block's largest magnitude
// 1.f * 2^b the least e with magnitude <= 6 * 2^e = 1.5 * 2^(e + 2) is b - 2, and one
// more for 1.f above 1.5.  At e = 126 codes above 3 would stand for 2^128: they stop there.
__device__ __forceinline__ uint32_t quantise(const f32x8v_t &x, bool finite, uint8_t &exponent) {
    uint32_t top = 0;
    static_for<0, 8>([&](auto i) { top = max(top, __float_as_uint(x[(int)i]) & 0x7fffffffu); });
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    if (!finite) {   // the row reads back as NaN
        exponent = 255;
        return 0;
    }
    const int e = max((int)(top >> 23) - 129 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0), kMinExp);
    const float f = __uint_as_float((uint32_t)(127 - e) << 23), most = e >= 126 ? 3.f : 6.f;
    float y[8];
    static_for<0, 8>([&](auto i) { y[i] = fminf(fmaxf(x[(int)i] * f, -most), most); });
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
    exponent = (uint8_t)(e + 127);
    return w;
}

// A work group takes one token's rows kRowThreads / LPR at a time (LPR = D / 8
// lanes a row, eight values a lane; a KV head's k and v are one row's work, as an
// infinity or NaN in either makes both NaN): blockIdx.x the token, blockIdx.y the
// rows.  The angles of the token are computed once a work group and shared.  Bound by the bytes of
// q, k and v: 2 cells of 4096 tokens, 32 q heads and 8 KV heads of 128, 173 MB, 35 to 44 us (3.9 to 4.9 TB/s).
template <int D, int CELLS>
__global__ __launch_bounds__(kRowThreads) void page_append_kernel(PageAppendArgs<CELLS> a) {
    using Lay = PageLayout<D>;
    constexpr int LPR = D / 8, ROWS = kRowThreads / LPR;
    __shared__ double2 s_cs[D / 2];
    const int ci = blockIdx.x / a.T, t = blockIdx.x % a.T, tid = threadIdx.x;
    if (t >= a.cells.count[ci]) return;
    const int c = (int)a.cells.cell[ci], row = a.cells.step[ci] + t;
    const int64_t token = (int64_t)c * a.T + t;
    const int page = a.tables[(int64_t)c * a.table_len + row / kPageRows];
    if (tid < a.half_rotary) {
        const double p = a.pos ? (double)a.pos[token] : (double)(a.Tp + row);
        s_cs[tid] = turned(p * (a.freq[tid] * 0.15915494309189533577), a.mscale);   // 1 / (2 pi)
    }
    __syncthreads();
    const int hd = blockIdx.y * ROWS + tid / LPR, l = tid % LPR;
    if (hd >= a.Hq + a.Hkv) return;   // whole rows of lanes
    const bool is_q = hd < a.Hq;
    const int g = is_q ? hd : hd - a.Hq;
    const __bf16 *src = (is_q ? a.q + token * a.q_stride : a.k + token * a.k_stride) + (int64_t)g * D;
    f32x8v_t x = __builtin_convertvector(*reinterpret_cast<const bf16x8v_t *>(src + 8 * l), f32x8v_t);
    const int d = 8 * l, half = a.half_rotary;
    // the lane's eight values, turned: turn(u, w, pair) is u cos + w sin of the pair's angle
    auto rotate = [&](auto turn) {
        if (a.interleaved) {
            static_for<0, 4>([&](auto i) {
                const float u = x[2 * (int)i], w = x[2 * (int)i + 1];
                x[2 * (int)i] = turn(u, -w, d / 2 + (int)i);
                x[2 * (int)i + 1] = turn(w, u, d / 2 + (int)i);
            });
        } else {
            const bool low = d < half;
            const f32x8v_t o = __builtin_convertvector(
                *reinterpret_cast<const bf16x8v_t *>(src + (low ? d + half : d - half)), f32x8v_t);
            const int f = low ? d : d - half;
            static_for<0, 8>([&](auto i) { x[(int)i] = turn(x[(int)i], low ? -o[(int)i] : o[(int)i], f + (int)i); });
        }
    };
    if (d < 2 * half) {
        // keys in 64 bits: the borders of their codes leave fp32's roundings no room.  What lies beyond fp32's range stays finite:
        // its code stops at 3 * 2^126 either way, and it is no infinity
        if (is_q) rotate([&](float u, float w, int pair) { return fmaf(u, (float)s_cs[pair].x, w * (float)s_cs[pair].y); });
        else rotate([&](float u, float w, int pair) {
            const double y = fma((double)u, s_cs[pair].x, (double)w * s_cs[pair].y);
            const float f = odd_float(y);
            return fabsf(f) == INFINITY && fabs(y) < INFINITY ? copysignf(FLT_MAX, f) : f;
        });
    }
    if (is_q) {
        *reinterpret_cast<bf16x8v_t *>(a.q_out + (token * a.Hq + g) * D + d) = __builtin_convertvector(x, bf16x8v_t);
        return;
    }
    const f32x8v_t y = __builtin_convertvector(
        *reinterpret_cast<const bf16x8v_t *>(a.v + token * a.v_stride + (int64_t)g * D + d), f32x8v_t);
    uint32_t top = 0;
    static_for<0, 8>([&](auto i) {
        top = max(top, __float_as_uint(x[(int)i]) & 0x7fffffffu);
        top = max(top, __float_as_uint(y[(int)i]) & 0x7fffffffu);
    });
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const bool finite = top < 0x7f800000u;
    uint8_t ke, ve;
    const uint32_t kw = quantise(x, finite, ke), vw = quantise(y, finite, ve);
    if (page < 0 || page >= a.n_pages) return;
    uint8_t *at = a.pool + ((int64_t)page * a.Hkv + g) * Lay::kBytes;
    const int r = row % kPageRows;
    *reinterpret_cast<uint32_t *>(at + Lay::k_code(r, l)) = kw;
    *reinterpret_cast<uint16_t *>(at + Lay::v_code(r, 2 * l)) = (uint16_t)vw;
    *reinterpret_cast<uint16_t *>(at + Lay::v_code(r, 2 * l + 1)) = (uint16_t)(vw >> 16);
    if (l % 4 == 0) {
        at[Lay::k_scale(r, l / 4)] = ke;
        at[Lay::v_scale(r, l / 4)] = ve;
    }
}

template <int CELLS>
struct PageReadArgs {
    const uint8_t *pool;
    const int32_t *tables;
    __bf16 *rows_k, *rows_v;
    int T, Hkv, n_pages, table_len;
    PageCells<CELLS> cells;
};

// Eight codes with one exponent byte as bf16, each exact.
__device__ __forceinline__ u32x4_t fp4_to_bf16(uint32_t w, uint32_t e) {
    if (e == 255) return u32x4_t{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    const float f = __uint_as_float(e << 23);
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, f, 3))};
}

// A lane reads eight values of K and V of one row: blockIdx.x (cell, KV head),
// blockIdx.y its rows, kRowThreads / LPR at a time.  Bound by the bytes written: the same cells' rows, 42 MB, 11 us
// (3.9 TB/s).
template <int D, int CELLS>
__global__ __launch_bounds__(kRowThreads) void page_read_kernel(PageReadArgs<CELLS> a) {
    using Lay = PageLayout<D>;
    constexpr int LPR = D / 8, ROWS = kRowThreads / LPR;
    const int ci = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, l = threadIdx.x % LPR;
    const int i = blockIdx.y * ROWS + threadIdx.x / LPR;
    if (i >= a.cells.count[ci]) return;
    const int c = (int)a.cells.cell[ci], row = a.cells.step[ci] + i, r = row % kPageRows;
    const int page = a.tables[(int64_t)c * a.table_len + row / kPageRows];
    if (page < 0 || page >= a.n_pages) return;
    const uint8_t *at = a.pool + ((int64_t)page * a.Hkv + g) * Lay::kBytes;
    const uint32_t kw = *reinterpret_cast<const uint32_t *>(at + Lay::k_code(r, l));
    const uint32_t vw = *reinterpret_cast<const uint16_t *>(at + Lay::v_code(r, 2 * l)) |
                        (uint32_t) * reinterpret_cast<const uint16_t *>(at + Lay::v_code(r, 2 * l + 1)) << 16;
    const int64_t to = (((int64_t)c * a.Hkv + g) * a.T + i) * D + 8 * l;
    *reinterpret_cast<u32x4_t *>(a.rows_k + to) = fp4_to_bf16(kw, at[Lay::k_scale(r, l / 4)]);
    *reinterpret_cast<u32x4_t *>(a.rows_v + to) = fp4_to_bf16(vw, at[Lay::v_scale(r, l / 4)]);
}

int32_t launched() { return hipGetLastError() == hipSuccess ? SPLICE_OK : SPLICE_EHIP; }

}  // namespace

extern "C" {

int64_t splice_page_bytes(const splice_shape *shape) {
    const int32_t rc = splice::validate_shape(shape);
    if (rc != SPLICE_OK) return rc;
    return splice::page_bytes(*shape);
}

int32_t splice_page_append(const splice_shape *shape, const splice_pages *pages, const splice_rope *rope,
                           const int32_t *cell_step, const int32_t *cell_new, const int32_t *tables, const int64_t *pos,
                           const double *freq, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                           const void *v, int64_t v_stride, void *q_out, void *pool, void *stream) {
    int32_t rc = splice::validate_pages(shape, pages);
    if (rc != SPLICE_OK) return rc;
    const splice_shape &sh = *shape;
    rc = splice::validate_page_cells(sh, *pages, cell_step, cell_new);
    if (rc != SPLICE_OK) return rc;
    const int D = sh.head_dim;
    if (!rope || (rope->layout != SPLICE_ROPE_HALF && rope->layout != SPLICE_ROPE_INTERLEAVED) || !isfinite(rope->mscale))
        return SPLICE_EINVAL;
    if (rope->rotary_dim < 0 || rope->rotary_dim > D || rope->rotary_dim % 16) return SPLICE_ESHAPE;
    if (sh.n_cells == 0) return SPLICE_OK;
    const int Hq = q || q_out ? sh.n_q_heads : 0;   // none: only rows are written
    if (!tables || !k || !v || !pool || (Hq > 0 && (!q || !q_out)) || (rope->rotary_dim > 0 && !freq)) return SPLICE_EINVAL;
    if (!splice::aligned(tables, 4) || !splice::aligned(pos, 8) || !splice::aligned(freq, 8)) return SPLICE_EINVAL;
    const void *ptrs[] = {q, k, v, q_out, pool};
    for (const void *p : ptrs)
        if (!splice::aligned(p, 16)) return SPLICE_EINVAL;
    const int64_t most = (int64_t)1 << 32;
    if (q_stride < (int64_t)Hq * D || k_stride < (int64_t)sh.n_kv_heads * D ||
        v_stride < (int64_t)sh.n_kv_heads * D || q_stride > most || k_stride > most || v_stride > most || q_stride % 8 ||
        k_stride % 8 || v_stride % 8)
        return SPLICE_ESHAPE;
    if (Hq > 0 && q == q_out && q_stride != (int64_t)Hq * D) return SPLICE_EINVAL;
    const int n = splice::cells_with_tokens(sh, *pages, cell_step, cell_new);
    if (n == 0) return SPLICE_OK;
    const dim3 grid((unsigned)(n * pages->n_tokens),
                    (unsigned)splice::ceil_div(Hq + sh.n_kv_heads, kRowThreads / (D / 8)));
    splice::with_head_dim(D, n, [&](auto d, auto room) {
        PageAppendArgs<decltype(room)::value> a{
            (const __bf16 *)q, (const __bf16 *)k, (const __bf16 *)v, (__bf16 *)q_out, (uint8_t *)pool, tables, pos, freq,
            q_stride, k_stride, v_stride, pages->n_tokens, Hq, sh.n_kv_heads, sh.prompt_len, rope->rotary_dim / 2,
            rope->layout == SPLICE_ROPE_INTERLEAVED, pages->n_pages, pages->table_len, rope->mscale, {}};
        splice::list_page_cells(sh, *pages, cell_step, cell_new, a.cells);
        hipLaunchKernelGGL((page_append_kernel<decltype(d)::value, decltype(room)::value>), grid, dim3(kRowThreads), 0,
                           (hipStream_t)stream, a);
    });
    return launched();
}

int32_t splice_page_read(const splice_shape *shape, const splice_pages *pages, const int32_t *cell_step,
                         const int32_t *cell_new, const int32_t *tables, const void *pool, void *rows_k, void *rows_v,
                         void *stream) {
    int32_t rc = splice::validate_pages(shape, pages);
    if (rc != SPLICE_OK) return rc;
    rc = splice::validate_page_cells(*shape, *pages, cell_step, cell_new);
    if (rc != SPLICE_OK) return rc;
    if (shape->n_cells == 0) return SPLICE_OK;
    if (!tables || !pool || !rows_k || !rows_v || !splice::aligned(tables, 4) || !splice::aligned(pool, 16) ||
        !splice::aligned(rows_k, 16) || !splice::aligned(rows_v, 16))
        return SPLICE_EINVAL;
    const int n = splice::cells_with_tokens(*shape, *pages, cell_step, cell_new);
    if (n == 0) return SPLICE_OK;
    const dim3 grid((unsigned)(n * shape->n_kv_heads),
                    (unsigned)splice::ceil_div(pages->n_tokens, kRowThreads / (shape->head_dim / 8)));
    splice::with_head_dim(shape->head_dim, n, [&](auto d, auto room) {
        PageReadArgs<decltype(room)::value> a{(const uint8_t *)pool, tables, (__bf16 *)rows_k, (__bf16 *)rows_v,
                                              pages->n_tokens, shape->n_kv_heads, pages->n_pages, pages->table_len, {}};
        splice::list_page_cells(*shape, *pages, cell_step, cell_new, a.cells);
        hipLaunchKernelGGL((page_read_kernel<decltype(d)::value, decltype(room)::value>), grid, dim3(kRowThreads), 0,
                           (hipStream_t)stream, a);
    });
    return launched();
}

}  // extern "C"
