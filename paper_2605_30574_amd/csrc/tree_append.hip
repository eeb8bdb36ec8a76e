// tree_append.hip -- the rows of a tree's nodes in the generated caches
// (splice_tree.h): rotated, rounded or quantised and written
// (splice_tree_append), read back (splice_tree_read), moved together
// (splice_tree_keep).

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "device_common.hpp"
#include "kv_format.hpp"
#include "tree_plan.hpp"

#pragma clang fp contract(off)

namespace {

using namespace splice_dev;
using splice::TreeCells;

constexpr int kAppendThreads = 256;
constexpr int kMinExp = -100;   // smallest exponent of an 8-bit row

typedef __bf16 bf16x8v_t __attribute__((ext_vector_type(8)));
typedef float f32x8v_t __attribute__((ext_vector_type(8)));

template <int CELLS>
struct AppendArgs {
    const __bf16 *q, *k, *v;
    __bf16 *q_out;
    char *gk, *gv;
    uint8_t *gke, *gve;
    const int32_t *depth;
    const int64_t *pos;
    const double *freq;
    int64_t q_stride, k_stride, v_stride;
    int T, Hq, Hkv, cap, Tp, half_rotary, interleaved;
    double mscale;
    TreeCells<CELLS> cells;
};

// Eight values of a cache row to 8-bit codes: x 2^-e, to the nearest, ties to
// even.  bits: the row's largest magnitude, as an unsigned word (a NaN is
// above every number).  With magnitude 1.f * 2^b the least e with
// magnitude <= 448 * 2^e = 1.75 * 2^(e + 8) is b - 8, and one more for 1.f
// above 1.75.  At e = 120 codes above 240 would stand for 2^128: they stop there.
__device__ __forceinline__ uint2 quantise(const f32x8v_t &x, uint32_t bits, uint8_t &exponent) {
    const int b = (int)(bits >> 23) - 127;
    if (b == 128) {   // an infinity or NaN: the row reads back as NaN
        exponent = 127;
        return make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
    }
    const int e = max(b - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), kMinExp);
    const float f = __uint_as_float((uint32_t)(127 - e) << 23), most = e >= 120 ? 240.f : 448.f;
    float y[8];
    static_for<0, 8>([&](auto i) { y[i] = fminf(fmaxf(x[(int)i] * f, -most), most); });
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    exponent = (uint8_t)(e + 127);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// (cos, sin) of so many turns, times a factor.  To the nearest quarter turn,
// then the series of sine and cosine on [-pi / 4, pi / 4], whose first term
// left out is below 2^-33.
__device__ __forceinline__ double2 turned(double turns, double factor) {
    turns -= rint(turns);
    const double n = rint(4. * turns);
    const double x = (turns - 0.25 * n) * 6.28318530717958647693, y = x * x;
    double sn = 1. / 39916800., cs = -1. / 3628800.;
    sn = fma(-sn, y, 1. / 362880.);
    cs = fma(cs, y, 1. / 40320.);
    sn = fma(sn, y, -1. / 5040.);
    cs = fma(cs, y, -1. / 720.);
    sn = fma(sn, y, 1. / 120.);
    cs = fma(cs, y, 1. / 24.);
    sn = fma(sn, y, -1. / 6.);
    cs = fma(cs, y, -1. / 2.);
    sn = fma(sn * y, x, x);
    cs = fma(cs, y, 1.);
    const int k = (int)n & 3;   // quarters
    const double c = k & 1 ? sn : cs, s = k & 1 ? cs : sn;
    return make_double2((k == 1 || k == 2 ? -c : c) * factor, (k & 2 ? -s : s) * factor);
}

// x in 32 bits so that a further rounding, to an 8-bit code, is that of x
// itself: of the two floats beside an inexact x the one with an odd last bit.
__device__ __forceinline__ float odd_float(double x) {
    const float f = (float)x;
    const double rest = x - (double)f;
    uint32_t b = __float_as_uint(f);
    if ((rest > 0. || rest < 0.) && !(b & 1) && fabsf(f) < INFINITY) b += (rest > 0.) != (x < 0.) ? 1 : -1;
    return __uint_as_float(b);
}

// A work group takes one node's heads kAppendThreads / LPR at a time (LPR = D / 8
// lanes a head row, eight values a lane): blockIdx.x the node, blockIdx.y the
// heads.  The angles of the node are computed once a work group and shared.  Launch and
// two rounds of loads (the depth, the row) bound it at few nodes, 3.6 us for 32
// tokens; the rows' bytes at many: 128 cells of 33 nodes, 32 + 2 x 8 heads of 128
// to an 8-bit cache, 95 MB in 26.8 us (3.5 TB/s; on the same inputs again, partly still
// cached, 21.6, and 19.2 with the keys rotated in 32 bits).
template <int D, bool F8, int CELLS>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs<CELLS> a) {
    constexpr int LPR = D / 8, ROWS = kAppendThreads / LPR;
    __shared__ float2 s_cs[D / 2];
    __shared__ double2 s_cs64[F8 ? D / 2 : 1];   // for the keys of an 8-bit cache
    const int ci = blockIdx.x / a.T, t = blockIdx.x % a.T, tid = threadIdx.x;
    const int c = (int)a.cells.cell[ci], step = a.cells.step[ci];
    const int64_t token = (int64_t)c * a.T + t;
    const int depth = a.depth[token];
    if (depth < 0) return;   // padding
    if (tid < a.half_rotary) {
        const double p = a.pos ? (double)a.pos[token] : (double)(a.Tp + step) + (double)min(depth, a.T - 1);
        const double2 cs = turned(p * (a.freq[tid] * 0.15915494309189533577), a.mscale);   // 1 / (2 pi)
        s_cs[tid] = make_float2((float)cs.x, (float)cs.y);
        if constexpr (F8) s_cs64[tid] = cs;
    }
    __syncthreads();
    const int hd = blockIdx.y * ROWS + tid / LPR, l = tid % LPR;
    if (hd >= a.Hq + 2 * a.Hkv) return;   // whole rows of lanes
    const bool is_q = hd < a.Hq, is_v = hd >= a.Hq + a.Hkv;
    const int g = is_q ? hd : (is_v ? hd - a.Hq - a.Hkv : hd - a.Hq);
    const __bf16 *src = (is_q ? a.q + token * a.q_stride : (is_v ? a.v + token * a.v_stride : a.k + token * a.k_stride)) +
                        (int64_t)g * D;
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
    if (!is_v && d < 2 * half) {
        // in 64 bits where an 8-bit code comes of it: its borders leave fp32's roundings no room
        if (F8 && !is_q) rotate([&](float u, float w, int pair) {
            const double2 cs = s_cs64[F8 ? pair : 0];
            return odd_float(fma((double)u, cs.x, (double)w * cs.y));
        });
        else rotate([&](float u, float w, int pair) { return fmaf(u, s_cs[pair].x, w * s_cs[pair].y); });
    }
    if (is_q) {
        *reinterpret_cast<bf16x8v_t *>(a.q_out + (token * a.Hq + g) * D + d) = __builtin_convertvector(x, bf16x8v_t);
        return;
    }
    const int64_t row = ((int64_t)c * a.Hkv + g) * a.cap + step + t;
    char *cache = is_v ? a.gv : a.gk;
    if constexpr (F8) {
        uint32_t top = 0;
        static_for<0, 8>([&](auto i) { top = max(top, __float_as_uint(x[(int)i]) & 0x7fffffffu); });
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        uint8_t e;
        const uint2 codes = quantise(x, top, e);
        *reinterpret_cast<uint2 *>(cache + row * D + d) = codes;
        if (l == 0) (is_v ? a.gve : a.gke)[row] = e;
    } else {
        *reinterpret_cast<bf16x8v_t *>(cache + (row * D + d) * 2) = __builtin_convertvector(x, bf16x8v_t);
    }
}

template <int CELLS>
struct RowsArgs {
    char *gk, *gv;
    uint8_t *gke, *gve;
    __bf16 *rows_k, *rows_v;
    const int32_t *keep;
    int T, Hkv, cap;
    TreeCells<CELLS> cells;
};

// One thread reads eight values of one row: blockIdx.x (active cell, KV head),
// blockIdx.y K or V.  Bound by its bytes: the rows of those 128 x 33 nodes,
// 26 MB in 6.6 us (5.2 where they are still cached).
template <int D, bool F8, int CELLS>
__global__ __launch_bounds__(kAppendThreads) void read_kernel(RowsArgs<CELLS> a) {
    constexpr int LPR = D / 8;
    const int ci = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv;
    const int64_t pair = (int64_t)a.cells.cell[ci] * a.Hkv + g, row0 = pair * a.cap + a.cells.step[ci];
    const char *cache = blockIdx.y ? a.gv : a.gk;
    const uint8_t *ex = blockIdx.y ? a.gve : a.gke;
    __bf16 *dst = (blockIdx.y ? a.rows_v : a.rows_k) + pair * a.T * D;
    for (int u = threadIdx.x; u < a.T * LPR; u += kAppendThreads) {
        const int64_t row = row0 + u / LPR;
        const int d = 8 * (u % LPR);
        u32x4_t w;
        if constexpr (F8) {
            const uint2 codes = *reinterpret_cast<const uint2 *>(cache + row * D + d);
            w = e4m3_to_bf16(codes, ex[row]);
        } else {
            w = *reinterpret_cast<const u32x4_t *>(cache + (row * D + d) * 2);
        }
        *reinterpret_cast<u32x4_t *>(dst + (int64_t)u * 8) = w;
    }
}

// Moves rows keep[0], keep[1], ... of one (cell, KV head, K or V) to rows
// 0, 1, ...: a work group loads all that move, waits until every load
// has come back, then stores, so that rows may overlap without a copy
// elsewhere.  A row's exponent moves with its first unit.  Launch and two
// rounds of memory bound it: 128 cells of 8 heads, up to 64 rows of 128
// bytes, 17 MB in 5.1 us (3.3 TB/s, 1.5 times a copy's time).
template <int ROW, bool F8, int CELLS>
__global__ __launch_bounds__(kAppendThreads) void keep_kernel(RowsArgs<CELLS> a) {
    constexpr int LPR = ROW / 16, U = SPLICE_MAX_NODES * LPR / kAppendThreads;
    __shared__ int s_from[SPLICE_MAX_NODES];
    const int ci = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, tid = threadIdx.x, lane = tid & 63;
    const int c = (int)a.cells.cell[ci];
    const int64_t row0 = ((int64_t)c * a.Hkv + g) * a.cap + a.cells.step[ci];
    char *cache = blockIdx.y ? a.gv : a.gk;
    uint8_t *ex = blockIdx.y ? a.gve : a.gke;
    // the list ends at the first entry that does not ascend within 0..T-1
    const int from = lane < a.T ? a.keep[(int64_t)c * a.T + lane] : -1;
    const int last = __shfl_up(from, 1);
    const uint64_t bad = __ballot(!(from >= 0 && from < a.T && (lane == 0 || from > last)));
    const int n = bad ? __builtin_ctzll(bad) : 64;
    if (tid < 64) s_from[tid] = from;
    __syncthreads();
    u32x4_t w[U];
    uint8_t e[U];
    static_for<0, U>([&](auto i) {
        const int u = tid + (int)i * kAppendThreads, r = u / LPR, b = u % LPR;
        if (r < n) {
            const int64_t row = row0 + s_from[r];
            w[i] = *reinterpret_cast<const u32x4_t *>(cache + row * ROW + 16 * b);
            if (F8 && b == 0) e[i] = ex[row];
        }
    });
    // every load of the group is back before any of its stores: rows overlap
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    static_for<0, U>([&](auto i) {
        const int u = tid + (int)i * kAppendThreads, r = u / LPR, b = u % LPR;
        if (r < n && s_from[r] != r) {
            *reinterpret_cast<u32x4_t *>(cache + (row0 + r) * ROW + 16 * b) = w[i];
            if (F8 && b == 0) ex[row0 + r] = e[i];
        }
    });
}

int32_t launched() { return hipGetLastError() == hipSuccess ? SPLICE_OK : SPLICE_EHIP; }

bool caches_ok(const splice_tree &tree, const void *gk, const void *gv, const void *gke, const void *gve) {
    if (!gk || !gv || !splice::aligned(gk, 16) || !splice::aligned(gv, 16)) return false;
    const bool f8 = tree.kv_format == SPLICE_KV_E4M3;
    return f8 ? gke && gve : !gke && !gve;
}

}  // namespace

extern "C" {

int32_t splice_tree_append(const splice_shape *shape, const splice_tree *tree, const splice_rope *rope,
                           const int32_t *cell_step, const int32_t *depth, const int64_t *pos, const double *freq,
                           const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                           int64_t v_stride, void *q_out, void *gen_k, void *gen_v, uint8_t *gen_k_exp,
                           uint8_t *gen_v_exp, void *stream) {
    int32_t rc = splice::validate_tree(shape, tree, cell_step);
    if (rc != SPLICE_OK) return rc;
    const splice_shape &sh = *shape;
    const int D = sh.head_dim;
    if (!rope || (rope->layout != SPLICE_ROPE_HALF && rope->layout != SPLICE_ROPE_INTERLEAVED) || !isfinite(rope->mscale))
        return SPLICE_EINVAL;
    if (rope->rotary_dim < 0 || rope->rotary_dim > D || rope->rotary_dim % 16) return SPLICE_ESHAPE;
    if (sh.n_cells == 0) return SPLICE_OK;
    if (!depth || !q || !k || !v || !q_out || (rope->rotary_dim > 0 && !freq)) return SPLICE_EINVAL;
    if (!splice::aligned(depth, 4) || !splice::aligned(pos, 8) || !splice::aligned(freq, 8)) return SPLICE_EINVAL;
    const void *ptrs[] = {q, k, v, q_out};
    for (const void *p : ptrs)
        if (!splice::aligned(p, 16)) return SPLICE_EINVAL;
    if (!caches_ok(*tree, gen_k, gen_v, gen_k_exp, gen_v_exp)) return SPLICE_EINVAL;
    const int64_t most = (int64_t)1 << 32;
    if (q_stride < (int64_t)sh.n_q_heads * D || k_stride < (int64_t)sh.n_kv_heads * D ||
        v_stride < (int64_t)sh.n_kv_heads * D || q_stride > most || k_stride > most || v_stride > most || q_stride % 8 ||
        k_stride % 8 || v_stride % 8)
        return SPLICE_ESHAPE;
    if (q == q_out && q_stride != (int64_t)sh.n_q_heads * D) return SPLICE_EINVAL;
    const int n = splice::active_cells(sh, cell_step);
    if (n == 0) return SPLICE_OK;
    const int rows = kAppendThreads / (D / 8);
    const dim3 grid((unsigned)(n * tree->n_nodes), (unsigned)splice::ceil_div(sh.n_q_heads + 2 * sh.n_kv_heads, rows));
    splice::with_format(D, tree->kv_format, n, [&](auto d, auto f8, auto room) {
        AppendArgs<decltype(room)::value> a{
            (const __bf16 *)q, (const __bf16 *)k, (const __bf16 *)v, (__bf16 *)q_out, (char *)gen_k, (char *)gen_v,
            gen_k_exp, gen_v_exp, depth, pos, freq, q_stride, k_stride, v_stride, tree->n_nodes, sh.n_q_heads,
            sh.n_kv_heads, sh.gen_capacity, sh.prompt_len, rope->rotary_dim / 2,
            rope->layout == SPLICE_ROPE_INTERLEAVED, rope->mscale, {}};
        splice::list_cells(sh, cell_step, a.cells);
        hipLaunchKernelGGL((append_kernel<decltype(d)::value, decltype(f8)::value, decltype(room)::value>), grid,
                           dim3(kAppendThreads), 0, (hipStream_t)stream, a);
    });
    return launched();
}

int32_t splice_tree_read(const splice_shape *shape, const splice_tree *tree, const int32_t *cell_step, const void *gen_k,
                         const void *gen_v, const uint8_t *gen_k_exp, const uint8_t *gen_v_exp, void *rows_k,
                         void *rows_v, void *stream) {
    int32_t rc = splice::validate_tree(shape, tree, cell_step);
    if (rc != SPLICE_OK) return rc;
    if (shape->n_cells == 0) return SPLICE_OK;
    if (!rows_k || !rows_v || !splice::aligned(rows_k, 16) || !splice::aligned(rows_v, 16) ||
        !caches_ok(*tree, gen_k, gen_v, gen_k_exp, gen_v_exp))
        return SPLICE_EINVAL;
    const int n = splice::active_cells(*shape, cell_step);
    if (n == 0) return SPLICE_OK;
    const dim3 grid((unsigned)(n * shape->n_kv_heads), 2);
    splice::with_format(shape->head_dim, tree->kv_format, n, [&](auto d, auto f8, auto room) {
        RowsArgs<decltype(room)::value> a{
            (char *)const_cast<void *>(gen_k), (char *)const_cast<void *>(gen_v), const_cast<uint8_t *>(gen_k_exp),
            const_cast<uint8_t *>(gen_v_exp), (__bf16 *)rows_k, (__bf16 *)rows_v, nullptr, tree->n_nodes,
            shape->n_kv_heads, shape->gen_capacity, {}};
        splice::list_cells(*shape, cell_step, a.cells);
        hipLaunchKernelGGL((read_kernel<decltype(d)::value, decltype(f8)::value, decltype(room)::value>), grid,
                           dim3(kAppendThreads), 0, (hipStream_t)stream, a);
    });
    return launched();
}

int32_t splice_tree_keep(const splice_shape *shape, const splice_tree *tree, const int32_t *cell_step,
                         const int32_t *keep, void *gen_k, void *gen_v, uint8_t *gen_k_exp, uint8_t *gen_v_exp,
                         void *stream) {
    int32_t rc = splice::validate_tree(shape, tree, cell_step);
    if (rc != SPLICE_OK) return rc;
    if (shape->n_cells == 0) return SPLICE_OK;
    if (!keep || !splice::aligned(keep, 4) || !caches_ok(*tree, gen_k, gen_v, gen_k_exp, gen_v_exp)) return SPLICE_EINVAL;
    const int n = splice::active_cells(*shape, cell_step);
    if (n == 0) return SPLICE_OK;
    const dim3 grid((unsigned)(n * shape->n_kv_heads), 2);
    splice::with_format(shape->head_dim, tree->kv_format, n, [&](auto d, auto f8, auto room) {
        constexpr int ROW = decltype(d)::value * (decltype(f8)::value ? 1 : 2);
        RowsArgs<decltype(room)::value> a{(char *)gen_k, (char *)gen_v, gen_k_exp, gen_v_exp, nullptr, nullptr, keep,
                                          tree->n_nodes, shape->n_kv_heads, shape->gen_capacity, {}};
        splice::list_cells(*shape, cell_step, a.cells);
        hipLaunchKernelGGL((keep_kernel<ROW, decltype(f8)::value, decltype(room)::value>), grid, dim3(kAppendThreads), 0,
                           (hipStream_t)stream, a);
    });
    return launched();
}

}  // extern "C"
