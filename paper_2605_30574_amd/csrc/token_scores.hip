// token_scores.hip -- what logits say about given tokens: log probability,
// log-sum, entropy, rank and the first k alternatives (splice_tree.h).
//
// One pass over a row: a lane keeps the running maximum m of the logits, and with
// z = (logit - m) scale log2(e) the sums s = sum 2^z and t = sum 2^z z; then
//   lse = m scale + ln2 log2 s,   entropy = ln2 (log2 s - t / s).
// When m rises, all z fall by some r: t becomes 2^-r (t - r s) and s 2^-r s.
// (m stays a logit: the lowest float, a usual mask, times log2(e) is no float.)  The k largest
// logits are kept sorted in a wave, one a lane, as 64-bit keys (the value's
// order, then the lower index); a logit below the k-th costs one comparison.
// A row is cut into parts when there are too few rows for the GPU, and a
// second kernel joins the parts' sums and lists.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "device_common.hpp"
#include "splice_tree.h"

namespace {

using namespace splice_dev;

constexpr int kScoreThreads = 256;
constexpr int kScoreWaves = kScoreThreads / 64;
constexpr int kChunks = 4;            // 16-byte chunks a thread has in flight
constexpr int kMaxParts = 64;
constexpr int kPartBytes = 16 << 10;  // a part is at least this long
constexpr int kPartsTarget = 2048;    // work groups that fill the GPU

struct PartSums {
    float m, s, t;
    int32_t before;   // tokens that come before the given one
};

struct ScoreArgs {
    const char *logits;
    const int64_t *tokens;
    float *logp, *lse, *entropy, *top_logp;
    int64_t *rank, *top;
    PartSums *sums;
    uint64_t *keys;
    int64_t stride;   // bytes from row to row
    int vocab, k, parts;
    float scale, scale2;   // scale; scale * log2(e)
};

// Orders floats as unsigned words, NaN above everything, -0 as 0; the low word
// makes the lower index the larger key.  No key is 0.
__device__ __forceinline__ uint64_t key_of(float x, int i) {
    uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    u = x != x ? 0xffffffffu : ((u >> 31) ? ~u : u | 0x80000000u);
    return ((uint64_t)u << 32) | (uint32_t)~i;
}
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return u == 0xffffffffu ? __uint_as_float(0x7fc00000u) : __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(uint64_t key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ uint64_t lane_value(uint64_t x, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, lane);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
    return ((uint64_t)hi << 32) | lo;
}

// The first k of all keys offered to a wave: lane i holds the i-th largest.
struct TopList {
    uint64_t key = 0;   // this lane's
    uint64_t least = 0; // the k-th
    int k;

    __device__ __forceinline__ explicit TopList(int k) : k(k) {}

    // Every lane of the wave offers one key (0: none).
    __device__ __forceinline__ void offer(uint64_t x) {
        const int lane = threadIdx.x & 63;
        uint64_t todo = __ballot(x > least);
        while (todo) {
            const int from = __builtin_ctzll(todo);
            const uint64_t y = lane_value(x, from);
            const int at = __popcll(__ballot(key > y));
            const uint64_t up = __shfl_up((unsigned long long)key, 1);
            key = lane < at ? key : (lane == at ? y : up);
            least = lane_value(key, k - 1);
            todo &= todo - 1;
            todo &= __ballot(x > least);
        }
    }
};

// Where weights are 0 their z, which may be -inf, stops here: 0 times a finite number.
constexpr float kLeastZ = -1e4f;

// Joins (m, s, t) of two parts of a row.
__device__ __forceinline__ void join(float scale2, float &m, float &s, float &t, float m2, float s2, float t2) {
    const float mm = fmaxf(m, m2), ref = mm == -INFINITY ? 0.f : mm;
    const float r1 = (m - ref) * scale2, r2 = (m2 - ref) * scale2;
    const float f1 = fast_exp2(r1), f2 = fast_exp2(r2);
    t = f1 * fmaf(fmaxf(r1, kLeastZ), s, t) + f2 * fmaf(fmaxf(r2, kLeastZ), s2, t2);
    s = f1 * s + f2 * s2;
    m = mm;
}

__device__ __forceinline__ void wave_join(float scale2, float &m, float &s, float &t, int &before) {
    for (int o = 32; o > 0; o >>= 1) {
        join(scale2, m, s, t, __shfl_xor(m, o), __shfl_xor(s, o), __shfl_xor(t, o));
        before += __shfl_xor(before, o);
    }
}

// The row's results from its joined sums; called by one wave.
template <bool BF16>
__device__ __forceinline__ void finish(const ScoreArgs &a, int64_t row, float m, float s, float t, int before,
                                       const TopList &list) {
    const int lane = threadIdx.x & 63;
    const float log_s = kLn2 * log2f(s);   // -inf for a row of nothing
    if (lane == 0) {
        const int64_t tok = a.tokens[row];
        const bool in = tok >= 0 && tok < a.vocab;
        float x = 0.f;
        if (in) {
            const char *p = a.logits + row * a.stride;
            x = BF16 ? bf16_hi((uint32_t)reinterpret_cast<const uint16_t *>(p)[tok] << 16) : reinterpret_cast<const float *>(p)[tok];
        }
        a.logp[row] = in ? (x - m) * a.scale - log_s : __uint_as_float(0x7fc00000u);
        a.lse[row] = fmaf(m, a.scale, log_s);
        a.entropy[row] = log_s - kLn2 * (t / s);
        a.rank[row] = in ? before : -1;
    }
    if (lane < a.k) {
        a.top[row * a.k + lane] = key_index(list.key);
        a.top_logp[row * a.k + lane] = (key_value(list.key) - m) * a.scale - log_s;
    }
}

template <bool BF16>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(ScoreArgs a) {
    constexpr int VE = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;   // values of a chunk, bytes of a value
    __shared__ PartSums s_sums[kScoreWaves];
    __shared__ uint64_t s_keys[kScoreWaves][64];
    const int64_t row = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x % a.parts), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const char *p = a.logits + row * a.stride;
    // 16-byte chunks from the last boundary at or below the row's start
    const int skew = (int)((uintptr_t)p & 15) / ES;
    const char *base = p - skew * ES;
    const int n_chunks = (int)(((int64_t)skew + a.vocab + VE - 1) / VE);
    const int per = (n_chunks + a.parts - 1) / a.parts, c0 = part * per, c1 = min(c0 + per, n_chunks);

    const int64_t tok = a.tokens[row];
    const bool in = tok >= 0 && tok < a.vocab;
    const int token = in ? (int)tok : 0;
    const float xt = BF16 ? bf16_hi((uint32_t)reinterpret_cast<const uint16_t *>(p)[token] << 16)
                          : reinterpret_cast<const float *>(p)[token];
    // before the token x >= xt comes first, behind it x > xt: the former is
    // x > the float below xt (a NaN for -inf: then every value comes first)
    const uint32_t xb = __float_as_uint(xt);
    const float below = xt == 0.f ? __uint_as_float(0x80000001u)
                        : xt == -INFINITY ? __uint_as_float(0x7fc00000u)
                                          : __uint_as_float((xb >> 31) ? xb + 1 : xb - 1);

    float m = -INFINITY, s = 0.f, t = 0.f;
    int before = 0;
    TopList list(a.k);
    float least = -INFINITY;

    for (int c = c0; c < c1; c += kScoreThreads * kChunks) {   // the same trips in every lane
        float x[kChunks][VE];
        static_for<0, kChunks>([&](auto u) {
            const int j = c + (int)u * kScoreThreads + tid, id0 = j * VE - skew;
            if (j < c1 && id0 >= 0 && id0 + VE <= a.vocab) {
                const u32x4_t w = *reinterpret_cast<const u32x4_t *>(base + (int64_t)j * 16);
                static_for<0, 4>([&](auto i) {
                    const uint32_t v = w[(int)i];
                    if constexpr (BF16) {
                        x[u][2 * i] = bf16_lo(v);
                        x[u][2 * i + 1] = bf16_hi(v);
                    } else {
                        x[u][i] = __uint_as_float(v);
                    }
                });
            } else {
                static_for<0, VE>([&](auto i) {   // a row's ends: only what is its own is read
                    const int id = id0 + (int)i;
                    x[u][i] = -INFINITY;
                    if (j < c1 && id >= 0 && id < a.vocab)
                        x[u][i] = BF16 ? bf16_hi((uint32_t)reinterpret_cast<const uint16_t *>(p)[id] << 16)
                                       : reinterpret_cast<const float *>(p)[id];
                });
            }
        });
        static_for<0, kChunks>([&](auto u) {
            const int j = c + (int)u * kScoreThreads + tid, id0 = j * VE - skew;
            float top = x[u][0];
            static_for<1, VE>([&](auto i) { top = fmaxf(top, x[u][i]); });
            if (top > m) {
                const float r = (m - top) * a.scale2, f = fast_exp2(r);
                t = f * fmaf(fmaxf(r, kLeastZ), s, t);
                s *= f;
                m = top;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            static_for<0, VE>([&](auto i) {
                const float z = (x[u][i] - ref) * a.scale2, e = fast_exp2(z);
                s += e;
                t = fmaf(e, fmaxf(z, kLeastZ), t);
            });
            if (xt == xt && id0 >= 0 && j < c1 && id0 + VE <= a.vocab && (token < id0 || token >= id0 + VE)) {
                const float bar = token >= id0 ? below : xt;
                static_for<0, VE>([&](auto i) { before += !(x[u][i] <= bar); });
            } else if (j < c1) {
                static_for<0, VE>([&](auto i) {
                    const int id = id0 + (int)i;
                    const float y = x[u][i];
                    const bool first = xt == xt ? (y > xt || y != y || (y == xt && id < token)) : (y != y && id < token);
                    before += id >= 0 && id < a.vocab && first;
                });
            }
            if (a.k > 0) {
                bool any = false;
                static_for<0, VE>([&](auto i) { any |= !(x[u][i] < least); });
                if (__any(any)) {
                    static_for<0, VE>([&](auto i) {
                        const int id = id0 + (int)i;
                        list.offer(j < c1 && id >= 0 && id < a.vocab ? key_of(x[u][i], id) : 0);
                    });
                    least = list.least ? key_value(list.least) : -INFINITY;
                }
            }
        });
    }

    wave_join(a.scale2, m, s, t, before);
    s_keys[wave][lane] = list.key;
    if (lane == 0) s_sums[wave] = PartSums{m, s, t, before};
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < kScoreWaves; ++w) {
        join(a.scale2, m, s, t, s_sums[w].m, s_sums[w].s, s_sums[w].t);
        before += s_sums[w].before;
        if (a.k > 0) list.offer(s_keys[w][lane]);
    }
    if (a.parts == 1) {
        finish<BF16>(a, row, m, s, t, before, list);
        return;
    }
    if (lane == 0) a.sums[blockIdx.x] = PartSums{m, s, t, before};
    if (lane < a.k) a.keys[(int64_t)blockIdx.x * a.k + lane] = list.key;
}

// Joins the parts of a row: one wave a row.
template <bool BF16>
__global__ __launch_bounds__(64) void score_join_kernel(ScoreArgs a) {
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    float m = -INFINITY, s = 0.f, t = 0.f;
    int before = 0;
    if (lane < a.parts) {
        const PartSums p = a.sums[row * a.parts + lane];
        m = p.m;
        s = p.s;
        t = p.t;
        before = p.before;
    }
    wave_join(a.scale2, m, s, t, before);
    TopList list(a.k);
    const int n = a.parts * a.k;
    for (int i = 0; i < n; i += 64) list.offer(i + lane < n ? a.keys[row * n + i + lane] : 0);
    finish<BF16>(a, row, m, s, t, before, list);
}

int parts_of(int64_t rows, int64_t vocab) {
    int64_t parts = (kPartsTarget + rows - 1) / rows;
    const int64_t most = (vocab * 2 + kPartBytes - 1) / kPartBytes;   // in bf16; the same for both types
    parts = parts < most ? parts : most;
    return (int)(parts < kMaxParts ? parts : kMaxParts);
}

bool takes(int64_t rows, int64_t vocab, int32_t k) {
    return rows >= 0 && rows <= 1 << 24 && vocab >= 1 && vocab <= 1 << 28 && k >= 0 && k <= SPLICE_MAX_TOP && k <= vocab;
}

}  // namespace

extern "C" {

int64_t splice_token_scores_workspace_bytes(int64_t rows, int64_t vocab, int32_t k) {
    if (!takes(rows, vocab, k)) return SPLICE_ESHAPE;
    if (rows == 0) return 0;
    const int parts = parts_of(rows, vocab);
    return parts == 1 ? 0 : rows * parts * ((int64_t)sizeof(PartSums) + 8 * k);
}

int32_t splice_token_scores(const void *logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                            float scale, const int64_t *tokens, int32_t k, float *logp, float *lse, float *entropy,
                            int64_t *rank, int64_t *top, float *top_logp, void *workspace, size_t workspace_bytes,
                            void *stream) {
    if (dtype != SPLICE_BF16 && dtype != SPLICE_F32) return SPLICE_EINVAL;
    const int64_t need = splice_token_scores_workspace_bytes(rows, vocab, k);
    if (need < 0) return (int32_t)need;
    if (!isfinite(scale) || !(scale > 0.f) || !isfinite(scale * kLog2e)) return SPLICE_EINVAL;
    if (row_stride < vocab || row_stride > (int64_t)1 << 32) return SPLICE_ESHAPE;
    if (rows == 0) return SPLICE_OK;
    const int es = dtype == SPLICE_BF16 ? 2 : 4;
    if (!logits || !tokens || !logp || !lse || !entropy || !rank || (k > 0 && (!top || !top_logp))) return SPLICE_EINVAL;
    if (!splice::aligned(logits, es) || !splice::aligned(tokens, 8) || !splice::aligned(logp, 4) ||
        !splice::aligned(lse, 4) || !splice::aligned(entropy, 4) || !splice::aligned(rank, 8) ||
        !splice::aligned(top, 8) || !splice::aligned(top_logp, 4))
        return SPLICE_EINVAL;
    if (need > 0 && (!workspace || !splice::aligned(workspace, 16) || workspace_bytes < (size_t)need))
        return SPLICE_EWORKSPACE;
    const int parts = parts_of(rows, vocab);
    ScoreArgs a{(const char *)logits, tokens, logp, lse, entropy, top_logp, rank, top, (PartSums *)workspace, nullptr,
                row_stride * es, (int)vocab, k, parts, scale, scale * kLog2e};
    if (parts > 1) a.keys = (uint64_t *)((char *)workspace + rows * parts * sizeof(PartSums));
    const dim3 grid((unsigned)(rows * parts));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == SPLICE_BF16) hipLaunchKernelGGL(score_kernel<true>, grid, dim3(kScoreThreads), 0, st, a);
    else hipLaunchKernelGGL(score_kernel<false>, grid, dim3(kScoreThreads), 0, st, a);
    if (parts > 1) {
        if (dtype == SPLICE_BF16) hipLaunchKernelGGL(score_join_kernel<true>, dim3((unsigned)rows), dim3(64), 0, st, a);
        else hipLaunchKernelGGL(score_join_kernel<false>, dim3((unsigned)rows), dim3(64), 0, st, a);
    }
    return hipGetLastError() == hipSuccess ? SPLICE_OK : SPLICE_EHIP;
}

}  // extern "C"
