// token_scores.hip -- what logits say about given tokens: log probability,
// log-sum, entropy, rank and the first k alternatives (splice_tree.h).
//
// One pass over a row: a lane keeps the running maximum m of the logits, and with
// z = (logit - m) scale log2(e) the sums s = sum 2^z and t = sum 2^z z; then
//   lse = m scale + ln2 log2 s,   entropy = ln2 (log2 s - t / s).
// When m rises, all z fall by some r: t becomes 2^-r (t - r s) and s 2^-r s.
// (m stays a logit: the lowest float, a usual mask, times log2(e) is no float.)
// The k largest logits, as 64-bit keys (the value's order, then the lower
// index), are the first k of the candidates that each wave keeps in a list in
// LDS: what is below a bound that k keys are not below costs a comparison a 16-byte
// chunk.  The bound comes from all four waves (each tells one that k / 4 of its
// keys are not below), so that together they list k (1 + ln(row / first trip))
// keys rather than four times as many; after the first trip they do not wait for each other.
// 1024 rows of 128256 bf16 logits: 54 us without alternatives (4.8 TB/s), 76 with
// 20 (92 with a bound a wave), 97 with 64 (162).
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
// 16-byte chunks a thread has in flight (us with 2 / 4 / 8: 1024 bf16 rows, k = 20, 79 / 76 / 98; 300 float32
// rows, k = 8, 51 / 48 / 56, k = 0 38 / 41 / 42)
constexpr int kChunks = 4;
constexpr int kMaxParts = 64;
constexpr int kPartBytes = 8 << 10;   // a part is at least this long (7 rows of 600 KB: 12 us; 32 KB 19)
// Work groups that fill the GPU (512 / 1024 / 2048: 300 float32 rows, k = 8, 56 / 48 / 52; 1024 bf16 rows, k = 20, 76 / 76 / 89)
constexpr int kPartsTarget = 1024;
constexpr int kWaveKeys = 256;        // a wave's list
constexpr int kCutKeys = 128;         // one longer than this is cut to its first k
constexpr int kCandidates = 1024;     // a work group's four lists; a row's parts have no more
static_assert(SPLICE_MAX_TOP < kCutKeys && kWaveKeys * kScoreWaves == kCandidates && kScoreWaves == 4, "");

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
__device__ __forceinline__ uint32_t word_of(float x) {
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return x != x ? 0xffffffffu : ((u >> 31) ? ~u : u | 0x80000000u);
}
__device__ __forceinline__ uint64_t key_of(float x, int i) { return ((uint64_t)word_of(x) << 32) | (uint32_t)~i; }
__device__ __forceinline__ float word_value(uint32_t u) { return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ float key_value(uint64_t key) { return word_value((uint32_t)(key >> 32)); }
__device__ __forceinline__ int key_index(uint64_t key) { return (int)~(uint32_t)key; }

// Lists of candidates, in any order; joined, n of them from the start.
struct Candidates {
    uint64_t key[kCandidates];
    uint64_t first[SPLICE_MAX_TOP];   // the first k of the list, in order
    uint64_t least;
    int n;
};

// The need-th largest of the wave's words, N a lane (0: none), with the bits
// below `last` zero: a bound that need words are not below.  Bit by bit, as a
// count of the words above is one comparison and a scalar popcount.
template <int N>
__device__ __forceinline__ uint32_t nth_word(const uint32_t (&u)[N], int need, int last) {
    uint32_t found = 0;
    for (int b = 31; b >= last; --b) {
        const uint32_t x = found | 1u << b;
        int count = 0;
        static_for<0, N>([&](auto i) { count += __popcll(__ballot(u[i] >= x)); });
        if (count >= need) found = x;
    }
    return found;
}
constexpr int kBoundBit = 12;   // of bounds: 20 steps rather than 32

// A wave's list: n keys (the same n in every lane), of which those that find
// room are there.
struct WaveList {
    static constexpr int PER = kWaveKeys / 64;
    uint64_t *key;
    int n;

    __device__ __forceinline__ void append(bool on, uint64_t x) {
        const uint64_t lanes = __ballot(on);
        if (lanes == 0) return;
        const int at = n + __popcll(lanes & ((1ull << (threadIdx.x & 63)) - 1));
        if (on && at < kWaveKeys) key[at] = x;
        n += __popcll(lanes);
    }

    // Entries lane, lane + 64, ... (0 beyond the list's end).
    template <int N>
    __device__ __forceinline__ void entries(uint64_t (&mine)[N]) {
        const int lane = threadIdx.x & 63;
        wave_fence();
        static_for<0, N>([&](auto i) { mine[i] = lane + 64 * (int)i < n ? key[lane + 64 * (int)i] : 0; });
        wave_fence();
    }

    // A bound on the value's word that q keys are not below; 0 of fewer than q.
    __device__ __forceinline__ uint32_t bound(int q) {
        auto of = [&](auto count) {
            uint64_t mine[decltype(count)::value];
            uint32_t u[decltype(count)::value];
            entries(mine);
            static_for<0, decltype(count)::value>([&](auto i) { u[i] = (uint32_t)(mine[i] >> 32); });
            return nth_word(u, q, kBoundBit);
        };
        return n <= 64 ? of(std::integral_constant<int, 1>{}) : of(std::integral_constant<int, PER>{});
    }

    // The k-th key of a list of at least k.
    __device__ __forceinline__ uint64_t kth(int k) {
        uint64_t mine[PER];
        uint32_t u[PER];
        entries(mine);
        static_for<0, PER>([&](auto i) { u[i] = (uint32_t)(mine[i] >> 32); });
        const uint32_t value = nth_word(u, k, 0);
        int above = 0, equal = 0;
        static_for<0, PER>([&](auto i) {
            above += __popcll(__ballot(u[i] > value));
            equal += __popcll(__ballot(u[i] == value));
            u[i] = u[i] == value ? (uint32_t)mine[i] : 0;
        });
        // of several with its value the low words tell
        return (uint64_t)value << 32 | (above + equal > k ? nth_word(u, k - above, 0) : 0);
    }

    // Only those of the first `had` keys that are not below x are left.
    __device__ __forceinline__ void only(int had, uint64_t x) {
        uint64_t mine[PER];
        n = had;
        entries(mine);
        n = 0;
        static_for<0, PER>([&](auto i) { append(mine[i] != 0 && mine[i] >= x, mine[i]); });
    }
};

// What does not fit is left out, and n tells.
__device__ __forceinline__ void append(Candidates &c, uint64_t key) {
    const int at = atomicAdd(&c.n, 1);
    if (at < kCandidates) c.key[at] = key;
}

// first[0..k) = the first k of the list's n entries (0 beyond n), in order: a
// thread counts for each of its entries the larger ones; keys are all
// different.  Called by all threads, after a barrier; ends in one.
__device__ __forceinline__ void rank_first(Candidates &c, int n, int k) {
    constexpr int PER = kCandidates / kScoreThreads;
    const int tid = threadIdx.x;
    uint64_t mine[PER];
    int rank[PER];
    static_for<0, PER>([&](auto i) {
        const int e = tid + (int)i * kScoreThreads;
        mine[i] = e < n ? c.key[e] : ~0ull;
        rank[i] = 0;
    });
    if (tid < k) c.first[tid] = 0;
    __syncthreads();
    if ((tid & ~63) >= n) {
        // no entries in this wave
    } else if (n <= kScoreThreads) {
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank[0] += c.key[j] > mine[0];
    } else {
#pragma unroll 2
        for (int j = 0; j < n; ++j) {
            const uint64_t x = c.key[j];
            static_for<0, PER>([&](auto i) { rank[i] += x > mine[i]; });
        }
    }
    static_for<0, PER>([&](auto i) {
        if (tid + (int)i * kScoreThreads < n && rank[i] < k) c.first[rank[i]] = mine[i];
    });
    __syncthreads();
}

// Where weights are 0 their z, which may be -inf, stops here: 0 times a finite number.
constexpr float kLeastZ = -1e4f;

// z = x scale2 - m scale2 in one operation where |m scale2| is below this: the
// product's rounding, 2^-17 at most, is then what a weight's exponent is off by.
// Beyond, where it grows with m (2^9 for logits of 1e10, weights of 0 or infinity)
// and the product may be no float, x - m comes first.
constexpr float kMostRef = 256.f;

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

template <bool BF16>
__device__ __forceinline__ float logit(const char *row, int i) {
    return BF16 ? bf16_hi((uint32_t)reinterpret_cast<const uint16_t *>(row)[i] << 16) : reinterpret_cast<const float *>(row)[i];
}

// The row's results from its joined sums and its first k keys; in, x: whether
// the token is one of the vocabulary, its logit.  Called by one wave.
__device__ __forceinline__ void finish(const ScoreArgs &a, int64_t row, bool in, float x, float m, float s, float t, int before,
                                       const uint64_t *first) {
    const int lane = threadIdx.x & 63;
    const float log_s = kLn2 * log2f(s);   // -inf for a row of nothing
    if (lane == 0) {
        a.logp[row] = in ? (x - m) * a.scale - log_s : __uint_as_float(0x7fc00000u);
        a.lse[row] = fmaf(m, a.scale, log_s);
        a.entropy[row] = log_s - kLn2 * (t / s);
        a.rank[row] = in ? before : -1;
    }
    if (lane < a.k) {
        const uint64_t key = first[lane];
        a.top[row * a.k + lane] = key_index(key);
        a.top_logp[row * a.k + lane] = (key_value(key) - m) * a.scale - log_s;
    }
}

template <bool BF16>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(ScoreArgs a) {
    constexpr int VE = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;   // values of a chunk, bytes of a value
    __shared__ PartSums s_sums[kScoreWaves];
    __shared__ Candidates s_top;
    __shared__ uint32_t s_bound[kScoreWaves];
    __shared__ int s_count[kScoreWaves];
    const int64_t row = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x % a.parts), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const char *p = a.logits + row * a.stride;
    // 16-byte chunks of the row; what lies before the first boundary and behind
    // the last are single values, which the first and the last part take, one a thread
    int head = (int)(-(uintptr_t)p & 15) / ES;
    head = min(head, a.vocab);
    const int n_chunks = (a.vocab - head) / VE, tail = a.vocab - head - n_chunks * VE;
    const char *base = p + head * ES;
    const int per = (n_chunks + a.parts - 1) / a.parts, c0 = min(part * per, n_chunks), c1 = min(c0 + per, n_chunks);

    u32x4_t w[kChunks];   // the next trip's; the first is on its way while the token's logit is looked up
    auto load = [&](int c) {
        static_for<0, kChunks>([&](auto u) {
            const int j = c + (int)u * kScoreThreads + tid;
            if (j < c1) w[u] = *reinterpret_cast<const u32x4_t *>(base + (int64_t)j * 16);
        });
    };
    load(c0);
    __builtin_amdgcn_sched_barrier(0);

    const int64_t tok = a.tokens[row];
    const bool in = tok >= 0 && tok < a.vocab;
    const int token = in ? (int)tok : 0;
    const float xt = logit<BF16>(p, token);
    const bool xt_nan = xt != xt;
    // before the token x >= xt comes first, behind it x > xt: the former is
    // x > the float below xt (a NaN for -inf: then every value comes first)
    const uint32_t xb = __float_as_uint(xt);
    const float below = xt == 0.f ? __uint_as_float(0x80000001u)
                        : xt == -INFINITY ? __uint_as_float(0x7fc00000u)
                                          : __uint_as_float((xb >> 31) ? xb + 1 : xb - 1);

    float m = -INFINITY, s = 0.f, t = 0.f;
    int before = 0;
    // The candidates: every key that is not below kth, of which k keys of the
    // row (or all that the part has) are not.  Each wave tells a bound that q of its keys are
    // not below, as it rises, and the j-th of the four bounds is one of j q >= k.
    WaveList list{s_top.key + wave * kWaveKeys, 0};
    uint64_t kth = 0;
    float least = -INFINITY;   // its value
    const int q = (a.k + kScoreWaves - 1) / kScoreWaves, j_th = a.k > 0 ? (a.k + q - 1) / q : 0;
    uint32_t told = 0;
    int told_n = 0;            // the list's length then
    auto tell = [&](uint32_t bound) {
        told_n = list.n;
        if (bound <= told) return;
        told = bound;
        if (lane == 0) *(volatile uint32_t *)&s_bound[wave] = bound;
    };
    auto hear = [&]() {
        const int mine = (int)*(volatile uint32_t *)&s_bound[lane & 3];
        uint32_t b[kScoreWaves];
        static_for<0, kScoreWaves>([&](auto i) { b[i] = (uint32_t)__builtin_amdgcn_readlane(mine, i); });
        auto order = [&](int x, int y) {
            const uint32_t hi = max(b[x], b[y]), lo = min(b[x], b[y]);
            b[x] = hi;
            b[y] = lo;
        };
        order(0, 1);
        order(2, 3);
        order(0, 2);
        order(1, 3);
        order(1, 2);
        const uint32_t bound = j_th == 1 ? b[0] : (j_th == 2 ? b[1] : (j_th == 3 ? b[2] : b[3]));
        if (bound > (uint32_t)(kth >> 32)) {
            kth = (uint64_t)bound << 32;
            least = bound < 0x00800000u ? -INFINITY : word_value(bound);   // -inf's word, its low bits cut, is no float's
        }
    };
    auto raise = [&](float top) {   // m to at least top
        if (top > m) {
            const float r = (m - top) * a.scale2, f = fast_exp2(r);
            t = f * fmaf(fmaxf(r, kLeastZ), s, t);
            s *= f;
            m = top;
        }
    };
    auto add = [&](float z) {
        const float e = fast_exp2(z);
        s += e;
        t = fmaf(e, fmaxf(z, kLeastZ), t);
    };

    float single = -INFINITY;
    int single_id = -1;
    if (part == 0 && tid < head) single_id = tid;
    if (part == a.parts - 1 && tid >= 64 && tid - 64 < tail) single_id = a.vocab - tail + tid - 64;
    if (single_id >= 0) {
        single = logit<BF16>(p, single_id);
        raise(single);
        add((single - (m == -INFINITY ? 0.f : m)) * a.scale2);
        before += xt_nan ? single != single && single_id < token
                         : single > xt || single != single || (single == xt && single_id < token);
    }
    if (a.k > 0) list.append(single_id >= 0, key_of(single, single_id));

    for (int c = c0; c < c1; c += kScoreThreads * kChunks) {   // the same trips in every lane
        float x[kChunks][VE], top[kChunks];
        static_for<0, kChunks>([&](auto u) {
            static_for<0, 4>([&](auto i) {
                const uint32_t v = w[u][(int)i];
                if constexpr (BF16) {
                    x[u][2 * i] = bf16_lo(v);
                    x[u][2 * i + 1] = bf16_hi(v);
                } else {
                    x[u][i] = __uint_as_float(v);
                }
            });
        });
        load(c + kScoreThreads * kChunks);
        static_for<0, kChunks>([&](auto u) {
            const int j = c + (int)u * kScoreThreads + tid, id0 = head + j * VE;
            top[u] = -INFINITY;
            if (j < c1) {
                static_for<0, VE>([&](auto i) { top[u] = fmaxf(top[u], x[u][i]); });
                raise(top[u]);
                const float ref = -m * a.scale2;
                if (__any(!(fabsf(ref) < kMostRef))) {
                    const float from = m == -INFINITY ? 0.f : m;
                    static_for<0, VE>([&](auto i) { add((x[u][i] - from) * a.scale2); });
                } else {
                    static_for<0, VE>([&](auto i) { add(fmaf(x[u][i], a.scale2, ref)); });
                }
                if (xt_nan) {
                    static_for<0, VE>([&](auto i) { before += x[u][i] != x[u][i] && id0 + (int)i < token; });
                } else {
                    const float bar = token >= id0 + VE ? below : xt;
                    static_for<0, VE>([&](auto i) { before += !(x[u][i] <= bar); });
                    if (token >= id0 && token < id0 + VE)
                        static_for<0, VE>([&](auto i) { before += x[u][i] == xt && id0 + (int)i < token; });
                }
            }
        });
        if (a.k == 0) continue;
        if (c == c0) {
            // to begin with: the lanes' maxima tell the bounds
            float best = top[0];
            static_for<1, kChunks>([&](auto u) { best = fmaxf(best, top[u]); });
            const uint32_t u[1] = {word_of(best)};
            told = nth_word(u, q, kBoundBit);
            if (lane == 0) s_bound[wave] = told;
            __syncthreads();
        }
        hear();
        for (;;) {
            const int had = list.n;
            static_for<0, kChunks>([&](auto u) {
                const int j = c + (int)u * kScoreThreads + tid;
                const bool any = j < c1 && (!(top[u] < least) || s != s);   // s is a NaN where a logit is
                if (__any(any)) {
                    int id0 = head + j * VE;
                    asm volatile("" : "+v"(id0));   // else every value's id and key are worked out before the loop
                    static_for<0, VE>([&](auto i) {
                        const bool maybe = any && !(x[u][i] < least);
                        if (__any(maybe)) {
                            float y = x[u][i];
                            asm volatile("" : "+v"(y));
                            const uint64_t key = key_of(y, id0 + (int)i);
                            list.append(maybe && key >= kth, key);
                        }
                    });
                }
            });
            if (list.n <= kCutKeys) break;
            const bool again = list.n > kWaveKeys;   // not all found room
            const uint64_t x = list.kth(a.k);
            if (x > kth) {
                kth = x;
                least = key_value(kth);
            }
            list.only(again ? had : list.n, kth);
            if (!again) break;   // else the trip again: its keys that are not below
        }
        if (c + kScoreThreads * kChunks < c1 && list.n >= told_n + (q + 1) / 2) tell(list.bound(q));
    }
    if (a.k > 0) {
        // the waves' lists together
        if (lane == 0) s_count[wave] = list.n;
        __syncthreads();
        if (s_count[0] + s_count[1] + s_count[2] + s_count[3] > kScoreThreads) {
            tell(list.bound(q));
            __syncthreads();
            hear();
        }
        uint64_t mine[WaveList::PER];
        list.entries(mine);
        if (tid == 0) s_top.n = 0;
        __syncthreads();
        static_for<0, WaveList::PER>([&](auto i) { if (mine[i] != 0 && mine[i] >= kth) append(s_top, mine[i]); });
        __syncthreads();
        rank_first(s_top, s_top.n, a.k);
    }

    wave_join(a.scale2, m, s, t, before);
    if (lane == 0) s_sums[wave] = PartSums{m, s, t, before};
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < kScoreWaves; ++w) {
        join(a.scale2, m, s, t, s_sums[w].m, s_sums[w].s, s_sums[w].t);
        before += s_sums[w].before;
    }
    if (a.parts == 1) {
        finish(a, row, in, xt, m, s, t, before, s_top.first);
        return;
    }
    if (lane == 0) a.sums[blockIdx.x] = PartSums{m, s, t, before};
    if (lane < a.k) a.keys[(int64_t)blockIdx.x * a.k + lane] = s_top.first[lane];
}

// Joins the parts of a row, a work group a row.  With q = ceil(k / parts), the
// ceil(k / q)-th of the parts' q-th keys has at least k keys not below it.
template <bool BF16>
__global__ __launch_bounds__(kScoreThreads) void score_join_kernel(ScoreArgs a) {
    __shared__ Candidates s_top;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // all that is read of the row, at once
    const int64_t tok = a.tokens[row];
    PartSums p{-INFINITY, 0.f, 0.f, 0};
    if (lane < a.parts) p = a.sums[row * a.parts + lane];
    const bool in = tok >= 0 && tok < a.vocab;
    const float xt = logit<BF16>(a.logits + row * a.stride, in ? (int)tok : 0);
    if (a.k > 0) {
        constexpr int PER = kCandidates / kScoreThreads;
        const int n = a.parts * a.k, q = (a.k + a.parts - 1) / a.parts;
        uint64_t key[PER];
        static_for<0, PER>([&](auto i) {
            const int e = tid + (int)i * kScoreThreads;
            key[i] = e < n ? a.keys[row * n + e] : 0;
        });
        if (wave == 0) {   // at most 64 parts
            const uint32_t u[1] = {lane < a.parts ? (uint32_t)(a.keys[row * n + lane * a.k + q - 1] >> 32) : 0};
            const uint32_t bound = nth_word(u, (a.k + q - 1) / q, kBoundBit);
            if (lane == 0) {
                s_top.least = (uint64_t)bound << 32;
                s_top.n = 0;
            }
        }
        __syncthreads();
        const uint64_t least = s_top.least;
        static_for<0, PER>([&](auto i) { if (key[i] != 0 && key[i] >= least) append(s_top, key[i]); });
        __syncthreads();
        rank_first(s_top, s_top.n, a.k);
    }
    if (wave != 0) return;
    wave_join(a.scale2, p.m, p.s, p.t, p.before);
    finish(a, row, in, xt, p.m, p.s, p.t, p.before, s_top.first);
}

int parts_of(int64_t rows, int64_t vocab, int k) {
    int64_t parts = (kPartsTarget + rows - 1) / rows;
    const int64_t most = (vocab * 2 + kPartBytes - 1) / kPartBytes;   // in bf16; the same for both types
    parts = parts < most ? parts : most;
    const int fit = k > 0 && kCandidates / k < kMaxParts ? kCandidates / k : kMaxParts;   // of the parts' lists in one
    return (int)(parts < fit ? parts : fit);
}

// (a work group a row: a launch has fewer than 2^32 threads)
bool takes(int64_t rows, int64_t vocab, int32_t k) {
    return rows >= 0 && rows < 1 << 24 && vocab >= 1 && vocab <= 1 << 28 && k >= 0 && k <= SPLICE_MAX_TOP && k <= vocab;
}

}  // namespace

extern "C" {

int64_t splice_token_scores_workspace_bytes(int64_t rows, int64_t vocab, int32_t k) {
    if (!takes(rows, vocab, k)) return SPLICE_ESHAPE;
    if (rows == 0) return 0;
    const int parts = parts_of(rows, vocab, k);
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
    const int parts = parts_of(rows, vocab, k);
    ScoreArgs a{(const char *)logits, tokens, logp, lse, entropy, top_logp, rank, top, (PartSums *)workspace, nullptr,
                row_stride * es, (int)vocab, k, parts, scale, scale * kLog2e};
    if (parts > 1) a.keys = (uint64_t *)((char *)workspace + rows * parts * sizeof(PartSums));
    const dim3 grid((unsigned)(rows * parts));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == SPLICE_BF16) hipLaunchKernelGGL(score_kernel<true>, grid, dim3(kScoreThreads), 0, st, a);
    else hipLaunchKernelGGL(score_kernel<false>, grid, dim3(kScoreThreads), 0, st, a);
    if (parts > 1) {
        if (dtype == SPLICE_BF16) hipLaunchKernelGGL(score_join_kernel<true>, dim3((unsigned)rows), dim3(kScoreThreads), 0, st, a);
        else hipLaunchKernelGGL(score_join_kernel<false>, dim3((unsigned)rows), dim3(kScoreThreads), 0, st, a);
    }
    return hipGetLastError() == hipSuccess ? SPLICE_OK : SPLICE_EHIP;
}

}  // extern "C"
