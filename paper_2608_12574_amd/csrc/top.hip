// The k best tokens of each row of logits, with their log probabilities.
//
// Mathematics.  lse = m + log sum_v exp(x_v - m) for any m; parts summed under their own maxima join the same way.  The best
// tokens are the largest of the keys (logit, lowest token first), which are all different.  For any partition of the logits the
// k-th largest of the parts' maxima is no larger than the k-th largest logit, so only logits from there on can be among the best.
//
// k_top: a block holds a span of a row in registers, read once.  Each thread finds its maximum and its sum; the k-th largest of
// the maxima of 64 or 256 groups of threads (found by one wave, which cuts the range of values) leaves few more than k
// candidates, which go to LDS and are ranked by counting.  Where thousands equal the bound, the first tokens of them are counted
// off (rows of zeros: 92 us for 33); where thousands are above it, the k-th key itself is found, in a turn through the span per bit.
// k_top_join: the spans' best, in the same way, and the sum of the sums.
// The bytes bound a large call, with the exponentials (a quarter of the rate) close behind: 256 bf16 rows over V = 262,144, 8 of
// each, 134 MB in 29 to 30.5 us (4.4 to 4.6 TB/s), 24 without looking for the best; the join 4 to 5.  A row of 32,000 is a chain of barriers in
// one block, 8 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"

namespace tam {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;
constexpr float kLog2e = 1.4426950408889634f;

// The order of logits, as unsigned integers: -0 and 0 alike, NaN above all.
__device__ inline uint32_t order_of(float x) {
    uint32_t bits = __float_as_uint(x);
    if (bits == 0x80000000u) bits = 0;
    if (x != x) bits = 0x7FFFFFFFu;
    return bits ^ ((bits & 0x80000000u) ? 0xFFFFFFFFu : 0x80000000u);
}

__device__ inline float logit_of(uint32_t order) { return __uint_as_float(order ^ ((order & 0x80000000u) ? 0x80000000u : 0xFFFFFFFFu)); }

constexpr uint32_t kNone = 0x007FFFFFu;  // the order of -inf

// Keys: the order in the upper half, then the lowest token first.  0: no token.
__device__ inline uint64_t key_of(float x, uint32_t token) { return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - token); }

// How a type's logits lie in a 16-byte vector.
template <typename T>
struct In;

template <>
struct In<float> {
    static constexpr int n = 4;
    static constexpr uint32_t kMinusInf = 0xFF800000u;  // a word of it
    static __device__ float get(u32x4 x, int i) { return __uint_as_float(x[i]); }
    static __device__ void drop(u32x4 &x, int i) { x[i] = kMinusInf; }
    static __device__ float load(const float *p) { return *p; }
};

template <>
struct In<uint16_t> {  // bf16
    static constexpr int n = 8;
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
    static __device__ float get(u32x4 x, int i) { return __uint_as_float(i & 1 ? x[i >> 1] & 0xFFFF0000u : x[i >> 1] << 16); }
    static __device__ void drop(u32x4 &x, int i) { x[i >> 1] = i & 1 ? (x[i >> 1] & 0xFFFFu) | 0xFF800000u : (x[i >> 1] & 0xFFFF0000u) | 0xFF80u; }
    static __device__ float load(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
};

// A sum of exponentials under their maximum.
struct Sum {
    float m, s;
};

__device__ inline Sum join(Sum a, Sum b) {
    const float m = fmaxf(a.m, b.m);
    const float f = a.m == m ? 1.f : __builtin_amdgcn_exp2f((a.m - m) * kLog2e), g = b.m == m ? 1.f : __builtin_amdgcn_exp2f((b.m - m) * kLog2e);
    return Sum{m, a.s * f + b.s * g};  // (a NaN in s stays)
}

// Of all threads, in a fixed order.
template <int kThreads>
__device__ inline Sum join_block(Sum x) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ Sum waves[kWaves];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x = join(x, Sum{__shfl_xor(x.m, d), __shfl_xor(x.s, d)});
    if (kWaves == 1) return x;
    if (threadIdx.x % kWave == 0) waves[threadIdx.x / kWave] = x;
    __syncthreads();
    x = waves[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) x = join(x, waves[w]);
    return x;
}

__device__ inline float log_of(Sum x) { return x.s == 0.f ? -INFINITY : x.m + logf(x.s); }

template <int kThreads>
__device__ inline int count_block(int mine) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ int waves[kWaves];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) mine += __shfl_xor(mine, d);
    if (kWaves == 1) return mine;
    __syncthreads();
    if (threadIdx.x % kWave == 0) waves[threadIdx.x / kWave] = mine;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += waves[w];
    return all;
}

// Sum over the threads before this one, and over all of them.
template <int kThreads>
__device__ inline int before_block(int mine, int *total) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ int waves[kWaves];
    int upto = mine;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int up = __shfl_up(upto, d);
        if ((int)threadIdx.x % kWave >= d) upto += up;
    }
    __syncthreads();
    if (threadIdx.x % kWave == kWave - 1) waves[threadIdx.x / kWave] = upto;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < (int)threadIdx.x / kWave) upto += waves[w];
        all += waves[w];
    }
    *total = all;
    return upto - mine;
}

// The k-th largest of the lanes' kPer values each, or a value under it that few more reach (kReach(k) at most where all are
// different); `low` if no more reach that.  X: an unsigned integer.  The range is cut into four in each turn: three counts side by
// side take hardly longer than one.
constexpr int kReach(int k) { return k + k / 4; }

template <int kPer, typename X>
__device__ inline X near_kth_of(const X (&x)[kPer], int k, X low) {
    auto reach = [&](X y) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < kPer; ++w) n += __popcll(__ballot(x[w] >= y));
        return n;
    };
    if (reach(low) <= kReach(k)) return low;
    X above = ~(X)0;  // the k-th largest lies in low .. above
    while (low < above) {
        const X step = (above - low) / 4 + 1;
        const X y1 = low + step, y2 = above - y1 >= step ? y1 + step : above, y3 = above - y2 >= step ? y2 + step : above;
        const int n1 = reach(y1), n2 = reach(y2), n3 = reach(y3);
        int n = INT_MAX;
        if (n3 >= k) low = y3, n = n3;
        else if (n2 >= k) low = y2, above = y3 - 1, n = n2;
        else if (n1 >= k) low = y1, above = y2 - 1, n = n1;
        else above = y1 - 1;
        if (n <= kReach(k)) break;
    }
    return low;
}

// A value that at least k of all threads' reach, and few more: of 64 groups' maxima for a small k, or 256 (of logits in
// any order, k of 4 k groups leave 1.15 k candidates).  The first wave finds it, since the others' instructions would only take
// turns with its own, and those of the blocks beside.
template <int kThreads, typename X>
__device__ inline X near_kth(X mine, int k, X low) {
    __shared__ X all[256], found;
    const bool few = k <= 16;
    const int lane = threadIdx.x, group = kThreads / (few ? 64 : 256);  // threads of a group
#pragma unroll
    for (int d = 1; d < kThreads / 64; d <<= 1)
        if (d < group) mine = max(mine, __shfl_xor(mine, d));
    if (threadIdx.x % group == 0) all[threadIdx.x / group] = mine;
    __syncthreads();
    if (threadIdx.x < kWave) {
        if (few) {
            const X x[1] = {all[lane]};
            low = near_kth_of<1, X>(x, k, low);
        } else {
            const X x[4] = {all[lane], all[lane + 64], all[lane + 128], all[lane + 192]};
            low = near_kth_of<4, X>(x, k, low);
        }
        if (lane == 0) found = low;
    }
    __syncthreads();
    return found;
}

struct Top {
    int64_t V, row_stride;
    int32_t k, parts;
    uint64_t *keys;  // [B][parts][k]
    Sum *sums;       // [B][parts]
    int32_t *tokens;
    float *logprobs, *lse;
};

__device__ inline void write(const Top &a, int64_t b, int i, uint64_t key, float lse) {
    a.tokens[b * a.k + i] = key ? (int32_t)(0xFFFFFFFFu - (uint32_t)key) : -1;
    a.logprobs[b * a.k + i] = key ? logit_of((uint32_t)(key >> 32)) - lse : -INFINITY;
}

// The candidates' ranks, by counting those before each, `group` threads to a candidate; the first k of them go to their places.
template <int kThreads, typename F>
__device__ inline void rank(const uint64_t *found, int n, int k, F put) {
    int group = 1;
    while (group < kWave && 2 * group * n <= kThreads) group *= 2;
    const int sub = threadIdx.x & (group - 1);
    for (int i = threadIdx.x / group; i < n; i += kThreads / group) {
        const uint64_t mine = found[i];
        int before = 0;
#pragma unroll 4
        for (int j = sub; j < n; j += group) before += found[j] > mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1)
            if (d < group) before += __shfl_xor(before, d);
        if (sub == 0 && before < k) put(before, mine);
    }
    for (int i = n + threadIdx.x; i < k; i += kThreads) put(i, 0);
}

// The candidates where there are too many and k or more of them above the bound: the order of the k-th key by halving, then how far in the tokens the keys of that order go.  The logits are read again in each turn, so that nothing of this
// takes registers from the usual way.
template <int kThreads, typename T>
__device__ __attribute__((noinline)) int collect_exactly(const T *row, int64_t from, int64_t to, int k, uint64_t *found, int32_t *count) {
    auto counted = [&](auto is) {
        int mine = 0;
        for (int64_t v = from + threadIdx.x; v < to; v += kThreads) mine += is(order_of(In<T>::load(row + v)), v);
        return count_block<kThreads>(mine);
    };
    uint32_t low = kNone + 1, above = ~0u;
    int n = counted([&](uint32_t o, int64_t) { return o >= low; });
    if (n < k) above = low;  // all of them
    while (low < above) {
        const uint32_t mid = low + (above - low) / 2 + 1;
        n = counted([&](uint32_t o, int64_t) { return o >= mid; });
        if (n >= k) low = mid;
        else above = mid - 1;
        if (n == k) break;
    }
    n = counted([&](uint32_t o, int64_t) { return o > low; });
    int64_t first = from, last = to;  // of the order `low` the tokens before `last`: k - n of them, or all
    while (first < last) {
        const int64_t mid = first + (last - first) / 2;
        if (n + counted([&](uint32_t o, int64_t v) { return o == low && v < mid; }) >= k) last = mid;
        else first = mid + 1;
    }
    last = min(last, to);
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    for (int64_t v = from + threadIdx.x; v < to; v += kThreads) {
        const float x = In<T>::load(row + v);
        const uint32_t o = order_of(x);
        if (o > low || (o == low && v < last)) found[atomicAdd(count, 1)] = key_of(x, (uint32_t)v);
    }
    __syncthreads();
    return *count;
}

template <typename T, int kVecs, int kThreads>
__global__ void __launch_bounds__(kThreads) k_top(const T *__restrict__ logits, Top a) {
    using I = In<T>;
    constexpr int N = I::n, kCandidates = 1024;
    __shared__ __align__(16) uint64_t found[kCandidates];
    __shared__ int32_t count;
    const int64_t b = blockIdx.x / (uint32_t)a.parts;
    const int part = (int)(blockIdx.x - b * a.parts);
    const T *row = logits + b * a.row_stride;
    // vector j of the row is its elements j N - skip on, `skip` being the row's place in its first 16 bytes
    const int skip = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const u32x4 *const from = reinterpret_cast<const u32x4 *>(row - skip);
    const int64_t j0 = (int64_t)part * kThreads * kVecs + threadIdx.x;
    const int64_t vectors = (a.V + skip + N - 1) / N;
    u32x4 x[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t j = j0 + i * kThreads;
        x[i] = j < vectors ? from[j] : u32x4{I::kMinusInf, I::kMinusInf, I::kMinusInf, I::kMinusInf};
    }
    if (threadIdx.x == 0) count = 0;
    // (no converted logits are kept from one pass over the registers to the next: they would take twice the room)
    auto fresh = [&]() {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) asm volatile("" : "+v"(x[i]));
    };
    float high[kVecs], most = -INFINITY;  // (a NaN stays one)
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t e = (j0 + i * kThreads) * N - skip;
        if (e < 0 || e + N > a.V) {  // elements of no token
#pragma unroll
            for (int c = 0; c < N; ++c)
                if (e + c < 0 || e + c >= a.V) I::drop(x[i], c);
        }
        high[i] = I::get(x[i], 0);
#pragma unroll
        for (int c = 1; c < N; ++c) high[i] = __builtin_elementwise_maximum(high[i], I::get(x[i], c));
        most = __builtin_elementwise_maximum(most, high[i]);
    }
    // (x - m is exact where it counts, however large both are.  -inf: 0, so that nothing is taken from it; infinity: the
    // largest number, and the sum is infinite.)
    Sum sum{most, 0.f};
    const float m = most == -INFINITY ? 0.f : fminf(most, 3.4028234663852886e38f);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        if (!__any(!(high[i] == -INFINITY))) continue;  // nothing in the wave's vectors
        asm volatile("" : "+v"(x[i]));
#pragma unroll
        for (int c = 0; c < N; ++c) sum.s += __builtin_amdgcn_exp2f((I::get(x[i], c) - m) * kLog2e);
    }
    if (sum.s != sum.s) sum.m = -INFINITY;
    sum = join_block<kThreads>(sum);
    fresh();
    // (comparisons that a NaN passes, as it is above all)
    const float low = logit_of(near_kth<kThreads, uint32_t>(order_of(most), a.k, kNone + 1));
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        if (!(high[i] < low)) {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const float y = I::get(x[i], c);
                if (!(y < low)) {
                    const int at = atomicAdd(&count, 1);
                    if (at < kCandidates) found[at] = key_of(y, (uint32_t)((j0 + i * kThreads) * N - skip + c));
                }
            }
        }
    }
    __syncthreads();
    int n = count;
    __syncthreads();
    if (n > kCandidates) {
        // equal logits: with fewer than k above `low` that is the k-th, and of those that equal it the first tokens are taken, a
        // vector of each thread after the other
        fresh();
        int above = 0;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (!(high[i] <= low)) {
#pragma unroll
                for (int c = 0; c < N; ++c) above += !(I::get(x[i], c) <= low);
            }
        above = count_block<kThreads>(above);
        if (above < a.k) {
            if (threadIdx.x == 0) count = 0;
            __syncthreads();
            auto take = [&](int i, int c) { found[atomicAdd(&count, 1)] = key_of(I::get(x[i], c), (uint32_t)((j0 + i * kThreads) * N - skip + c)); };
            int need = a.k - above;
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                asm volatile("" : "+v"(x[i]));
                if (!(high[i] <= low)) {
#pragma unroll
                    for (int c = 0; c < N; ++c)
                        if (!(I::get(x[i], c) <= low)) take(i, c);
                }
                if (need > 0) {
                    int equal = 0, all;
#pragma unroll
                    for (int c = 0; c < N; ++c) equal += I::get(x[i], c) == low;
                    int before = before_block<kThreads>(equal, &all);
                    if (equal && before < need) {
#pragma unroll
                        for (int c = 0; c < N; ++c)
                            if (I::get(x[i], c) == low && before++ < need) take(i, c);
                    }
                    need -= all;
                }
            }
            __syncthreads();
            n = count;
        }
    }
    if (n > kCandidates) {
        const int64_t begin = (int64_t)part * kThreads * kVecs * N - skip, end = begin + kThreads * kVecs * N;
        n = collect_exactly<kThreads, T>(row, max(begin, (int64_t)0), min(end, a.V), a.k, found, &count);
    }
    if (a.parts == 1) {
        const float lse = log_of(sum);
        rank<kThreads>(found, n, a.k, [&](int i, uint64_t y) { write(a, b, i, y, lse); });
        if (a.lse && threadIdx.x == 0) a.lse[b] = lse;
    } else {
        const int64_t at = b * a.parts + part;
        rank<kThreads>(found, n, a.k, [&](int i, uint64_t y) { a.keys[at * a.k + i] = y; });
        if (threadIdx.x == 0) a.sums[at] = sum;
    }
}

// A thread's keys: of up to 8,192, which the entry point's limits on V and k and split_of keep to.  The keys are all different, so
// that no more than kReach(k) groups' of near_kth are candidates.
constexpr int kJoin = 512, kJoinKeys = 16, kFewKeys = 128, kJoinCandidates = kReach(TAM_MAX_TOP) * kJoinKeys * (kJoin / 256);
static_assert(kJoinCandidates >= kReach(16) * kJoinKeys * (kJoin / 64) && kJoinCandidates >= kFewKeys, "room for the candidates");

__global__ void __launch_bounds__(kJoin) k_top_join(Top a) {
    __shared__ __align__(16) uint64_t found[kJoinCandidates];
    __shared__ int32_t count;
    const int64_t b = blockIdx.x;
    int n = a.parts * a.k;
    const uint64_t *const keys = a.keys + b * n;
    if (threadIdx.x == 0) count = 0;
    Sum sum{-INFINITY, 0.f};
    if ((int)threadIdx.x < a.parts) sum = a.sums[b * a.parts + threadIdx.x];
    if (n <= kFewKeys) {  // few enough to rank them all
        const uint64_t x = (int)threadIdx.x < n ? keys[threadIdx.x] : 0;
        sum = join_block<kJoin>(sum);
        if (x) found[atomicAdd(&count, 1)] = x;
        __syncthreads();
        n = count;
    } else {
        uint64_t x[kJoinKeys], most = 0;
#pragma unroll
        for (int i = 0; i < kJoinKeys; ++i) {
            // the parts' best ones first, so that they lie in groups of their own
            const int j = threadIdx.x + i * kJoin, place = j / a.parts;
            x[i] = j < n ? keys[(j - place * a.parts) * a.k + place] : 0;
            most = max(most, x[i]);
        }
        sum = join_block<kJoin>(sum);
        const uint64_t low = near_kth<kJoin, uint64_t>(most, a.k, 1);
#pragma unroll
        for (int i = 0; i < kJoinKeys; ++i)
            if (x[i] >= low) found[atomicAdd(&count, 1)] = x[i];
        __syncthreads();
        n = count;
    }
    const float lse = log_of(sum);
    rank<kJoin>(found, n, a.k, [&](int i, uint64_t y) { write(a, b, i, y, lse); });
    if (a.lse && threadIdx.x == 0) a.lse[b] = lse;
}

struct Split {
    int vecs, threads, parts;
};

constexpr int kParts = kJoin * kJoinKeys / TAM_MAX_TOP;  // of a row, whose best k_top_join holds

// Blocks of 256 threads, since smaller ones leave k_top_join more and larger ones wait for one another (us per call of 256 bf16
// rows over V = 262,144, k_top and k_top_join, 64 threads: 32.3 and 7.4, 128: 30.1 and 4.7, 256: 29.6 and 4.1, 512: 35.7 and
// 4.8, 1,024: 66 and 5), with as many vectors each as leave the chip 2,048 blocks; more threads only where a row would have more
// parts than k_top_join holds.  Short rows, no more than there are CUs, take a block each, which leaves the second launch out (us
// per call of 1, 64, 256 and 512 fp32 rows over V = 32,000, 4 of each: 8.1, 9.1, 11.9 and 22.9, in parts 8.1, 10.2, 15.2 and 21.5, and
// 3 less on the host; 64 of each: 10.2, 11.5, 13.9 and 26.7, in parts 14.9, 17.3, 24.1 and 31.9).  More short rows than CUs go in parts:
// of the 512's 21.5 k_top takes 16.4, k_top_join 4.0 (64 of each: 23.2 and 9.1); k_top's waves wait in 46 cycles of 100, at the barriers and
// for the loads, and for their turn to issue in 35.  Twice as long ones do not
// fit a block's registers: 256 bf16 rows over V = 128,256 27, in parts 22.
template <typename T>
Split split_of(int64_t B, int64_t V) {
    const int64_t vectors = (V + 2 * In<T>::n - 2) / In<T>::n;
    Split s{4, 256, 1};
    auto parts = [&] { return (int)((vectors + s.threads * s.vecs - 1) / (s.threads * s.vecs)); };
    while (s.vecs < 16 && (B * parts() > 2048 || parts() > kParts)) s.vecs *= 2;
    if (parts() > kParts) s.threads = 512;
    if (B <= 256 && vectors <= 8192) s.vecs = vectors <= 4096 ? 4 : 8, s.threads = 1024;
    s.parts = parts();
    return s;
}

// Whether some row has too many vectors for kParts parts of 256 threads: of fp32, whose widest rows (from TAM_MAX_TOP_COLUMNS - 2 on)
// may lie over one vector more.  These take blocks of 512 threads (256 rows, 8 of each: 343 us, in the short rows' blocks of 1,024 568).
template <typename T>
constexpr bool kWide = (TAM_MAX_TOP_COLUMNS + 2 * In<T>::n - 2) / In<T>::n > kParts * 256 * 16;

template <typename T>
hipError_t launch(const void *logits, int64_t B, Top a, const Split &sp, hipStream_t s) {
    void (*kernel)(const T *, Top) = sp.threads == 1024 ? (sp.vecs == 4 ? k_top<T, 4, 1024> : k_top<T, 8, 1024>)
                                     : sp.vecs == 4     ? k_top<T, 4, 256>
                                     : sp.vecs == 8     ? k_top<T, 8, 256>
                                                        : k_top<T, 16, 256>;
    if constexpr (kWide<T>) {
        if (sp.threads == 512) kernel = k_top<T, 16, 512>;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)(B * sp.parts)), dim3((unsigned)sp.threads), 0, s, static_cast<const T *>(logits), a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || sp.parts == 1) return e;
    hipLaunchKernelGGL(k_top_join, dim3((unsigned)B), dim3(kJoin), 0, s, a);
    return hipGetLastError();
}

Split split_of(int64_t B, int64_t V, int dtype) { return dtype == TAM_DTYPE_FP32 ? split_of<float>(B, V) : split_of<uint16_t>(B, V); }

}  // namespace

int64_t top_work_bytes(int64_t B, int64_t V, int k, int dtype) {
    const Split s = split_of(B, V, dtype);
    return s.parts == 1 ? 0 : B * s.parts * (8 * (int64_t)k + (int64_t)sizeof(Sum));
}

hipError_t launch_top_tokens(const void *logits, int dtype, int64_t B, int64_t V, int64_t row_stride, int k, int32_t *tokens,
                             float *logprobs, float *lse, void *work, hipStream_t s) {
    const Split sp = split_of(B, V, dtype);
    uint64_t *const keys = static_cast<uint64_t *>(work);
    const Top a{V, row_stride, k, sp.parts, keys, reinterpret_cast<Sum *>(keys + B * sp.parts * k), tokens, logprobs, lse};
    return dtype == TAM_DTYPE_FP32 ? launch<float>(logits, B, a, sp, s) : launch<uint16_t>(logits, B, a, sp, s);
}

}  // namespace tam
