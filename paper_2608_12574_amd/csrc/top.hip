// The k best tokens of each row of logits, with their log probabilities.
//
// Mathematics.  lse = m + log sum_v exp(x_v - m) for any m; parts summed under their own maxima join the same way.  The best
// tokens are the largest of the keys (logit, lowest token first), which are all different.  For any partition of the logits the
// k-th largest of the parts' maxima is no larger than the k-th largest logit, so only logits from there on can be among the best.
//
// k_top: a block holds a span of a row in registers, read once.  Each thread finds its maximum and its sum; the k-th largest of
// the threads' maxima (found by halving, in each wave by itself) leaves a few more than k candidates, which go to LDS and
// are ranked by counting.  Where equal logits leave too many, the k-th key itself is found by halving.
// k_top_join: the spans' best, in the same way, and the sum of the sums.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <type_traits>

#include "step.hpp"

namespace tam {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

constexpr int kWave = 64, kThreads = 512, kWaves = kThreads / kWave;
constexpr int kCandidates = 1280;
constexpr float kLog2e = 1.4426950408889634f;

// Keys: the logit's order in the upper half (-0 and 0 alike, NaN above all), then the lowest token first.  0: no token.
__device__ inline uint64_t key_of(uint32_t bits, uint32_t token) {
    if (bits == 0x80000000u) bits = 0;
    if ((bits & 0x7FFFFFFFu) > 0x7F800000u) bits = 0x7FFFFFFFu;
    const uint32_t order = bits ^ ((bits & 0x80000000u) ? 0xFFFFFFFFu : 0x80000000u);
    return (uint64_t)order << 32 | (0xFFFFFFFFu - token);
}

__device__ inline float logit_of(uint64_t key) {
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float(order ^ ((order & 0x80000000u) ? 0x80000000u : 0xFFFFFFFFu));
}

// How a type's logits lie in a 16-byte vector, and their order as signed integers (-0 under 0; a NaN with a sign under -inf).
template <typename T>
struct In;

template <>
struct In<float> {
    static constexpr int n = 4;
    static constexpr uint32_t kMinusInf = 0xFF800000u;  // a word of it
    static constexpr int32_t kLowest = (int32_t)0x80800000u, kAbove = INT_MAX;  // orders of what lies just above -inf; of all
    static __device__ uint32_t bits(u32x4 x, int i) { return x[i]; }
    static __device__ void drop(u32x4 &x, int i) { x[i] = kMinusInf; }
    static __device__ int32_t order(u32x4 x, int i) { return (int32_t)(x[i] ^ ((uint32_t)((int32_t)x[i] >> 31) & 0x7FFFFFFFu)); }
    static __device__ int32_t highest(u32x4 x) { return max(max(order(x, 0), order(x, 1)), max(order(x, 2), order(x, 3))); }
    static __device__ float value(int32_t order) { return __int_as_float(order ^ (int32_t)((uint32_t)(order >> 31) & 0x7FFFFFFFu)); }
};

template <>
struct In<uint16_t> {  // bf16
    static constexpr int n = 8;
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
    static constexpr int32_t kLowest = -32640, kAbove = 32767;
    static __device__ uint32_t bits(u32x4 x, int i) { return i & 1 ? x[i >> 1] & 0xFFFF0000u : x[i >> 1] << 16; }
    static __device__ void drop(u32x4 &x, int i) { x[i >> 1] = i & 1 ? (x[i >> 1] & 0xFFFFu) | 0xFF800000u : (x[i >> 1] & 0xFFFF0000u) | 0xFF80u; }
    static __device__ i16x2 orders(uint32_t w) {
        const i16x2 x = __builtin_bit_cast(i16x2, w);
        return x ^ ((x >> (int16_t)15) & (int16_t)0x7FFF);
    }
    static __device__ int32_t order(u32x4 x, int i) {
        const int16_t y = (int16_t)(x[i >> 1] >> 16 * (i & 1));
        return (int16_t)(y ^ ((y >> 15) & 0x7FFF));
    }
    static __device__ int32_t highest(u32x4 x) {
        const i16x2 y = __builtin_elementwise_max(__builtin_elementwise_max(orders(x[0]), orders(x[1])),
                                                  __builtin_elementwise_max(orders(x[2]), orders(x[3])));
        return max((int32_t)y[0], (int32_t)y[1]);
    }
    static __device__ float value(int32_t order) {
        return __uint_as_float((uint32_t)(order ^ ((order >> 31) & 0x7FFF)) << 16);
    }
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
__device__ inline Sum join_block(Sum x) {
    __shared__ Sum waves[kWaves];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x = join(x, Sum{__shfl_xor(x.m, d), __shfl_xor(x.s, d)});
    __syncthreads();
    if (threadIdx.x % kWave == 0) waves[threadIdx.x / kWave] = x;
    __syncthreads();
    x = waves[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) x = join(x, waves[w]);
    return x;
}

__device__ inline float log_of(Sum x) { return x.s == 0.f ? -INFINITY : x.m + logf(x.s); }

__device__ inline int count_block(int mine) {
    __shared__ int waves[kWaves];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) mine += __shfl_xor(mine, d);
    __syncthreads();
    if (threadIdx.x % kWave == 0) waves[threadIdx.x / kWave] = mine;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += waves[w];
    return all;
}

// A value that at least k of the threads' maxima reach and not many more do (where they are all different: k + k / 4 at
// most), or `low` if no more than k reach that.  X: a signed integer, at most `high`; each wave looks at all of them.
template <typename X>
__device__ inline X near_kth(X mine, int k, X low, X high) {
    using U = std::make_unsigned_t<X>;
    __shared__ X all[kThreads];
    all[threadIdx.x] = mine;
    __syncthreads();
    X x[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x[w] = all[w * kWave + threadIdx.x % kWave];
    auto reach = [&](X y) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) n += __popcll(__ballot(x[w] >= y));
        return n;
    };
    if (reach(low) <= k) return low;
    // reach(low) > k; what lies above `high` is reached by none
    X above = high;
    while (low < above) {
        const X mid = (X)((U)low + ((U)above - (U)low) / 2 + 1);  // (low < mid <= above but for above = low + 1: mid = above)
        const int n = reach(mid);
        if (n >= k) low = mid;
        else above = mid - 1;
        if (n >= k && n <= k + k / 4) break;
    }
    return low;
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
    a.logprobs[b * a.k + i] = key ? logit_of(key) - lse : -INFINITY;
}

// The candidates' ranks; the first k of them go to their places.
template <typename F>
__device__ inline void rank(const uint64_t *found, int n, int k, F put) {
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t mine = found[i];
        int before = 0;
        for (int j = 0; j < n; ++j) before += found[j] > mine;
        if (before < k) put(before, mine);
    }
    for (int i = n + threadIdx.x; i < k; i += kThreads) put(i, 0);
}

template <typename T, int kVecs>
__global__ void __launch_bounds__(kThreads) k_top(const T *__restrict__ logits, Top a) {
    using I = In<T>;
    constexpr int N = I::n;
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
    int32_t high[kVecs], most = INT_MIN;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t e = (j0 + i * kThreads) * N - skip;
        if (e < 0 || e + N > a.V) {  // elements of no token
#pragma unroll
            for (int c = 0; c < N; ++c)
                if (e + c < 0 || e + c >= a.V) I::drop(x[i], c);
        }
        high[i] = I::highest(x[i]);
        most = max(most, high[i]);
    }
    // (-inf: 0, so that nothing is taken from it; infinity: the largest number, and the sum is infinite)
    const float m = I::value(most), under = m == -INFINITY ? 0.f : fminf(m, 3.4028234663852886e38f);
    Sum sum{m, 0.f};
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int c = 0; c < N; ++c) sum.s += __builtin_amdgcn_exp2f((__uint_as_float(I::bits(x[i], c)) - under) * kLog2e);
    const bool odd = sum.s != sum.s;
    if (odd) sum.m = -INFINITY;
    sum = join_block(sum);
    if (sum.s != sum.s) {  // a NaN, which may have a sign: above all
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const uint32_t y = I::bits(x[i], c);
                if ((y & 0x7FFFFFFFu) > 0x7F800000u) {
                    if constexpr (N == 4) x[i][c] = 0x7FFFFFFFu;
                    else x[i][c >> 1] |= 0x7FFFu << 16 * (c & 1), x[i][c >> 1] &= ~(0x8000u << 16 * (c & 1));
                }
            }
            high[i] = I::highest(x[i]);
            most = max(most, high[i]);
        }
    }
    int32_t low = near_kth<int32_t>(most, a.k, I::kLowest, I::kAbove);
    if (low == 0) low = -1;  // -0 is as high as 0
    auto key = [&](int i, int c) { return key_of(I::bits(x[i], c), (uint32_t)((j0 + i * kThreads) * N - skip + c)); };
    auto collect = [&](auto is) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (high[i] < low) continue;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                if (!is(i, c)) continue;
                const int at = atomicAdd(&count, 1);
                if (at < kCandidates) found[at] = key(i, c);
            }
        }
    };
    collect([&](int i, int c) { return I::order(x[i], c) >= low; });
    __syncthreads();
    int n = count;
    if (n > kCandidates) {  // the k-th key itself
        uint64_t floor = 1, above = ~0ull;
        while (floor < above) {
            const uint64_t mid = floor + (above - floor) / 2 + 1;
            int mine = 0;
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
                for (int c = 0; c < N; ++c) mine += I::order(x[i], c) >= low && key(i, c) >= mid;
            const int all = count_block(mine);
            if (all >= a.k) floor = mid;
            else above = mid - 1;
            if (all == a.k) break;
        }
        __syncthreads();
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        collect([&](int i, int c) { return I::order(x[i], c) >= low && key(i, c) >= floor; });
        __syncthreads();
        n = count;
    }
    if (a.parts == 1) {
        const float lse = log_of(sum);
        rank(found, n, a.k, [&](int i, uint64_t y) { write(a, b, i, y, lse); });
        if (a.lse && threadIdx.x == 0) a.lse[b] = lse;
    } else {
        const int64_t at = b * a.parts + part;
        rank(found, n, a.k, [&](int i, uint64_t y) { a.keys[at * a.k + i] = y; });
        if (threadIdx.x == 0) a.sums[at] = sum;
    }
}

// A thread's keys: of up to 8,192, which the entry point's limits on V and k and split_of keep to.  The keys are all different, so
// that no more than 80 threads' are candidates.
constexpr int kJoinKeys = 16;
static_assert(kCandidates >= (TAM_MAX_TOP + TAM_MAX_TOP / 4) * kJoinKeys, "room for the join's candidates");

__global__ void __launch_bounds__(kThreads) k_top_join(Top a) {
    __shared__ __align__(16) uint64_t found[kCandidates];
    __shared__ int32_t count;
    const int64_t b = blockIdx.x;
    const int n = a.parts * a.k;
    const uint64_t *const keys = a.keys + b * n;
    uint64_t x[kJoinKeys], most = 0;
#pragma unroll
    for (int i = 0; i < kJoinKeys; ++i) {
        const int j = threadIdx.x + i * kThreads;
        x[i] = j < n ? keys[j] : 0;
        most = max(most, x[i]);
    }
    if (threadIdx.x == 0) count = 0;
    Sum sum{-INFINITY, 0.f};
    if ((int)threadIdx.x < a.parts) sum = a.sums[b * a.parts + threadIdx.x];
    sum = join_block(sum);
    // (keys with their upper bit turned are signed integers in the same order)
    constexpr uint64_t kTop = 1ull << 63;
    const uint64_t low = (uint64_t)near_kth<int64_t>((int64_t)(most ^ kTop), a.k, (int64_t)(1 ^ kTop), INT64_MAX) ^ kTop;
#pragma unroll
    for (int i = 0; i < kJoinKeys; ++i) {
        if (x[i] < low) continue;
        found[atomicAdd(&count, 1)] = x[i];
    }
    __syncthreads();
    const float lse = log_of(sum);
    rank(found, count, a.k, [&](int i, uint64_t y) { write(a, b, i, y, lse); });
    if (a.lse && threadIdx.x == 0) a.lse[b] = lse;
}

struct Split {
    int vecs, parts;
};

template <typename T>
Split split_of(int64_t B, int64_t V) {
    const int64_t vectors = (V + 2 * In<T>::n - 2) / In<T>::n;
    Split s{1, 1};
    for (;; s.vecs *= 2) {
        s.parts = (int)((vectors + kThreads * s.vecs - 1) / (kThreads * s.vecs));
        if (s.vecs == 16 || (B * s.parts <= 1024 && s.parts <= 128)) return s;
    }
}

template <typename T>
hipError_t launch(const void *logits, int64_t B, Top a, const Split &sp, hipStream_t s) {
    void (*kernel)(const T *, Top) = sp.vecs == 1   ? k_top<T, 1>
                                     : sp.vecs == 2 ? k_top<T, 2>
                                     : sp.vecs == 4 ? k_top<T, 4>
                                     : sp.vecs == 8 ? k_top<T, 8>
                                                    : k_top<T, 16>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(B * sp.parts)), dim3(kThreads), 0, s, static_cast<const T *>(logits), a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || sp.parts == 1) return e;
    hipLaunchKernelGGL(k_top_join, dim3((unsigned)B), dim3(kThreads), 0, s, a);
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
