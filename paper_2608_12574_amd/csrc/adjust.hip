// Penalties, biases and the grammar's mask on [B, V] logits, in place.
//
// A block takes one span of one row's vocabulary.  It counts the row's text in a
// table in LDS with one word per token of the span (an integer sum, so the order of
// the atomics does not matter), and then goes through the span's logits in 16-byte
// chunks: a chunk without a valid token is stored as -inf and not read, one
// whose valid tokens are not named is left alone or merged, and only the named
// tokens are computed.  So a logit is read and written at most once, and the text
// is all that is read beside the mask; each block of a row reads that again, from L2.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"

namespace tam {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A table word: occurrences after the prompt (bits 0-18), seen in the prompt (bit
// 19), the last entry of the bias list that names the token, plus one (bits 20-31).
constexpr uint32_t kSeen = 1u << 19, kCount = kSeen - 1;
constexpr int kEntry = 20;
static_assert(TAM_MAX_HISTORY == kCount && TAM_MAX_BIASES == (1 << (32 - kEntry)) - 1, "fields of a table word");

constexpr int kThreads = 256;
constexpr int kSpan = 4096;  // tokens of a block

template <typename T>
struct Lane;
template <>
struct Lane<float> {
    static constexpr int n = 4;
    static __device__ float get(u32x4 x, int i) { return __uint_as_float(x[i]); }
    static __device__ void put(u32x4 &x, int i, float v) { x[i] = __float_as_uint(v); }
    static __device__ void minus_inf(u32x4 &x, int i) { x[i] = 0xFF800000u; }
    static constexpr uint32_t kMinusInf = 0xFF800000u;  // a word of -inf
};
template <>
struct Lane<uint16_t> {  // bf16
    static constexpr int n = 8;
    static __device__ float get(u32x4 x, int i) { return __uint_as_float((x[i >> 1] >> (16 * (i & 1))) << 16); }
    static __device__ void set(u32x4 &x, int i, uint32_t h) {
        const int sh = 16 * (i & 1);
        x[i >> 1] = (x[i >> 1] & ~(0xFFFFu << sh)) | (h << sh);
    }
    static __device__ void put(u32x4 &x, int i, float v) {  // to nearest, ties to even; a NaN stays one
        const uint32_t u = __float_as_uint(v);
        set(x, i, v != v ? (u >> 16) | 0x40u : (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
    }
    static __device__ void minus_inf(u32x4 &x, int i) { set(x, i, 0xFF80u); }
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
};

struct Edits {
    float repetition, frequency, presence;
    const float *bias;
};

__device__ float edited(float x, uint32_t w, const Edits &e) {
#pragma clang fp contract(off)
    const uint32_t n = w & kCount;
    if (w & (kSeen | kCount)) x = x > 0.f ? x / e.repetition : x * e.repetition;
    if (n) {
        x = x - e.frequency * (float)n;
        x = x - e.presence;
    }
    if (w >> kEntry) x = x + e.bias[(w >> kEntry) - 1];
    return x;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_adjust(const uint64_t *__restrict__ rows, int64_t num_rows,
                                                     int64_t rows_stride, const int32_t *__restrict__ ids, tam_edits e,
                                                     int64_t V, T *__restrict__ logits, int64_t row_stride) {
    constexpr int N = Lane<T>::n;
    __shared__ __align__(16) uint32_t tab[kSpan];
    __shared__ uint32_t bits[kSpan / 32 + 2];
    const int64_t b = blockIdx.y;
    T *row = logits + b * row_stride;
    // chunk k of the row covers elements [k N - a, (k + 1) N - a), a being the row's
    // place in its first 16 bytes; v0 is the span's first element (-a in the first block)
    const int a = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const int64_t v0 = (int64_t)blockIdx.x * kSpan - a;
    if (v0 >= V) return;
    const int span = (int)min((int64_t)kSpan, V - v0);  // elements of the span, those before 0 among them

    for (int i = threadIdx.x * 4; i < kSpan; i += kThreads * 4) *reinterpret_cast<u32x4 *>(&tab[i]) = u32x4{0, 0, 0, 0};
    bool dead = false;
    if (rows) {
        const int64_t r = ids[b];
        dead = r < 0 || r >= num_rows;
        if (!dead) {  // the span's bits, shifted so that bit 0 is element v0
            const uint32_t *src = reinterpret_cast<const uint32_t *>(rows + r * rows_stride);
            const int64_t words = (V + 31) / 32;
            const int sh = (int)(v0 & 31);
            const int64_t w0 = (v0 - sh) / 32;
            for (int i = threadIdx.x; i < kSpan / 32 + 1; i += kThreads) {
                const int64_t w = w0 + i;
                const uint32_t lo = w >= 0 && w < words ? src[w] : 0u, hi = w + 1 < words ? src[w + 1] : 0u;
                bits[i] = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
            }
        }
    }
    __syncthreads();
    if (!dead) {
        if (e.bias_ids) {
            const int32_t *named = e.bias_ids + b * e.bias_stride;
            for (int i = threadIdx.x; i < (int)e.biases; i += kThreads) {
                const int64_t v = named[i], o = v - v0;
                if (v >= 0 && o >= 0 && o < span) atomicMax(&tab[o], (uint32_t)(i + 1) << kEntry);
            }
            __syncthreads();  // the entry's field is final before the counts are added below it
        }
        if (e.tokens) {
            const int32_t *text = e.tokens + b * e.tokens_stride;
            const int len = e.length ? min(max(e.length[b], 0), (int)e.history) : (int)e.history;
            const int prompt = e.prompt ? e.prompt[b] : 0;
            for (int i = threadIdx.x; i < len; i += kThreads) {
                const int64_t v = text[i], o = v - v0;
                if (v >= 0 && o >= 0 && o < span) {
                    if (i < prompt)
                        atomicOr(&tab[o], kSeen);
                    else
                        atomicAdd(&tab[o], 1u);
                }
            }
            __syncthreads();
        }
    }
    const Edits ed{e.repetition ? e.repetition[b] : 1.f, e.frequency ? e.frequency[b] : 0.f,
                   e.presence ? e.presence[b] : 0.f, e.bias ? e.bias + b * e.bias_stride : nullptr};
    constexpr uint32_t kAll = (1u << N) - 1;
    for (int o = threadIdx.x * N; o < span; o += kThreads * N) {
        uint32_t inside = kAll;  // elements of the chunk that the row has
        if (v0 + o < 0) inside &= kAll << (int)-(v0 + o);
        if (o + N > span) inside &= kAll >> (o + N - span);
        uint32_t valid = kAll;
        if (rows) valid = dead ? 0u : (bits[o >> 5] >> (o & 31)) & kAll;
        u32x4 *at = reinterpret_cast<u32x4 *>(row + (v0 + o));
        if (!(valid & inside)) {
            if (inside == kAll) {
                constexpr uint32_t m = Lane<T>::kMinusInf;
                __builtin_nontemporal_store(u32x4{m, m, m, m}, at);
                continue;
            }
        }
        uint32_t named = 0;
        if (valid) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(&tab[o + i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) named |= (w[j] != 0u) << (i + j);
            }
            named &= valid;
        }
        const uint32_t edit = (named | ~valid) & inside;
        if (!edit) continue;
        if (inside == kAll) {
            u32x4 x = *at;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!(valid >> i & 1)) Lane<T>::minus_inf(x, i);
                else if (named >> i & 1) Lane<T>::put(x, i, edited(Lane<T>::get(x, i), tab[o + i], ed));
            }
            __builtin_nontemporal_store(x, at);
        } else {  // the row's ends: element by element
            for (int i = 0; i < N; ++i) {
                if (!(edit >> i & 1)) continue;
                u32x4 x{0, 0, 0, 0};
                T *p = row + (v0 + o + i);
                if (!(valid >> i & 1)) {
                    Lane<T>::minus_inf(x, 0);
                } else {
                    uint32_t raw = 0;
                    __builtin_memcpy(&raw, p, sizeof(T));
                    x[0] = raw;
                    Lane<T>::put(x, 0, edited(Lane<T>::get(x, 0), tab[o + i], ed));
                }
                const uint32_t raw = x[0];
                __builtin_memcpy(p, &raw, sizeof(T));
            }
        }
    }
}

template <typename T>
hipError_t launch(const uint64_t *rows, int64_t num_rows, int64_t rows_stride, const int32_t *ids, tam_edits e,
                  int64_t B, int64_t V, T *logits, int64_t row_stride, hipStream_t s) {
    // a row may start up to 15 bytes into a chunk, which moves its end as far
    const unsigned gx = (unsigned)((V + Lane<T>::n - 1 + kSpan - 1) / kSpan);
    for (int64_t r0 = 0; r0 < B; r0 += 65535) {
        const int64_t n = std::min<int64_t>(B - r0, 65535);
        hipLaunchKernelGGL((k_adjust<T>), dim3(gx, (unsigned)n), dim3(kThreads), 0, s, rows, num_rows, rows_stride,
                           ids ? ids + r0 : nullptr, e, V, logits + r0 * row_stride, row_stride);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        if (e.tokens) e.tokens += n * e.tokens_stride;
        if (e.bias_ids) e.bias_ids += n * e.bias_stride, e.bias += n * e.bias_stride;
        for (const int32_t **p : {&e.length, &e.prompt})
            if (*p) *p += n;
        for (const float **p : {&e.repetition, &e.frequency, &e.presence})
            if (*p) *p += n;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_adjust(const uint64_t *rows, int64_t num_rows, int64_t rows_stride, const int32_t *ids,
                         const tam_edits &e, int64_t B, int64_t V, void *logits, int dtype, int64_t row_stride,
                         hipStream_t s) {
    if (dtype == TAM_DTYPE_BF16)
        return launch(rows, num_rows, rows_stride, ids, e, B, V, static_cast<uint16_t *>(logits), row_stride, s);
    return launch(rows, num_rows, rows_stride, ids, e, B, V, static_cast<float *>(logits), row_stride, s);
}

}  // namespace tam
