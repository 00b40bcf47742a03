// Penalties, biases and the grammar's mask on [B, V] logits, in place.
//
// k_adjust: a block takes one span of one row's vocabulary.  A span without a valid token (most of
// a constrained row's) is -inf, and nothing else is looked at.  Else the block counts
// the row's text in a table in LDS with one word per token of the span (an integer sum,
// so the order of the atomics does not matter), and then goes through the span's logits
// in 16-byte chunks: a chunk without a valid token is stored as -inf and not read, one
// whose valid tokens are not named is left alone or merged, and only the named
// tokens are computed.  So a logit is read and written at most once, and the text
// is all that is read beside the mask; each block of a row reads that again, from L2.
//
// k_edit: without a mask, or before it, only the named tokens are gone to.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"
#include "tam_internal.hpp"

namespace tam {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A table word: occurrences after the prompt (bits 0-18), seen in the prompt (bit
// 19), the last entry of the bias list that names the token, plus one (bits 20-31).
constexpr uint32_t kSeen = 1u << 19, kCount = kSeen - 1;
constexpr int kEntry = 20;
static_assert(TAM_MAX_HISTORY == kCount && TAM_MAX_BIASES == (1 << (32 - kEntry)) - 1, "fields of a table word");

// Threads and tokens of a block, with a mask and without.  The text is read again by each block of a row,
// but more threads hold more of the chip back while one waits: us per call of 256 bf16 rows over
// V = 262,144 (texts of 2,048, a mask) with 256 threads and 4,096 tokens 47, 512 and 8,192 50, 512 and
// 4,096 68, 1,024 and 8,192 78, 128 and 2,048 56 (before the named tokens had a bitmap, which made 45 of the 47); of 64 fp32 rows over V = 128,255 (texts of 8,192, no
// mask) 21, 18, 21, 20, 26.
constexpr int kMaskThreads = 256, kMaskSpan = 4096, kFreeThreads = 512, kFreeSpan = 8192;

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

template <typename T, int kThreads, int kSpan>
__global__ void __launch_bounds__(kThreads) k_adjust(const uint64_t *__restrict__ rows, int64_t num_rows,
                                                     int64_t rows_stride, const int32_t *__restrict__ ids, tam_edits e,
                                                     int64_t V, T *__restrict__ logits, int64_t row_stride) {
    constexpr int N = Lane<T>::n;
    __shared__ __align__(16) uint32_t tab[kSpan];
    __shared__ uint32_t bits[kSpan / 32 + 2], named_bits[kSpan / 32];
    const int64_t b = blockIdx.y;
    T *row = logits + b * row_stride;
    // chunk k of the row covers elements [k N - a, (k + 1) N - a), a being the row's
    // place in its first 16 bytes; v0 is the span's first element (-a in the first block)
    const int a = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const int64_t v0 = (int64_t)blockIdx.x * kSpan - a;
    if (v0 >= V) return;
    const int span = (int)min((int64_t)kSpan, V - v0);  // elements of the span, those before 0 among them

    // What needs no other answer sets out first: the row's numbers and its first ids, kBatch per thread.
    constexpr int kBatch = 8;
    const int32_t *text = e.tokens + b * e.tokens_stride;
    const int history = e.tokens ? (int)e.history : 0;
    int32_t ids0[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
        const int i = threadIdx.x + j * kThreads;
        ids0[j] = i < history ? text[i] : -1;
    }
    const int len = e.length ? min(max(e.length[b], 0), history) : history;
    const int prompt = e.prompt ? e.prompt[b] : 0;
    const Edits ed{e.repetition ? e.repetition[b] : 1.f, e.frequency ? e.frequency[b] : 0.f,
                   e.presence ? e.presence[b] : 0.f, e.bias ? e.bias + b * e.bias_stride : nullptr};
    for (int i = threadIdx.x * 4; i < kSpan; i += kThreads * 4) *reinterpret_cast<u32x4 *>(&tab[i]) = u32x4{0, 0, 0, 0};
    for (int i = threadIdx.x; i < kSpan / 32; i += kThreads) named_bits[i] = 0;
    bool any = true;  // some token of the span is valid
    if (rows) {
        const int64_t r = ids[b];
        uint32_t mine = 0;
        if (r >= 0 && r < num_rows) {  // the span's bits, shifted so that bit 0 is element v0
            const uint32_t *src = reinterpret_cast<const uint32_t *>(rows + r * rows_stride);
            const int64_t words = (V + 31) / 32;
            const int sh = (int)(v0 & 31);
            const int64_t w0 = (v0 - sh) / 32;
            for (int i = threadIdx.x; i < kSpan / 32 + 1; i += kThreads) {
                const int64_t w = w0 + i;
                const uint32_t lo = w >= 0 && w < words ? src[w] : 0u, hi = w + 1 < words ? src[w + 1] : 0u;
                bits[i] = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
                mine |= bits[i];
            }
        }
        any = __syncthreads_or(mine);
    } else {
        __syncthreads();
    }
    // The span's chunks, kChunks per thread: without a valid token -inf at once; those that hold both
    // kinds are read while the text is counted.
    constexpr uint32_t kAll = (1u << N) - 1;
    constexpr int kChunks = kSpan / (N * kThreads);
    uint32_t valid[kChunks], inside[kChunks];
    u32x4 x[kChunks];
    const bool inner = v0 >= 0 && span == kSpan;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
        const int o = (threadIdx.x + k * kThreads) * N;
        inside[k] = kAll;  // elements of the chunk that the row has
        if (!inner) {
            if (o >= span) inside[k] = 0;
            if (v0 + o < 0) inside[k] &= kAll << (int)-(v0 + o);
            if (o < span && o + N > span) inside[k] &= kAll >> (o + N - span);
        }
        valid[k] = !rows ? kAll : any ? (bits[o >> 5] >> (o & 31)) & kAll : 0u;
        u32x4 *at = reinterpret_cast<u32x4 *>(row + (v0 + o));
        if (inside[k] == kAll) {
            if (!valid[k]) {
                constexpr uint32_t m = Lane<T>::kMinusInf;
                __builtin_nontemporal_store(u32x4{m, m, m, m}, at);
            } else if (valid[k] != kAll) {
                x[k] = *at;
            }
        }
    }
    if (any) {
        if (e.bias_ids) {
            const int32_t *named = e.bias_ids + b * e.bias_stride;
            for (int i = threadIdx.x; i < (int)e.biases; i += kThreads) {
                const int32_t v = named[i];
                const uint32_t o = (uint32_t)v - (uint32_t)v0;
                if (o < (uint32_t)span) {
                    atomicMax(&tab[o], (uint32_t)(i + 1) << kEntry);
                    atomicOr(&named_bits[o >> 5], 1u << (o & 31));
                }
            }
            __syncthreads();  // the entry's field is final before the counts are added below it
        }
        auto count = [&](int32_t v, int i) {
            // (an id below 0 falls outside, or before the row's first element, where nothing is edited)
            const uint32_t o = (uint32_t)v - (uint32_t)v0;
            if (o < (uint32_t)span && i < len) {
                if (i < prompt)
                    atomicOr(&tab[o], kSeen);
                else
                    atomicAdd(&tab[o], 1u);
                atomicOr(&named_bits[o >> 5], 1u << (o & 31));
            }
        };
#pragma unroll
        for (int j = 0; j < kBatch; ++j) count(ids0[j], threadIdx.x + j * kThreads);
        for (int i0 = threadIdx.x + kThreads * kBatch; i0 < len; i0 += kThreads * kBatch) {
            int32_t v[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) v[j] = i0 + j * kThreads < len ? text[i0 + j * kThreads] : -1;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) count(v[j], i0 + j * kThreads);
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
        const int o = (threadIdx.x + k * kThreads) * N;
        const bool whole = inside[k] == kAll;
        if (!inside[k] || (whole && !valid[k])) continue;
        const uint32_t named = (named_bits[o >> 5] >> (o & 31)) & valid[k];
        const uint32_t edit = (named | ~valid[k]) & inside[k];
        if (!edit) continue;
        if (whole) {
            u32x4 *at = reinterpret_cast<u32x4 *>(row + (v0 + o));
            u32x4 y = valid[k] == kAll ? *at : x[k];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!(valid[k] >> i & 1)) Lane<T>::minus_inf(y, i);
                else if (named >> i & 1) Lane<T>::put(y, i, edited(Lane<T>::get(y, i), tab[o + i], ed));
            }
            __builtin_nontemporal_store(y, at);
        } else {  // the row's ends: element by element
            for (int i = 0; i < N; ++i) {
                if (!(edit >> i & 1)) continue;
                u32x4 y{0, 0, 0, 0};
                T *p = row + (v0 + o + i);
                if (!(valid[k] >> i & 1)) {
                    Lane<T>::minus_inf(y, 0);
                } else {
                    uint32_t raw = 0;
                    __builtin_memcpy(&raw, p, sizeof(T));
                    y[0] = raw;
                    Lane<T>::put(y, 0, edited(Lane<T>::get(y, 0), tab[o + i], ed));
                }
                const uint32_t raw = y[0];
                __builtin_memcpy(p, &raw, sizeof(T));
            }
        }
    }
}

// The edits alone.  A block gathers a row's text and list of biases in a hash table in LDS (a token's word is
// as above), then goes through the table's tokens: only their logits are read and written, and their mask words
// before, where there is a mask.  Its chain of trips to memory bounds it (text, table, mask words, logits: 9.5 us for 9 MB), and for
// long texts the scattered lines.  us per call without a mask, against k_adjust: 64 fp32
// rows over V = 128,256 with texts of 1,024 5.7 and 10.7; 256 bf16 rows over V = 262,144 with texts of 256 6.5 and 35, of
// 2,048 15 and 52, of 8,192 49 and 84.  Where texts name a large part of the vocabulary, going through all
// of it is faster: 64 fp32 rows over V = 128,255 with texts of 8,192 24 and 17.
constexpr int kEditThreads = 1024;
constexpr int kEditMost = 12288;  // entries of text and biases: three quarters of the largest table
constexpr int kEditShare = 16;    // and no more than the vocabulary's 16th part
constexpr int kEditLine = 64;     // neighbouring tokens, a line or two of logits, that go to one block of the row's
// Up to eight blocks share a row while there are no more of them than this (us per call with 1 and 8 blocks a row:
// 16 rows 5.4 and 5.0, 64 rows 5.7 and 6.3).
constexpr int kEditBlocks = 128;
// With a mask, from this many bytes of logits on: the edits of the valid tokens first, then the mask's own pass, whose
// blocks then wait for no text (us per call, in one pass and in two: 256 bf16 rows over V = 262,144 with texts of 2,048
// 45 and 38, over 128,256 with texts of 256 24 and 21; 64 fp32 rows over 128,256 14 and 17).
constexpr int64_t kApartBytes = 48ll << 20;

template <typename T, int kEach>
__global__ void __launch_bounds__(kEditThreads) k_edit(const uint64_t *__restrict__ rows, int64_t num_rows, int64_t rows_stride,
                                                       const int32_t *__restrict__ ids, tam_edits e, int64_t V,
                                                       T *__restrict__ logits, int64_t row_stride) {
    constexpr int kSlots = kEach * kEditThreads, kLog = __builtin_ctz(kSlots);
    extern __shared__ __align__(16) uint32_t table[];  // ids, then words
    uint32_t *const id_of = table, *const word_of = table + kSlots;
    const int64_t b = blockIdx.y;
    const uint64_t *mask = nullptr;  // with a mask: the row's, to leave out tokens that become -inf
    if (rows) {
        const int64_t r = ids[b];
        if (r < 0 || r >= num_rows) return;
        mask = rows + r * rows_stride;
    }
    const uint32_t parts = gridDim.x - 1, part = blockIdx.x;  // (a power of two) - 1; this block's
    T *row = logits + b * row_stride;
    constexpr int kBatch = 4;
    constexpr uint32_t kNone = 0xFFFFFFFFu;  // no token
    const int32_t *text = e.tokens + b * e.tokens_stride;
    const int history = e.tokens ? (int)e.history : 0;
    int32_t ids0[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
        const int i = threadIdx.x + j * kEditThreads;
        ids0[j] = i < history ? text[i] : -1;
    }
    const int len = e.length ? min(max(e.length[b], 0), history) : history;
    const int prompt = e.prompt ? e.prompt[b] : 0;
    const Edits ed{e.repetition ? e.repetition[b] : 1.f, e.frequency ? e.frequency[b] : 0.f,
                   e.presence ? e.presence[b] : 0.f, e.bias ? e.bias + b * e.bias_stride : nullptr};
#pragma unroll
    for (int i = threadIdx.x * 4; i < kSlots; i += kEditThreads * 4) {
        *reinterpret_cast<u32x4 *>(&id_of[i]) = u32x4{kNone, kNone, kNone, kNone};
        *reinterpret_cast<u32x4 *>(&word_of[i]) = u32x4{0, 0, 0, 0};
    }
    __syncthreads();
    auto ours = [&](int32_t v) { return v >= 0 && v < V && ((uint32_t)v / kEditLine & parts) == part; };
    // a token's place: there are more places than entries, so a free one is found
    auto place = [&](int32_t v) {
        uint32_t at = ((uint32_t)v * 0x9E3779B1u) >> (32 - kLog);
        while (true) {
            const uint32_t was = atomicCAS(&id_of[at], kNone, (uint32_t)v);
            if (was == kNone || was == (uint32_t)v) return at;
            at = (at + 1) & (uint32_t)(kSlots - 1);
        }
    };
    if (e.bias_ids) {
        const int32_t *named = e.bias_ids + b * e.bias_stride;
        for (int i = threadIdx.x; i < (int)e.biases; i += kEditThreads) {
            const int32_t v = named[i];
            if (ours(v)) atomicMax(&word_of[place(v)], (uint32_t)(i + 1) << kEntry);
        }
        __syncthreads();  // the entry's field is final before the counts are added below it
    }
    auto count = [&](int32_t v, int i) {
        if (i < len && ours(v)) {
            uint32_t *const w = &word_of[place(v)];
            if (i < prompt)
                atomicOr(w, kSeen);
            else
                atomicAdd(w, 1u);
        }
    };
#pragma unroll
    for (int j = 0; j < kBatch; ++j) count(ids0[j], threadIdx.x + j * kEditThreads);
    for (int i0 = threadIdx.x + kEditThreads * kBatch; i0 < len; i0 += kEditThreads * kBatch) {
        int32_t v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) v[j] = i0 + j * kEditThreads < len ? text[i0 + j * kEditThreads] : -1;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) count(v[j], i0 + j * kEditThreads);
    }
    __syncthreads();
    uint32_t v[kEach];
    uint64_t word[kEach];
    T x[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        v[j] = id_of[threadIdx.x + j * kEditThreads];
        if (mask) word[j] = v[j] != kNone ? mask[v[j] / 64] : 0;
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (mask && !(word[j] >> (v[j] % 64) & 1)) v[j] = kNone;
        if (v[j] != kNone) x[j] = row[v[j]];
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (v[j] == kNone) continue;
        u32x4 y{0, 0, 0, 0};
        uint32_t raw = 0;
        __builtin_memcpy(&raw, &x[j], sizeof(T));
        y[0] = raw;
        Lane<T>::put(y, 0, edited(Lane<T>::get(y, 0), word_of[threadIdx.x + j * kEditThreads], ed));
        raw = y[0];
        __builtin_memcpy(&row[v[j]], &raw, sizeof(T));
    }
}

// the edits of the rows after the first n
void next_rows(tam_edits &e, int64_t n) {
    if (e.tokens) e.tokens += n * e.tokens_stride;
    if (e.bias_ids) e.bias_ids += n * e.bias_stride, e.bias += n * e.bias_stride;
    for (const int32_t **p : {&e.length, &e.prompt})
        if (*p) *p += n;
    for (const float **p : {&e.repetition, &e.frequency, &e.presence})
        if (*p) *p += n;
}

template <typename T, int kThreads, int kSpan>
hipError_t launch(const uint64_t *rows, int64_t num_rows, int64_t rows_stride, const int32_t *ids, tam_edits e,
                  int64_t B, int64_t V, T *logits, int64_t row_stride, hipStream_t s) {
    // a row may start up to 15 bytes into a chunk, which moves its end as far
    const unsigned gx = (unsigned)((V + Lane<T>::n - 1 + kSpan - 1) / kSpan);
    for (int64_t r0 = 0; r0 < B; r0 += 65535) {
        const int64_t n = std::min<int64_t>(B - r0, 65535);
        hipLaunchKernelGGL((k_adjust<T, kThreads, kSpan>), dim3(gx, (unsigned)n), dim3(kThreads), 0, s, rows, num_rows,
                           rows_stride, ids ? ids + r0 : nullptr, e, V, logits + r0 * row_stride, row_stride);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        next_rows(e, n);
    }
    return hipSuccess;
}

template <typename T, int kEach>
hipError_t launch_edit(const uint64_t *rows, int64_t num_rows, int64_t rows_stride, const int32_t *ids, tam_edits e,
                       int64_t B, int64_t V, T *logits, int64_t row_stride, hipStream_t s) {
    unsigned parts = 1;
    while (parts < 8 && B * parts * 2 <= kEditBlocks) parts *= 2;
    for (int64_t r0 = 0; r0 < B; r0 += 65535) {
        const int64_t n = std::min<int64_t>(B - r0, 65535);
        hipLaunchKernelGGL((k_edit<T, kEach>), dim3(parts, (unsigned)n), dim3(kEditThreads), 8 * kEach * kEditThreads, s, rows,
                           num_rows, rows_stride, ids ? ids + r0 : nullptr, e, V, logits + r0 * row_stride, row_stride);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        next_rows(e, n);
    }
    return hipSuccess;
}

// Whether the mask can have a pass of its own.  (That looks at the neighbour of a row's last mask word where logits
// are not 16-byte aligned, and rows of a wider stride may have nothing there.)
template <typename T>
bool own_pass(int64_t rows_stride, int64_t V, const T *logits, int64_t row_stride) {
    const bool aligned = (reinterpret_cast<uintptr_t>(logits) | (uint64_t)(row_stride * sizeof(T))) % 16 == 0;
    return aligned || rows_stride == (V + 63) / 64;
}

template <typename T>
hipError_t launch_type(const uint64_t *rows, int64_t num_rows, int64_t rows_stride, const int32_t *ids,
                       const tam_edits &e, int64_t B, int64_t V, void *logits, int64_t row_stride, hipStream_t s) {
    T *p = static_cast<T *>(logits);
    const int64_t entries = e.history + (e.bias_ids ? e.biases : 0);
    const bool few = entries <= kEditMost && entries <= V / kEditShare, large = B * V * (int64_t)sizeof(T) >= kApartBytes;
    if (rows ? (!entries || (few && large)) && own_pass(rows_stride, V, p, row_stride) : few) {
        if (entries) {
            // tables of 4,096, 8,192 or 16,384 places, at most three quarters of them taken
            const auto edit = entries <= 3 * kEditThreads   ? launch_edit<T, 4>
                              : entries <= 6 * kEditThreads ? launch_edit<T, 8>
                                                            : launch_edit<T, 16>;
            const hipError_t err = edit(rows, num_rows, rows_stride, ids, e, B, V, p, row_stride, s);
            if (err != hipSuccess || !rows) return err;
        }
        DevTables t{};
        t.table = const_cast<uint64_t *>(rows);
        t.Wp = rows_stride;
        t.N = num_rows;
        t.V = V;
        return launch_apply(t, ids, B, logits, sizeof(T) == 2 ? TAM_DTYPE_BF16 : TAM_DTYPE_FP32, row_stride, s);
    }
    return rows ? launch<T, kMaskThreads, kMaskSpan>(rows, num_rows, rows_stride, ids, e, B, V, p, row_stride, s)
                : launch<T, kFreeThreads, kFreeSpan>(rows, num_rows, rows_stride, ids, e, B, V, p, row_stride, s);
}

}  // namespace

hipError_t launch_adjust(const uint64_t *rows, int64_t num_rows, int64_t rows_stride, const int32_t *ids,
                         const tam_edits &e, int64_t B, int64_t V, void *logits, int dtype, int64_t row_stride,
                         hipStream_t s) {
    if (dtype == TAM_DTYPE_BF16)
        return launch_type<uint16_t>(rows, num_rows, rows_stride, ids, e, B, V, logits, row_stride, s);
    return launch_type<float>(rows, num_rows, rows_stride, ids, e, B, V, logits, row_stride, s);
}

}  // namespace tam
