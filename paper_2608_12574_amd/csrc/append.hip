// The new tokens' K, turned by their positions, and V into their pages, and their queries, turned alike.
//
// Mathematics.  A vector's pairs (x, y) are points of a plane each; pair i of a token at position p turns by the angle p f_i:
//     x' = x cos - y sin,   y' = y cos + x sin
// so that the product of a query and a key depends on how far apart they are.  p f_i reaches 10^5 and more, and what counts is
// its rest after whole turns: the product and the rest are 64-bit (in 32 bits the rest of 10^5 is off by 2^-8), then the
// fraction of a turn, its sine and cosine and the rotation are fp32, and the result is rounded once to the type.
//
// A block takes a token; the sines and cosines are one wave's work, into LDS.  The bytes bound a large call, each read and written
// once: 3,994 tokens of 32 and 8 heads of 128, 98 MB, in 17.8 to 20.5 us (4.8 to 5.5 TB/s; a large
// copy reaches 5.1).  A small one is its chain of reads (the row, its
// slot, length and page): 3 to 5 us.  (With the vectors asked for before the row is known: 21.7 and 4 to 5.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"

namespace tam {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWave = 64, kThreads = 256;

struct Append {
    uint16_t *k, *v;
    int64_t page_stride, head_stride, token_stride;
    const uint16_t *k_new, *v_new, *q;
    uint16_t *out;
    int64_t k_token, k_head, v_token, v_head, q_token, q_head, out_token, out_head;
    const int32_t *table, *length, *offsets, *slot_ids, *depth;
    const float *frequencies;
    int64_t table_stride, slots, max_pages, pages, rows, tokens;
    int32_t shift, heads, kv_heads, dim, pairs;
};

// The row of a token, the last one that starts at or before it, and where it and the next one start: row < 0 for a token of no row.
// A wave looks at 64 offsets in each turn, so that up to 64 rows take one trip to memory.
struct Where {
    int64_t row;
    int32_t first, next;
};

__device__ inline Where where_is(const int32_t *offsets, int64_t rows, int64_t t) {
    const int lane = threadIdx.x % kWave;
    int64_t lo = 0, n = rows;  // offsets[lo] <= t < offsets[lo + n]
    int32_t first = offsets[0];
    const int32_t end = offsets[rows];
    while (true) {
        const int64_t step = (n + kWave - 1) / kWave, at = (lane + 1) * step;
        const int32_t x = offsets[lo + min(at, n)];
        if (t < first || t >= end) return Where{-1, 0, 0};
        const int skip = __popcll(__ballot(at < n && x <= t));
        if (skip) first = __builtin_amdgcn_readlane(x, skip - 1);
        lo += skip * step;
        n = min(step, n - skip * step);
        if (n <= 1) return Where{lo, first, __builtin_amdgcn_readlane(x, min(skip, kWave - 1))};
    }
}

template <bool kHalf>
__device__ inline float to_float(uint32_t x) {
    if constexpr (kHalf) return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
    else return __uint_as_float(x << 16);
}

template <bool kHalf>
__device__ inline uint32_t pack(float x, float y) {  // rounded to nearest, ties to even
    if constexpr (kHalf) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, h2{(_Float16)x, (_Float16)y});
    } else {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, b2{(__bf16)x, (__bf16)y});
    }
}

constexpr int kMaxPairs = 64;  // of a head of 128

// A head's vector in pieces of eight elements: four pairs, as elements 4 j .. of the first half and of the second, or as eight
// adjacent ones; what is not turned follows, in eights (halves of a multiple of four: see the entry point's checks).
template <bool kHalf, bool kAdjacent>
__global__ void __launch_bounds__(kThreads) k_append(Append a) {
    __shared__ float cosines[kMaxPairs], sines[kMaxPairs];
    const int64_t t = blockIdx.x;
    int64_t row = t, j = 0, n = 1;
    if (a.offsets) {
        const Where w = where_is(a.offsets, a.rows, t);
        if (w.row < 0) return;
        row = w.row;
        j = t - w.first;
        n = (int64_t)w.next - w.first;
    } else if (t >= a.rows) {
        return;
    }
    const int64_t slot = a.slot_ids ? a.slot_ids[row] : row;
    const bool in = slot >= 0 && slot < a.slots;
    const int64_t begin = (in ? (int64_t)a.length[slot] : 0) - n, place = begin + j;
    if ((int)threadIdx.x < a.pairs) {
        const double turns = (double)(a.depth ? begin + a.depth[t] : place) * (double)a.frequencies[threadIdx.x] * 0.15915494309189533577;
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        cosines[threadIdx.x] = c;
        sines[threadIdx.x] = s;
    }
    __syncthreads();
    int64_t to = -1;
    if (in && place >= 0 && (place >> a.shift) < a.max_pages) {
        const int64_t page = a.table[slot * a.table_stride + (place >> a.shift)];
        if (page >= 0 && page < a.pages) to = page * a.page_stride + (place & ((1ll << a.shift) - 1)) * a.token_stride;
    }
    const int pieces = a.dim / 8, turned = a.pairs / 4;
    const int vectors = a.heads + 2 * a.kv_heads;
    for (int x = threadIdx.x; x < vectors * pieces; x += kThreads) {
        const int head = x / pieces, p = x - head * pieces;
        const uint16_t *src;
        uint16_t *dst;
        bool turn = p < turned;
        if (head < a.heads) {
            src = a.q + t * a.q_token + head * a.q_head;
            dst = a.out + t * a.out_token + head * a.out_head;
        } else if (to < 0) {
            break;
        } else if (head < a.heads + a.kv_heads) {
            src = a.k_new + t * a.k_token + (head - a.heads) * a.k_head;
            dst = a.k + to + (head - a.heads) * a.head_stride;
        } else {
            src = a.v_new + t * a.v_token + (head - a.heads - a.kv_heads) * a.v_head;
            dst = a.v + to + (head - a.heads - a.kv_heads) * a.head_stride;
            turn = false;
        }
        const bool split = !kAdjacent && p < turned;  // the piece's two fours lie apart
        const int d0 = split ? 4 * p : 8 * p, d1 = split ? d0 + a.pairs : d0 + 4;
        const u32x2 l = *reinterpret_cast<const u32x2 *>(src + d0), h = *reinterpret_cast<const u32x2 *>(src + d1);
        if (!turn) {
            *reinterpret_cast<u32x2 *>(dst + d0) = l;
            *reinterpret_cast<u32x2 *>(dst + d1) = h;
            continue;
        }
        uint32_t e[8];  // elements
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = l[i / 2] >> 16 * (i % 2) & 0xFFFFu;
            e[4 + i] = h[i / 2] >> 16 * (i % 2) & 0xFFFFu;
        }
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int u = kAdjacent ? 2 * i : i, w = kAdjacent ? 2 * i + 1 : 4 + i;
            const float c = cosines[4 * p + i], s = sines[4 * p + i], f = to_float<kHalf>(e[u]), g = to_float<kHalf>(e[w]);
            y[u] = f * c - g * s;
            y[w] = g * c + f * s;
        }
        *reinterpret_cast<u32x2 *>(dst + d0) = u32x2{pack<kHalf>(y[0], y[1]), pack<kHalf>(y[2], y[3])};
        *reinterpret_cast<u32x2 *>(dst + d1) = u32x2{pack<kHalf>(y[4], y[5]), pack<kHalf>(y[6], y[7])};
    }
}

}  // namespace

hipError_t launch_pages_append(const tam_chunk &c, const tam_rotation &r, const Fresh &x, hipStream_t s) {
    const Append a{static_cast<uint16_t *>(c.k), static_cast<uint16_t *>(c.v), c.page_stride, c.head_stride, c.token_stride,
                   static_cast<const uint16_t *>(x.k), static_cast<const uint16_t *>(x.v), static_cast<const uint16_t *>(x.q),
                   static_cast<uint16_t *>(x.out), x.k_token, x.k_head, x.v_token, x.v_head, x.q_token, x.q_head, x.out_token,
                   x.out_head, c.table, c.length, c.offsets, c.slot_ids, r.depth, r.frequencies, c.table_stride, c.slots,
                   c.max_pages, c.num_pages, c.rows, c.tokens, __builtin_ctzll((unsigned long long)c.page_tokens),
                   (int32_t)x.heads, (int32_t)c.kv_heads, (int32_t)c.head_dim, (int32_t)r.pairs};
    const bool half = c.dtype == TAM_DTYPE_FP16;
    void (*kernel)(Append) = half ? (r.adjacent ? k_append<true, true> : k_append<true, false>)
                                  : (r.adjacent ? k_append<false, true> : k_append<false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)c.tokens), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace tam
