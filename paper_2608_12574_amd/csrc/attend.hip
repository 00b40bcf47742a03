// Attention of a chunk of new tokens per sequence over a paged K/V cache.
//
// k_attend_rows: a wave per (token, head), 64 keys at a time: each lane takes one
// key's product with the query, the running maximum and sum of the softmax go over the
// wave, then every lane adds the weighted V of its dimensions.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"

namespace tam {
namespace {

constexpr int kWave = 64;

struct Attend {
    const uint16_t *k, *v, *q;
    uint16_t *out;
    float *lse;
    int64_t page_stride, head_stride, token_stride, q_token, q_head, out_token, out_head;
    const int32_t *table, *length, *offsets, *slot_ids;
    int64_t table_stride, slots, max_pages, rows, tokens;
    int32_t pages, shift, heads, kv_heads, dim;
    float scale;
};

template <bool kHalf>
__device__ float wide(uint16_t h) {
    if constexpr (kHalf) return (float)__builtin_bit_cast(_Float16, h);
    return __uint_as_float((uint32_t)h << 16);
}
template <bool kHalf>
__device__ uint16_t narrow(float x) {
    if constexpr (kHalf) return __builtin_bit_cast(uint16_t, (_Float16)x);
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

template <bool kHalf>
__global__ void __launch_bounds__(kWave) k_attend_rows(Attend a) {
    __shared__ float weight[kWave];
    __shared__ int64_t place[kWave];
    const int64_t t = blockIdx.x;
    const int h = blockIdx.y, lane = threadIdx.x;
    int64_t row = t, j = 0, n = 1;
    if (a.offsets) {
        if (t < a.offsets[0] || t >= a.offsets[a.rows]) return;
        int64_t hi = a.rows;
        row = 0;
        while (hi - row > 1) {
            const int64_t mid = (row + hi) >> 1;
            if (a.offsets[mid] <= t) row = mid;
            else hi = mid;
        }
        j = t - a.offsets[row];
        n = (int64_t)a.offsets[row + 1] - a.offsets[row];
    } else if (t >= a.rows) {
        return;
    }
    const int64_t slot = a.slot_ids ? a.slot_ids[row] : row;
    const int64_t most = a.max_pages << a.shift;
    const int64_t len = slot >= 0 && slot < a.slots ? a.length[slot] : 0;
    const int64_t keys = min(len - n + j + 1, most);  // visible keys
    const uint16_t *q = a.q + t * a.q_token + h * a.q_head;
    const int kvh = h / (a.heads / a.kv_heads);
    float top = -INFINITY, sum = 0.f, acc[2] = {0.f, 0.f};
    for (int64_t k0 = 0; k0 < keys; k0 += kWave) {
        const int64_t key = k0 + lane;
        float s = -INFINITY;
        int64_t at = -1;
        if (key < keys) {
            const int32_t page = a.table[slot * a.table_stride + (key >> a.shift)];
            if ((uint32_t)page < (uint32_t)a.pages) {
                at = page * a.page_stride + kvh * a.head_stride + (key & ((1ll << a.shift) - 1)) * a.token_stride;
                s = 0.f;
                for (int d = 0; d < a.dim; ++d) s += wide<kHalf>(q[d]) * wide<kHalf>(a.k[at + d]);
                s *= a.scale;
            }
        }
        float m = s;
        for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
        m = fmaxf(m, top);
        const float p = m == -INFINITY ? 0.f : __expf(s - m), keep = m == -INFINITY ? 1.f : __expf(top - m);
        float total = p;
        for (int d = 1; d < kWave; d <<= 1) total += __shfl_xor(total, d);
        sum = sum * keep + total;
        top = m;
        weight[lane] = p;
        place[lane] = at;
        __syncthreads();
        for (int i = 0; i < 2; ++i) {
            const int d = lane + i * kWave;
            acc[i] *= keep;
            if (d < a.dim)
                for (int x = 0; x < kWave; ++x)
                    if (place[x] >= 0) acc[i] += weight[x] * wide<kHalf>(a.v[place[x] + d]);
        }
        __syncthreads();
    }
    for (int i = 0; i < 2; ++i) {
        const int d = lane + i * kWave;
        if (d < a.dim)
            a.out[t * a.out_token + h * a.out_head + d] = narrow<kHalf>(sum > 0.f ? acc[i] / sum : 0.f);
    }
    if (lane == 0 && a.lse) a.lse[t * a.heads + h] = sum > 0.f ? top + __logf(sum) : -INFINITY;
}

}  // namespace

int64_t attend_work_bytes(const tam_chunk &, int64_t) { return 0; }

hipError_t launch_attend(const tam_chunk &c, const Queries &q, void *, hipStream_t s) {
    const Attend a{static_cast<const uint16_t *>(c.k), static_cast<const uint16_t *>(c.v),
                   static_cast<const uint16_t *>(q.q), static_cast<uint16_t *>(q.out), q.lse, c.page_stride,
                   c.head_stride, c.token_stride, q.q_token, q.q_head, q.out_token, q.out_head, c.table, c.length,
                   c.offsets, c.slot_ids, c.table_stride, c.slots, c.max_pages, c.rows, c.tokens, (int32_t)c.num_pages,
                   __builtin_ctzll((unsigned long long)c.page_tokens), (int32_t)q.heads, (int32_t)c.kv_heads,
                   (int32_t)c.head_dim, q.scale};
    const dim3 grid((unsigned)c.tokens, (unsigned)q.heads);
    if (c.dtype == TAM_DTYPE_FP16)
        hipLaunchKernelGGL((k_attend_rows<true>), grid, dim3(kWave), 0, s, a);
    else
        hipLaunchKernelGGL((k_attend_rows<false>), grid, dim3(kWave), 0, s, a);
    return hipGetLastError();
}

}  // namespace tam
