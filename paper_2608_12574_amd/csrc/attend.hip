// Attention of a chunk of new tokens per sequence over a paged K/V cache.
//
// Mathematics.  For a query q, o = sum_j w_j v_j / sum_j w_j with w_j = exp(scale (q k_j - m)),
// for any m; in one pass over the keys m is the running maximum, and what was summed
// under an older m is scaled when m grows.  Parts of the keys summed apart join the
// same way.  m is let lag by up to 2^8 in w before it is moved, which the fp32 sums
// and the 16-bit weights hold, so that the sums are scaled a few times per row and
// not in each step.
//
// A tile is `tq` tokens of one row, times the heads that share a K/V head (their
// rows of a product are side by side, so K and V are read once for all of them).
// A unit is a tile's product with kKeys keys.  All units of a call, row after row,
// head after head, tile after tile, are one line, cut into equal pieces for as
// many blocks as the chip holds: any mix of long and short rows and chunks fills
// it evenly.  A tile that a cut goes through leaves partial sums in the scratch, which
// k_join adds up.  The lengths lie on the device: each block finds its piece from
// them by a prefix sum over the rows.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"

namespace tam {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kWave = 64;
constexpr int kThreads = 256;

// Bad page numbers point here: V of zeros.  (Addresses of memory are told from those of LDS
// here, so that a load does not wait as if it could be of either.)
__device__ u32x4 kZeros[16];
typedef __attribute__((address_space(1))) const uint16_t global_u16;
typedef __attribute__((address_space(1))) const u32x4 global_u32x4;
typedef __attribute__((address_space(1))) const u32x2 global_u32x2;
__device__ inline global_u16 *zeros() { return (global_u16 *)kZeros; }

struct Attend {
    const uint16_t *k, *v, *q;
    uint16_t *out;
    float *lse;
    int64_t page_stride, head_stride, token_stride, q_token, q_head, out_token, out_head;
    const int32_t *table, *length, *offsets, *slot_ids;
    int64_t table_stride, slots, max_pages, rows, tokens;
    int32_t pages, shift, heads, kv_heads, dim;
    float scale;
    // the cut: tiles of `tq` tokens by `group` heads, `parts` of them per K/V head
    int32_t tq, group, parts, blocks;
    int32_t least;  // units of a block, at least
    float *sums;    // [2 blocks][tile rows][DP] partial sums, then [2 blocks][tile rows][2] their m and sum of weights
    struct Cut *cuts;  // [blocks] what each block's piece begins with
};

// The tile that a block's piece begins in, if in its middle (units done before it: > 0).
struct Cut {
    int64_t done, units, piece;
    int32_t token, n, head, heads;  // its first token and query head, and how many
};

// a value that is the same in all lanes, to the compiler too
__device__ inline int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
    return (int64_t)(uint32_t)uniform((int32_t)x) | (int64_t)uniform((int32_t)(x >> 32)) << 32;
}

// ------------------------------------------------------------------ the cut ---

// sum of floor((a t + b) / m) over t in [0, n), by Euclid's steps on (a, m)
__device__ inline int64_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
    int64_t sum = 0;
    while (true) {
        if (a >= m) {
            sum += (int64_t)n * (n - 1) / 2 * (a / m);
            a %= m;
        }
        if (b >= m) {
            sum += (int64_t)n * (b / m);
            b %= m;
        }
        const uint64_t y = (uint64_t)a * n + b;
        if (y < m) return sum;
        n = (uint32_t)(y / m);
        b = (uint32_t)(y % m);
        const uint32_t t = m;
        m = a;
        a = t;
    }
}

struct Row {
    int32_t n, base;    // tokens of the chunk; tokens of the sequence before it (may be negative)
    int32_t first;      // the chunk's first token
    int64_t slot;
};

__device__ inline Row row_at(const Attend &a, int64_t i) {
    Row r;
    if (a.offsets) {
        const int64_t lo = max((int64_t)a.offsets[i], (int64_t)0), hi = min((int64_t)a.offsets[i + 1], a.tokens);
        r.first = (int32_t)lo;
        r.n = (int32_t)max(hi - lo, (int64_t)0);
    } else {
        r.first = (int32_t)i;
        r.n = i < a.tokens;
    }
    r.slot = a.slot_ids ? a.slot_ids[i] : i;
    int64_t len = 0;
    if (r.slot >= 0 && r.slot < a.slots) len = min(max((int64_t)a.length[r.slot], (int64_t)0), a.max_pages << a.shift);
    r.base = (int32_t)(len - r.n);
    return r;
}

// the same for a row number that all lanes share
__device__ inline Row shared_row(const Attend &a, int64_t i) {
    Row r = row_at(a, i);
    r.n = uniform(r.n);
    r.base = uniform(r.base);
    r.first = uniform(r.first);
    r.slot = uniform(r.slot);
    return r;
}

// Units of the tiles before tile t of a row (all of them full).
template <int kKeys>
__device__ inline int64_t units_before(const Attend &a, const Row &r, uint32_t t) {
    return t ? floor_sum(t, kKeys, a.tq, max(r.base, 0) + a.tq + kKeys - 1) : 0;
}

template <int kKeys>
__device__ inline int64_t row_units(const Attend &a, const Row &r) {
    if (r.n == 0) return 0;
    const uint32_t tiles = (r.n + a.tq - 1) / a.tq;
    return units_before<kKeys>(a, r, tiles - 1) + (max(r.base, 0) + r.n + kKeys - 1) / kKeys;
}

// A place on the line of units.
struct Place {
    int64_t row, total;   // the row; units of all rows
    int64_t rest;         // units of the row before this place
};

// The place of unit number `share * piece` (share: this block's number), and the units of a
// piece.  All threads of the block call it; row < 0 past the line's end.
template <int kKeys, int kN = kThreads>
__device__ inline Place find(const Attend &a, int64_t share, int64_t *piece) {
    __shared__ int64_t sums[kN / kWave];
    __shared__ int64_t found[2];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t per = (a.rows + kN - 1) / kN, lo = threadIdx.x * per, hi = min(lo + per, a.rows);
    const int64_t heads = (int64_t)a.kv_heads * a.parts;
    int64_t mine = 0;
    for (int64_t i = lo; i < hi; ++i) mine += heads * row_units<kKeys>(a, row_at(a, i));
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int64_t up = __shfl_up(upto, d);
        if (lane >= d) upto += up;
    }
    if (lane == kWave - 1) sums[wave] = upto;
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    Place p;
    p.total = 0;
#pragma unroll
    for (int w = 0; w < kN / kWave; ++w) {
        if (w < wave) upto += sums[w];
        p.total += sums[w];
    }
    p.total = uniform(p.total);
    *piece = max((int64_t)a.least, (p.total + a.blocks - 1) / a.blocks);
    const int64_t at = share * *piece;
    if (at >= upto - mine && at < upto) {  // one thread: walk its rows
        int64_t rest = at - (upto - mine);
        int64_t i = lo;
        for (; i < hi; ++i) {
            const int64_t u = heads * row_units<kKeys>(a, row_at(a, i));
            if (rest < u) break;
            rest -= u;
        }
        found[0] = i;
        found[1] = rest;
    }
    __syncthreads();
    p.row = uniform(found[0]);
    p.rest = uniform(found[1]);
    return p;
}

// A tile, and the units of it before the place.
struct Tile {
    int32_t head, part, tile;     // K/V head and part of its group; number in the row
    int32_t first, n;             // its first token in the chunk, and its tokens
    int32_t heads;                // query heads of the part
    int64_t units, done;
};

template <int kKeys>
__device__ inline Tile tile_at(const Attend &a, const Row &r, int64_t rest) {
    const int64_t u = row_units<kKeys>(a, r);
    const int64_t vh = rest / u;
    rest -= vh * u;
    const uint32_t tiles = (r.n + a.tq - 1) / a.tq;
    uint32_t lo = 0, hi = tiles;  // units_before(lo) <= rest < units_before(hi)
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (units_before<kKeys>(a, r, mid) <= rest) lo = mid;
        else hi = mid;
    }
    Tile t;
    t.head = (int32_t)(vh / a.parts);
    t.part = (int32_t)(vh - (int64_t)t.head * a.parts);
    t.tile = (int32_t)lo;
    t.first = t.tile * a.tq;
    t.n = min(a.tq, r.n - t.first);
    t.heads = min(a.group, a.heads / a.kv_heads - t.part * a.group);
    t.done = rest - units_before<kKeys>(a, r, lo);
    t.units = (max(r.base, 0) + min((int32_t)((lo + 1) * a.tq), r.n) + kKeys - 1) / kKeys;
    return t;
}

// What the block's piece begins with, for k_join.
__device__ inline void note(const Attend &a, int64_t block, const Row &r, const Tile &t, int64_t piece) {
    if (threadIdx.x == 0)
        a.cuts[block] = Cut{t.done, t.units, piece, r.first + t.first, t.n,
                            t.head * (a.heads / a.kv_heads) + t.part * a.group, t.heads};
}

// ------------------------------------------------------------------ products ---

template <bool kHalf>
__device__ inline f32x4 mfma16(u32x4 x, u32x4 y, f32x4 z) {
    if constexpr (kHalf)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), z, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), z, 0, 0, 0);
}

template <bool kHalf>
__device__ inline f32x16 mfma32(u32x4 x, u32x4 y, f32x16 z) {
    if constexpr (kHalf)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), z, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), z, 0, 0, 0);
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

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLag = 8.f;  // m may lag by this much, in powers of two

// A tile of at most 16 kBlocks kRowWaves rows by all its keys, 32 keys per wave and
// step; kRowWaves waves share the rows and the others the keys of a unit.  The bytes of
// K and V bound it, so the fragments come straight from memory into registers, the next
// step's while this one is computed, and LDS only joins the waves' sums at the end.
// S^T = K Q^T leaves each lane the weights of one query, for the same eight keys that it
// then holds as the second factor of O^T = V^T P^T: no weight changes lanes.  V's columns
// are paired in registers (v_perm).
template <int DP, int kBlocks, int kRowWaves, bool kHalf>
__global__ void __launch_bounds__(kThreads, kBlocks == 1 ? 2 : 1) k_attend_narrow(Attend a) {
    constexpr int kKeyWaves = 4 / kRowWaves, kKeys = 32 * kKeyWaves;
    constexpr int kSteps = DP / 32;  // products of 32 dimensions
    constexpr int kCols = DP / 16;   // dimensions per lane of 16: adjacent ones
    constexpr int kRows = 16 * kBlocks * kRowWaves;
    __shared__ float joint[4][16][DP + 4];
    __shared__ float tops[4][16 * kBlocks], weights[4][16 * kBlocks];
    const int lane = threadIdx.x % kWave, wave = uniform((int32_t)threadIdx.x / kWave);
    const int rw = wave / kKeyWaves, kw = wave % kKeyWaves;
    const int col = lane % 16, grp = lane / 16;
    int64_t piece;
    Place p = find<kKeys>(a, blockIdx.x, &piece);
    if (p.row < 0) {
        if (threadIdx.x == 0) a.cuts[blockIdx.x].done = 0;
        return;
    }
    const int64_t from = blockIdx.x * piece;
    const int64_t whole_piece = min(piece, p.total - from);
    int64_t left = whole_piece;
    const float c = a.scale * kLog2e;
    while (left > 0) {
        const Row r = shared_row(a, p.row);
        const int64_t in_row = row_units<kKeys>(a, r) * a.kv_heads * a.parts;
        if (p.rest >= in_row) {
            ++p.row;
            p.rest = 0;
            continue;
        }
        const Tile t = tile_at<kKeys>(a, r, p.rest);
        const int64_t take = min(t.units - t.done, left);
        if (left == whole_piece) note(a, blockIdx.x, r, t, piece);
        // queries, one per lane of 16 and block; rows past the tile's see no key.  Lanes
        // past the last dimension read others of the vector (queries: zero).
        u32x4 q[kBlocks][kSteps];
        int32_t seen[kBlocks];  // keys that the query sees
        const int32_t all = max(0, r.base + r.n);  // tokens of the sequence, chunk included
        const int32_t most = max(0, min(r.base + t.first + t.n, all)), least = max(0, min(r.base + t.first + 1, all));
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int row = 16 * (kBlocks * rw + b) + col, tok = row / t.heads, h = row - tok * t.heads;
            const bool is = tok < t.n;
            seen[b] = is ? max(0, min(r.base + t.first + tok + 1, all)) : 0;
            const uint16_t *src = a.q + (int64_t)(r.first + t.first + tok) * a.q_token +
                                  (int64_t)(t.head * (a.heads / a.kv_heads) + t.part * a.group + h) * a.q_head;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int d = 32 * s + 8 * grp;
                q[b][s] = is && d < a.dim ? *reinterpret_cast<const u32x4 *>(src + d) : u32x4{0, 0, 0, 0};
            }
        }
        f32x4 o[kBlocks][kCols];
        float m[kBlocks], l[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            m[b] = -INFINITY;
            l[b] = 0.f;
#pragma unroll
            for (int j = 0; j < kCols; ++j) o[b][j] = f32x4{0, 0, 0, 0};
        }
        global_u16 *kh = (global_u16 *)(a.k + (int64_t)t.head * a.head_stride);
        global_u16 *vh = (global_u16 *)(a.v + (int64_t)t.head * a.head_stride + (kCols * col < a.dim ? kCols * col : 0));
        const int32_t *pages = a.table + r.slot * a.table_stride;
        const int32_t place = (1 << a.shift) - 1;

        struct Step {
            u32x4 k[2][kSteps];
            u32x4 v[8];  // kCols * 2 bytes of each are used
            uint32_t bad;  // bit j: key j of the lane's eight lies in no page
        };
        // The keys of a step; those past the last one that the tile sees stand for it.
        auto load = [&](int32_t k0, Step &x) {
            x.bad = 0;
            global_u16 *src[8];
            const int32_t first = k0 + 4 * grp;
            if (k0 + 32 <= most && a.shift >= 2) {  // four keys lie side by side
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int32_t key = first + 16 * i, page = pages[key >> a.shift];
                    const bool ok = (uint32_t)page < (uint32_t)a.pages;
                    if (!ok) x.bad |= 15u << 4 * i;
                    global_u16 *at = ok ? vh + (int64_t)page * a.page_stride + (int64_t)(key & place) * a.token_stride : zeros();
                    const int64_t step = ok ? a.token_stride : 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) src[4 * i + j] = at + j * step;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int32_t key = min(first + 16 * (j / 4) + j % 4, most - 1), page = pages[key >> a.shift];
                    const bool ok = (uint32_t)page < (uint32_t)a.pages;
                    if (!ok) x.bad |= 1u << j;
                    src[j] = ok ? vh + (int64_t)page * a.page_stride + (int64_t)(key & place) * a.token_stride : zeros();
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int32_t key = min(k0 + 16 * i + col, most - 1), page = pages[key >> a.shift];
                global_u16 *at = kh + (int64_t)((uint32_t)page < (uint32_t)a.pages ? page : 0) * a.page_stride +
                                     (int64_t)(key & place) * a.token_stride;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int d = 32 * s + 8 * grp;
                    x.k[i][s] = *(global_u32x4 *)(at + (d < a.dim ? d : 0));
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (kCols == 8) {
                    x.v[j] = *(global_u32x4 *)src[j];
                } else {
                    const u32x2 y = *(global_u32x2 *)src[j];
                    x.v[j] = u32x4{y[0], y[1], 0, 0};
                }
            }
        };
        auto compute = [&](int32_t k0, const Step &x) {
            u32x4 v[kCols];
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[j][i] = __builtin_amdgcn_perm(x.v[2 * i + 1][j / 2], x.v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
            const bool masked = k0 + 32 > least || __any(x.bad);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                f32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int d = 0; d < kSteps; ++d) s[i] = mfma16<kHalf>(x.k[i][d], q[b][d], s[i]);
                if (masked) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (k0 + 16 * (j / 4) + 4 * grp + j % 4 >= seen[b] || (x.bad >> j & 1)) s[j / 4][j % 4] = -INFINITY;
                }
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, s[j / 4][j % 4]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (__any((top - m[b]) * c > kLag)) {  // NaN (both -inf): no
                    const float now = fmaxf(m[b], top);
                    const float keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[b] - now) * c);
                    m[b] = now;
                    l[b] *= keep;
#pragma unroll
                    for (int j = 0; j < kCols; ++j) o[b][j] *= keep;
                }
                const float mc = m[b] == -INFINITY ? 0.f : m[b] * c;
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j / 4][j % 4], c, -mc));
                    l[b] += w[j];
                }
                u32x4 pw;
#pragma unroll
                for (int i = 0; i < 4; ++i) pw[i] = pack<kHalf>(w[2 * i], w[2 * i + 1]);
#pragma unroll
                for (int j = 0; j < kCols; ++j) o[b][j] = mfma16<kHalf>(v[j], pw, o[b][j]);
            }
        };
        const int32_t k_end = (int32_t)min((t.done + take) * kKeys, (int64_t)most);
        int32_t k0 = (int32_t)(t.done * kKeys) + 32 * kw;
        if (k0 < k_end) {
            Step x, y;
            load(k0, x);
            while (true) {
                int32_t k1 = k0 + kKeys;
                if (k1 < k_end) load(k1, y);
                compute(k0, x);
                if (k1 >= k_end) break;
                k0 = k1 + kKeys;
                if (k0 < k_end) load(k0, x);
                compute(k1, y);
                if (k0 >= k_end) break;
            }
        }
        // join the waves that shared the keys: the largest m, then the sums under it
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            l[b] += __shfl_xor(l[b], 16);
            l[b] += __shfl_xor(l[b], 32);
            if (grp == 0) {
                tops[wave][16 * b + col] = m[b];
                weights[wave][16 * b + col] = l[b];
            }
        }
        __syncthreads();
        const bool whole = take == t.units;
        const int64_t at = 2 * (int64_t)blockIdx.x + (t.done == 0);  // a cut tile's partial sums
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kKeyWaves; ++w) top = fmaxf(top, tops[rw * kKeyWaves + w][16 * b + col]);
            const float keep = m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[b] - top) * c);
            // o[b][j][i] is dimension kCols (4 grp + i) + j of query `col`
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kCols; j += 4)
                    *reinterpret_cast<f32x4 *>(&joint[wave][col][kCols * (4 * grp + i) + j]) =
                        f32x4{o[b][j][i], o[b][j + 1][i], o[b][j + 2][i], o[b][j + 3][i]} * keep;
            __syncthreads();
            // a thread takes one query of each wave's rows and kCols dimensions
            const int qr = threadIdx.x / 16, d0 = kCols * (threadIdx.x % 16);
#pragma unroll
            for (int x = 0; x < kRowWaves; ++x) {
                const int out_row = 16 * (kBlocks * x + b) + qr, tok = out_row / t.heads, h = out_row - tok * t.heads;
                if (tok >= t.n) continue;
                float sum[kCols] = {}, lsum = 0.f, mx = -INFINITY;
#pragma unroll
                for (int w = 0; w < kKeyWaves; ++w) mx = fmaxf(mx, tops[x * kKeyWaves + w][16 * b + qr]);
#pragma unroll
                for (int w = 0; w < kKeyWaves; ++w) {
                    const int of = x * kKeyWaves + w;
                    const float mw = tops[of][16 * b + qr];
                    if (mw > -INFINITY) lsum += weights[of][16 * b + qr] * __builtin_amdgcn_exp2f((mw - mx) * c);
#pragma unroll
                    for (int j = 0; j < kCols; ++j) sum[j] += joint[of][qr][d0 + j];
                }
                if (whole) {
                    const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
                    const int64_t token = r.first + t.first + tok;
                    const int64_t head = t.head * (a.heads / a.kv_heads) + t.part * a.group + h;
                    uint16_t *dst = a.out + token * a.out_token + head * a.out_head + d0;
                    if (d0 < a.dim) {
                        uint32_t y[kCols / 2];
#pragma unroll
                        for (int j = 0; j < kCols / 2; ++j) y[j] = pack<kHalf>(sum[2 * j] * inv, sum[2 * j + 1] * inv);
                        if constexpr (kCols == 8) *reinterpret_cast<u32x4 *>(dst) = u32x4{y[0], y[1], y[2], y[3]};
                        else *reinterpret_cast<u32x2 *>(dst) = u32x2{y[0], y[1]};
                    }
                    if (a.lse && d0 == 0)
                        a.lse[token * a.heads + head] = lsum > 0.f ? mx * a.scale + logf(lsum) : -INFINITY;
                } else {
                    float *dst = a.sums + (at * kRows + out_row) * DP + d0;
#pragma unroll
                    for (int j = 0; j < kCols; j += 4)
                        *reinterpret_cast<f32x4 *>(dst + j) = f32x4{sum[j], sum[j + 1], sum[j + 2], sum[j + 3]};
                    if (d0 == 0) {
                        float *ml = a.sums + 2 * (int64_t)a.blocks * kRows * DP + (at * kRows + out_row) * 2;
                        ml[0] = mx;
                        ml[1] = lsum;
                    }
                }
            }
            __syncthreads();
        }
        p.rest += take;
        left -= take;
    }
}

// -------------------------------------------------------------------- wide ---

// A tile of 256 rows, 64 to a wave, by 64 keys a unit: the matrix products bound it.
// K and V go through LDS, two units of each; the next one's bytes are on their way in
// registers while this one is computed.  Their 16-byte pieces lie in an order that leaves
// no bank asked twice.  As above S^T = K Q^T, O^T = V^T P^T (V read from LDS by columns),
// so the weights stay in their lanes.  A wave has its matrix unit to itself, and 64 rows,
// since with 32 the reads of K and V from LDS take as long as the products.  So that the
// matrix unit does not wait for the softmax, a half unit (32 keys) is in three stages at
// once: the products of the next half's scores and of the last half's weights with V run
// beside this half's exponentials.
constexpr int kWideKeys = 64, kWideRows = 256;

template <int DP, bool kHalf>
__global__ void __launch_bounds__(kThreads, 1) k_attend_wide(Attend a) {
    constexpr int kPieces = DP / 8;            // 16-byte pieces of a key
    constexpr int kSteps = DP / 16;            // products over 16 dimensions
    constexpr int kCols = DP / 32;             // blocks of 32 output dimensions
    constexpr int kLoads = kPieces * kWideKeys / kThreads;
    constexpr uint32_t kUnit = kWideKeys * DP;
    __shared__ __align__(16) uint16_t bufs[4 * kUnit];  // two units of K, two of V
    uint16_t *const kbuf = bufs, *const vbuf = bufs + 2 * kUnit;
    const int lane = threadIdx.x % kWave, wave = uniform((int32_t)threadIdx.x / kWave);
    const int col = lane % 32, half = lane / 32;
    // blocks go to the eight dies in turn: neighbouring pieces, which share K and V, to one die
    const int64_t block = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    int64_t piece;
    Place p = find<kWideKeys>(a, block, &piece);
    if (p.row < 0) {
        if (threadIdx.x == 0) a.cuts[block].done = 0;
        return;
    }
    const int64_t whole_piece = min(piece, p.total - block * piece);
    int64_t left = whole_piece;
    const float c = a.scale * kLog2e;
    const int32_t place = (1 << a.shift) - 1;

    // where piece x of key k lies in its row of LDS
    auto k_at = [](uint32_t key, uint32_t x) { return x ^ (kPieces == 16 ? key & 15 : (key >> 1) & 7); };
    auto v_at = [](uint32_t key, uint32_t x) { return x ^ (kPieces == 16 ? 2 * (key & 7) : 2 * ((key >> 1) & 3)); };
    // this lane's reads: K rows as the first factor; V by columns: four keys of one dimension
    uint32_t k_read[kSteps], v_read[kCols];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) k_read[s] = col * DP + 8 * k_at(col, 2 * s + half);
    const uint32_t vk = 4 * half + (lane % 16) / 4;  // key of the lane's 8 bytes (+ 8, 16, 24)
#pragma unroll
    for (int d = 0; d < kCols; ++d) {
        const uint32_t dim = 32 * d + 16 * (lane / 16 % 2) + 4 * (lane % 4);
        v_read[d] = vk * DP + 8 * v_at(vk, dim / 8) + dim % 8;
    }

    while (left > 0) {
        const Row r = shared_row(a, p.row);
        const int64_t in_row = row_units<kWideKeys>(a, r) * a.kv_heads * a.parts;
        if (p.rest >= in_row) {
            ++p.row;
            p.rest = 0;
            continue;
        }
        const Tile t = tile_at<kWideKeys>(a, r, p.rest);
        const int64_t take = min(t.units - t.done, left);
        if (left == whole_piece) note(a, block, r, t, piece);
        const int32_t all = max(0, r.base + r.n);
        const int32_t most = max(0, min(r.base + t.first + t.n, all));
        u32x4 q[2][kSteps];
        int32_t seen[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int row = 64 * wave + 32 * b + col, tok = row / t.heads, h = row - tok * t.heads;
            const bool is = tok < t.n;
            seen[b] = is ? max(0, min(r.base + t.first + tok + 1, all)) : 0;
            const uint16_t *src = a.q + (int64_t)(r.first + t.first + tok) * a.q_token +
                                  (int64_t)(t.head * (a.heads / a.kv_heads) + t.part * a.group + h) * a.q_head;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int d = 16 * s + 8 * half;
                q[b][s] = is && d < a.dim ? *reinterpret_cast<const u32x4 *>(src + d) : u32x4{0, 0, 0, 0};
            }
        }
        // keys that every query of the wave's sees
        const int32_t least = (64 * wave + 63) / t.heads < t.n
                                  ? max(0, min(r.base + t.first + 64 * wave / t.heads + 1, all)) : 0;
        f32x16 o[2][kCols], sa[2], sb[2];
        u32x4 pa[2][2], pb[2][2];
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, top[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int d = 0; d < kCols; ++d) o[b][d] = f32x16{};
#pragma unroll
            for (int i = 0; i < 2; ++i) pa[b][i] = u32x4{0, 0, 0, 0};
        }
        global_u16 *kh = (global_u16 *)(a.k + (int64_t)t.head * a.head_stride);
        global_u16 *vh = (global_u16 *)(a.v + (int64_t)t.head * a.head_stride);
        const int32_t *pages = a.table + r.slot * a.table_stride;

        // A unit's keys, one per lane: its page, and where its vectors lie (-1: in no page).  Keys past
        // the last one that the tile sees stand for it.
        auto key_of = [&](int32_t unit) { return min(unit * kWideKeys + lane, most - 1); };
        auto page_of = [&](int32_t unit) { return pages[key_of(unit) >> a.shift]; };
        auto place_of = [&](int32_t unit, int32_t page) -> int64_t {
            return (uint32_t)page < (uint32_t)a.pages
                       ? (int64_t)page * a.page_stride + (int64_t)(key_of(unit) & place) * a.token_stride : -1;
        };
        u32x4 k_in[kLoads], v_in[kLoads];
        auto load_k = [&](int64_t where) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int at = i * kThreads + threadIdx.x, d = 8 * (at % kPieces);
                const int64_t off = __shfl(where, at / kPieces);
                k_in[i] = *(global_u32x4 *)(kh + max(off, (int64_t)0) + (d < a.dim ? d : 0));
            }
        };
        auto load_v = [&](int64_t where) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int at = i * kThreads + threadIdx.x, d = 8 * (at % kPieces);
                const int64_t off = __shfl(where, at / kPieces);
                v_in[i] = *(global_u32x4 *)(off < 0 ? zeros() : vh + off + (d < a.dim ? d : 0));
            }
        };
        auto store_k = [&](uint32_t buf) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t at = i * kThreads + threadIdx.x, key = at / kPieces;
                *reinterpret_cast<u32x4 *>(kbuf + buf + key * DP + 8 * k_at(key, at % kPieces)) = k_in[i];
            }
        };
        auto store_v = [&](uint32_t buf) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t at = i * kThreads + threadIdx.x, key = at / kPieces;
                *reinterpret_cast<u32x4 *>(vbuf + buf + key * DP + 8 * v_at(key, at % kPieces)) = v_in[i];
            }
        };
        auto read_k = [&](uint32_t at, int s) { return *reinterpret_cast<const u32x4 *>(kbuf + at + k_read[s]); };
        auto read_v = [&](uint32_t at, int d, int i) -> u32x4 {  // keys 16 i + 4 half + (0..3, 8..11)
            typedef __attribute__((address_space(3))) i16x4 lds;
            const uint16_t *from = vbuf + at + v_read[d] + 16 * i * DP;
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds *)from));
            const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds *)(from + 8 * DP)));
            return u32x4{x[0], x[1], y[0], y[1]};
        };
        auto highest = [&](const f32x16 &s) {
            float x = s[0];
#pragma unroll
            for (int i = 1; i < 15; i += 2) x = fmaxf(fmaxf(x, s[i]), s[i + 1]);
            x = fmaxf(x, s[15]);
            const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
            return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
        };
        auto scores = [&](uint32_t at, f32x16 (&s)[2]) {
            s[0] = s[1] = f32x16{};
#pragma unroll
            for (int d = 0; d < kSteps; ++d) {
                const u32x4 k = read_k(at, d);
                s[0] = mfma32<kHalf>(k, q[0][d], s[0]);
                s[1] = mfma32<kHalf>(k, q[1][d], s[1]);
            }
        };
        auto gather = [&](uint32_t at, const u32x4 (&w)[2][2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < kCols; ++d) {
                    const u32x4 v = read_v(at, d, i);
                    o[0][d] = mfma32<kHalf>(v, w[0][i], o[0][d]);
                    o[1][d] = mfma32<kHalf>(v, w[1][i], o[1][d]);
                }
        };
        // scores of the half unit at key k0: those not seen are -inf
        auto settle = [&](int32_t k0, uint32_t ok, f32x16 (&s)[2]) {
            if (k0 + 32 > least || ~ok) {
                asm volatile("");  // a branch, not selections in every turn
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int32_t rest = seen[b] - k0 - 4 * half;
                    const uint32_t have = ok >> 4 * half;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = 8 * (i / 4) + i % 4;
                        if (key >= rest || !(have >> key & 1)) s[b][i] = -INFINITY;
                    }
                    top[b] = highest(s[b]);
                }
            }
        };
        // m follows when it lags too far; the weights w, which are under the old one, go to O first
        auto follow = [&](uint32_t at, u32x4 (&w)[2][2]) {
            if (__any((top[0] - m[0]) * c > kLag || (top[1] - m[1]) * c > kLag)) {
                asm volatile("");
                gather(at, w);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const float now = fmaxf(m[b], top[b]);
                    const float keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[b] - now) * c);
                    m[b] = now;
                    l[b] *= keep;
#pragma unroll
                    for (int d = 0; d < kCols; ++d) o[b][d] *= keep;
                    w[b][0] = w[b][1] = u32x4{0, 0, 0, 0};
                }
            }
        };
        // One half unit: its weights from s into w, the next scores into s1, the last weights w0 into O.
        // A step is the two products with one fragment of K or V, the reads of a fragment further on, and
        // a share of the softmax; the compiler keeps to the steps' order, which feeds the matrix unit.
        auto stage = [&](const f32x16 (&s)[2], u32x4 (&w)[2][2], uint32_t k, f32x16 (&s1)[2], uint32_t v,
                         const u32x4 (&w0)[2][2]) {
            constexpr int kFrags = kSteps + 2 * kCols, kAhead = 2, kEach = 32 / kFrags;
            constexpr int kTop = (16 + kFrags - kSteps - 2) / (kFrags - kSteps - 1);  // scores looked at in a step
            const float mc[2] = {m[0] == -INFINITY ? 0.f : m[0] * c, m[1] == -INFINITY ? 0.f : m[1] * c};
            u32x4 frag[kAhead + 1];
            auto fetch = [&](int f) {
                frag[f % (kAhead + 1)] = f < kSteps ? read_k(k, f) : read_v(v, (f - kSteps) % kCols, (f - kSteps) / kCols);
            };
            auto multiply = [&](int f, int b) {
                const u32x4 x = frag[f % (kAhead + 1)];
                if (f < kSteps) {
                    s1[b] = mfma32<kHalf>(x, q[b][f], f == 0 ? f32x16{} : s1[b]);
                } else {
                    const int d = (f - kSteps) % kCols, i = (f - kSteps) / kCols;
                    o[b][d] = mfma32<kHalf>(x, w0[b][i], o[b][d]);
                }
            };
            float odd;
            auto weigh = [&](int e) {  // element e of the half unit's weights; two are packed together
                const int b = e / 16, i = e % 16;
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -mc[b]));
                l[b] += x;
                if (i % 2 == 0) odd = x;
                else {
                    uint32_t y = pack<kHalf>(odd, x);
                    asm volatile("" : "+v"(y));  // here, not where it is first used
                    w[b][i / 8][i % 8 / 2] = y;
                }
            };
#pragma unroll
            for (int f = 0; f < kAhead; ++f) fetch(f);
#pragma unroll
            for (int f = 0; f < kFrags; ++f) {
                if (f + kAhead < kFrags) fetch(f + kAhead);
#pragma unroll
                for (int e = 0; e < kEach / 2; ++e) weigh(kEach * f + e);
                multiply(f, 0);
#pragma unroll
                for (int e = kEach / 2; e < kEach; ++e) weigh(kEach * f + e);
                multiply(f, 1);
                if (f > kSteps) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int i = kTop * (f - kSteps - 1); i < min(16, kTop * (f - kSteps)); ++i)
                            top[b] = i ? fmaxf(top[b], s1[b][i]) : s1[b][0];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(top[b]), __float_as_uint(top[b]), false, false);
                top[b] = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
            }
        };

        const int32_t u0 = (int32_t)t.done, u1 = (int32_t)(u0 + take);
        if (u0 * kWideKeys < most) {
            int32_t page0 = page_of(u0), page1 = page_of(u0 + 1), page2 = page_of(u0 + 2);
            int64_t where = place_of(u0, page0);
            uint64_t ok = __ballot(where >= 0);  // keys of unit u, of the one after it, that lie in a page
            load_k(where);
            load_v(where);
            int64_t v_where = place_of(u0 + 1, page1);
            uint64_t ok1 = __ballot(v_where >= 0);
            __syncthreads();  // the last tile is done with the buffers
            store_k(0);
            store_v(0);
            load_k(v_where);
            // the half unit before the first has weights of zero and a V of zeros
#pragma unroll
            for (int i = 0; i < 32 * DP / 8 / kThreads; ++i)
                *reinterpret_cast<u32x4 *>(vbuf + kUnit + 32 * DP + 8 * (i * kThreads + threadIdx.x)) = u32x4{0, 0, 0, 0};
            store_k(kUnit);
            __syncthreads();
            scores(0, sa);
#pragma unroll
            for (int b = 0; b < 2; ++b) top[b] = highest(sa[b]);
            settle(u0 * kWideKeys, (uint32_t)ok, sa);
            m[0] = top[0];
            m[1] = top[1];
            uint32_t x = 0;  // of unit u's buffers
            for (int32_t u = u0; u < u1; ++u) {
                const uint32_t y = kUnit - x;
                const int64_t k_where = place_of(u + 2, page2);
                load_k(k_where);
                load_v(v_where);
                page2 = page_of(u + 3);
                stage(sa, pb, x + 32 * DP, sb, y + 32 * DP, pa);
                settle(u * kWideKeys + 32, (uint32_t)(ok >> 32), sb);
                __syncthreads();  // the next unit's K and this one's V are there, the buffers behind them free
                follow(x, pb);
                v_where = k_where;
                ok = ok1;
                ok1 = __ballot(k_where >= 0);
                stage(sb, pa, y, sa, x, pb);
                settle(u * kWideKeys + 64, (uint32_t)ok, sa);
                if (u + 1 < u1) follow(x + 32 * DP, pa);
                store_k(x);  // unit u + 2
                store_v(y);  // unit u + 1
                x = y;
            }
            gather(kUnit - x + 32 * DP, pa);
        }
        // o[b][d][i] is dimension 32 d + 8 (i / 4) + 4 half + i % 4 of query `col`
        const bool whole = take == t.units;
        const int64_t at = 2 * block + (t.done == 0);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[b]), __float_as_uint(l[b]), false, false);
            const float sum = __uint_as_float(y[0]) + __uint_as_float(y[1]);
            const int row = 64 * wave + 32 * b + col, tok = row / t.heads, h = row - tok * t.heads;
            if (tok >= t.n) continue;
            if (whole) {
                const float inv = sum > 0.f ? 1.f / sum : 0.f;
                const int64_t token = r.first + t.first + tok, head = t.head * (a.heads / a.kv_heads) + t.part * a.group + h;
                uint16_t *dst = a.out + token * a.out_token + head * a.out_head;
#pragma unroll
                for (int d = 0; d < kCols; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int dim = 32 * d + 2 * i + 4 * half;
                        if (dim < a.dim)
                            *reinterpret_cast<u32x2 *>(dst + dim) =
                                u32x2{pack<kHalf>(o[b][d][i] * inv, o[b][d][i + 1] * inv),
                                      pack<kHalf>(o[b][d][i + 2] * inv, o[b][d][i + 3] * inv)};
                    }
                if (a.lse && half == 0)
                    a.lse[token * a.heads + head] = sum > 0.f ? m[b] * a.scale + logf(sum) : -INFINITY;
            } else {
                float *dst = a.sums + (at * kWideRows + row) * DP;
#pragma unroll
                for (int d = 0; d < kCols; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *reinterpret_cast<f32x4 *>(dst + 32 * d + 2 * i + 4 * half) =
                            f32x4{o[b][d][i], o[b][d][i + 1], o[b][d][i + 2], o[b][d][i + 3]};
                if (half == 0) {
                    float *ml = a.sums + 2 * (int64_t)a.blocks * kWideRows * DP + (at * kWideRows + row) * 2;
                    ml[0] = m[b];
                    ml[1] = sum;
                }
            }
        }
        p.rest += take;
        left -= take;
    }
}

// ---------------------------------------------------------------------- join ---

// Partial sums of the tiles that a cut goes through.  blockIdx.x is the cut after
// block x, and works on the tile it is the first cut of; blockIdx.y takes kJoin rows of it.
// A group of threads takes a row; where the tile is in many pieces, all groups share a
// row's pieces and their sums meet in LDS.  The partial sums' bytes bound it.
template <int DP, int kRows, int kJoin, bool kHalf>
__global__ void __launch_bounds__(kThreads) k_join(Attend a) {
    constexpr int kLanes = DP / 4, kGroups = kThreads / kLanes;
    __shared__ float part[kGroups][DP];
    __shared__ float part_l[kGroups];
    const int64_t cut = blockIdx.x + 1;
    const Cut t = a.cuts[cut];
    if (t.done == 0 || t.done > t.piece) return;  // between two tiles, or not the tile's first cut
    const int row0 = blockIdx.y * kJoin, row1 = min(row0 + kJoin, t.n * t.heads);
    if (row0 >= row1) return;
    const int64_t last = cut + (t.units - t.done - 1) / t.piece;  // the block with the tile's end
    const float c = a.scale * kLog2e;
    const float *ml = a.sums + 2 * (int64_t)a.blocks * kRows * DP;
    const int lane = threadIdx.x % kLanes, g = threadIdx.x / kLanes;
    // the first piece begins the tile, the others go on with it
    auto slot_of = [&](int64_t i) { return i < cut ? 2 * i + 1 : 2 * i; };
    auto write = [&](int row, f32x4 x, float l, float mx) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const int tok = row / t.heads, h = row - tok * t.heads;
        const int64_t token = t.token + tok, head = t.head + h;
        if (4 * lane < a.dim)
            *reinterpret_cast<u32x2 *>(a.out + token * a.out_token + head * a.out_head + 4 * lane) =
                u32x2{pack<kHalf>(x[0] * inv, x[1] * inv), pack<kHalf>(x[2] * inv, x[3] * inv)};
        if (a.lse && lane == 0) a.lse[token * a.heads + head] = l > 0.f ? mx * a.scale + logf(l) : -INFINITY;
    };
    if (last - cut < 4) {
        for (int row = row0 + g; row < row1; row += kGroups) {
            float mx = -INFINITY;
            for (int64_t i = cut - 1; i <= last; ++i) mx = fmaxf(mx, ml[(slot_of(i) * kRows + row) * 2]);
            f32x4 sum{0, 0, 0, 0};
            float l = 0.f;
            for (int64_t i = cut - 1; i <= last; ++i) {
                const int64_t at = slot_of(i) * kRows + row;
                const float mi = ml[at * 2];
                const float keep = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mi - mx) * c);
                sum += *reinterpret_cast<const f32x4 *>(a.sums + at * DP + 4 * lane) * keep;
                l += ml[at * 2 + 1] * keep;
            }
            write(row, sum, l, mx);
        }
        return;
    }
    for (int row = row0; row < row1; ++row) {
        float mx = -INFINITY;
        for (int64_t i = cut - 1 + threadIdx.x % kWave; i <= last; i += kWave) mx = fmaxf(mx, ml[(slot_of(i) * kRows + row) * 2]);
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
        f32x4 sum{0, 0, 0, 0};
        float l = 0.f;
#pragma unroll 4
        for (int64_t i = cut - 1 + g; i <= last; i += kGroups) {
            const int64_t at = slot_of(i) * kRows + row;
            const float mi = ml[at * 2], li = ml[at * 2 + 1];
            const f32x4 x = *reinterpret_cast<const f32x4 *>(a.sums + at * DP + 4 * lane);
            const float keep = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mi - mx) * c);
            sum += x * keep;
            l += li * keep;
        }
        __syncthreads();
        *reinterpret_cast<f32x4 *>(&part[g][4 * lane]) = sum;
        if (lane == 0) part_l[g] = l;
        __syncthreads();
        if (threadIdx.x < kLanes) {
            f32x4 x{0, 0, 0, 0};
            float y = 0.f;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                x += *reinterpret_cast<const f32x4 *>(&part[i][4 * lane]);
                y += part_l[i];
            }
            write(row, x, y, mx);
        }
    }
}

// -------------------------------------------------------------------- launch ---

struct Shape {
    int blocks, row_waves;  // of k_attend_narrow; 256 rows are k_attend_wide's
    int grid;
    int rows() const { return 16 * blocks * row_waves; }
};

Shape shape_of(const tam_chunk &c, int64_t heads) {
    const int64_t longest = c.longest ? std::min(c.longest, c.tokens) : c.tokens;
    const int64_t rows = longest * (heads / c.kv_heads);
    if (rows <= 16) return Shape{1, 1, 512};
    if (rows <= 32) return Shape{2, 1, 256};
    if (rows <= 64) return Shape{2, 2, 256};
    if (rows <= 128) return Shape{2, 4, 256};
    return Shape{4, 4, 256};
}

int padded(int64_t dim) { return dim <= 64 ? 64 : 128; }

template <int DP, int kBlocks, int kRowWaves, bool kHalf>
hipError_t launch_narrow(const Attend &a, hipStream_t s) {
    constexpr int kRows = 16 * kBlocks * kRowWaves, kJoin = 4;
    hipLaunchKernelGGL((k_attend_narrow<DP, kBlocks, kRowWaves, kHalf>), dim3((unsigned)a.blocks), dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_join<DP, kRows, kJoin, kHalf>), dim3((unsigned)a.blocks - 1, (unsigned)(kRows / kJoin)),
                       dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <int DP, bool kHalf>
hipError_t launch(const Attend &a, const Shape &sh, hipStream_t s) {
    if (sh.rows() == 16) return launch_narrow<DP, 1, 1, kHalf>(a, s);
    if (sh.rows() == 32) return launch_narrow<DP, 2, 1, kHalf>(a, s);
    if (sh.rows() == 64) return launch_narrow<DP, 2, 2, kHalf>(a, s);
    if (sh.rows() == 128) return launch_narrow<DP, 2, 4, kHalf>(a, s);
    hipLaunchKernelGGL((k_attend_wide<DP, kHalf>), dim3((unsigned)a.blocks), dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_join<DP, kWideRows, 32, kHalf>), dim3((unsigned)a.blocks - 1, kWideRows / 32),
                       dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int64_t attend_work_bytes(const tam_chunk &c, int64_t heads) {
    const Shape sh = shape_of(c, heads);
    return 2 * (int64_t)sh.grid * sh.rows() * (padded(c.head_dim) + 2) * 4 + sh.grid * (int64_t)sizeof(Cut);
}

hipError_t launch_attend(const tam_chunk &c, const Queries &q, void *work, hipStream_t s) {
    const Shape sh = shape_of(c, q.heads);
    const int64_t group = q.heads / c.kv_heads;
    Attend a{static_cast<const uint16_t *>(c.k), static_cast<const uint16_t *>(c.v),
             static_cast<const uint16_t *>(q.q), static_cast<uint16_t *>(q.out), q.lse, c.page_stride,
             c.head_stride, c.token_stride, q.q_token, q.q_head, q.out_token, q.out_head, c.table, c.length,
             c.offsets, c.slot_ids, c.table_stride, c.slots, c.max_pages, c.rows, c.tokens, (int32_t)c.num_pages,
             __builtin_ctzll((unsigned long long)c.page_tokens), (int32_t)q.heads, (int32_t)c.kv_heads,
             (int32_t)c.head_dim, q.scale, 0, 0, 0, 0, 0, nullptr, nullptr};
    a.group = (int32_t)std::min<int64_t>(group, sh.rows());
    a.parts = (int32_t)((group + a.group - 1) / a.group);
    a.tq = sh.rows() / a.group;
    a.blocks = sh.grid;
    a.least = 1;
    a.sums = static_cast<float *>(work);
    a.cuts = reinterpret_cast<Cut *>(a.sums + 2 * (int64_t)sh.grid * sh.rows() * (padded(c.head_dim) + 2));
    const bool half = c.dtype == TAM_DTYPE_FP16;
    if (padded(c.head_dim) == 64) return half ? launch<64, true>(a, sh, s) : launch<64, false>(a, sh, s);
    return half ? launch<128, true>(a, sh, s) : launch<128, false>(a, sh, s);
}

}  // namespace tam
