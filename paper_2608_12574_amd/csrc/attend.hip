// Attention of a chunk of new tokens per sequence over a paged K/V cache.
//
// Mathematics.  For a query q, o = sum_j w_j v_j / sum_j w_j with w_j = exp(scale (q k_j - m)),
// for any m; in one pass over the keys m is the running maximum, and what was summed
// under an older m is scaled when m grows.  Parts of the keys summed apart join the
// same way.  m is let lag by up to 2^8 in w before it is moved (Range), which the fp32
// sums and the 16-bit weights hold, so that the sums are scaled a few times per row and
// not in each step.
//
// Scores, maxima, sums and lse are fp32.  The weights are rounded to K and V's type, since 16-bit matrix
// instructions multiply them with V; the sum of weights is that of the unrounded ones.  Against 64 bits the outputs' error is 1.2 to
// 1.4 times that of fp32 weights and the same output type (bf16 0.0023 and 0.0017 of the output's size, fp16 0.00029 and 0.00021).
//
// A tile is `tq` tokens of one row, times the heads that share a K/V head (their
// rows of a product are side by side, so K and V are read once for all of them).
// A unit is a tile's product with kKeys keys.  The keys that the tiles of a call see, row
// after row, head after head, tile after tile, are one line, cut into equal pieces for as
// many blocks as the chip holds: any mix of long and short rows and chunks fills
// it evenly.  A tile begins with `extra` keys that stand for its own cost (queries, first
// reads, output).  A cut inside a tile moves back to the unit it falls in; the tile's parts
// leave partial sums in the scratch, which k_join adds up.  The lengths lie on the
// device: each block finds its piece from them by a prefix sum over the rows.
//
// With a mask among the row's new tokens (kSeen; trees of drafted tokens) a token sees all that lies before the row's first one and
// those of its tokens whose bits are set.  The bits are looked at in the units at the row's end alone, 32 keys of a token at a time.
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

// Memory's addresses, told from LDS's, so that a load does not wait as if it could be of either.
typedef __attribute__((address_space(1))) const uint8_t global_u8;
typedef __attribute__((address_space(1))) const u32x4 global_u32x4;
typedef __attribute__((address_space(1))) const u32x2 global_u32x2;

struct Attend {
    const uint16_t *k, *v, *q;
    uint16_t *out;
    float *lse;
    int64_t page_stride, head_stride, token_stride, q_token, q_head, out_token, out_head;
    const int32_t *table, *length, *offsets, *slot_ids;
    int64_t table_stride, slots, max_pages, rows, tokens;
    int32_t pages, shift, heads, kv_heads, per_kv, dim;  // per_kv: query heads to a K/V head
    float scale;
    // the cut: tiles of `tq` tokens by `group` heads, `parts` of them per K/V head
    int32_t tq, group, parts, blocks;
    int32_t unit, extra;  // keys of a unit, a power of two; keys that stand for a tile's own cost
    float *sums;    // [2 blocks][tile rows][DP] partial sums, then [2 blocks][tile rows][2] their m and sum of weights
    struct Cut *cuts;  // [blocks] what each block's piece begins with
    // kSeen: which of the row's tokens each one sees
    const uint64_t *seen;
    int64_t seen_stride, seen_words;
};

// The tile in whose middle a block's piece begins.
struct alignas(16) Cut {
    int32_t is;       // a tile is cut here, behind its first unit
    int32_t back, more;  // the cuts of the tile before this one, and after it
    int32_t token, n, head, heads;  // the tile's first token and query head, and how many
};

// a value that is the same in all lanes, to the compiler too
__device__ inline int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
    return (int64_t)(uint32_t)uniform((int32_t)x) | (int64_t)uniform((int32_t)(x >> 32)) << 32;
}

// x, of which the compiler knows nothing from here on: what is computed from it is computed where it is used. Else all that
// does not change from tile to tile is computed before the first one, and waits in registers (one request's 16 tokens over 700, 32/8
// heads of 128: 10.1 us with it and 10.9 without, medians of eight; four of up to 250 over 116,700, 16/2 heads of 64: 91.5 and 91.0).
__device__ inline int32_t here(int32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}

// ------------------------------------------------------------------ the cut ---

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

// a row that is the same in all lanes, to the compiler too
__device__ inline Row uniform(Row r) {
    r.n = uniform(r.n);
    r.base = uniform(r.base);
    r.first = uniform(r.first);
    r.slot = uniform(r.slot);
    return r;
}

// In what follows, kSeen: a token sees what lies before its row's tokens, and those of them that its bits name, so that all tiles
// of a row go through all of its keys.

// Keys on the line before tile t of a row and head: tile i < t sees base + (i + 1) tq, or all.
template <bool kSeen>
__device__ inline int64_t keys_before(const Attend &a, const Row &r, int64_t t) {
    if constexpr (kSeen) return t * ((int64_t)max(r.base, 0) + r.n + a.extra);
    return t * (max(r.base, 0) + a.extra) + a.tq * (t * (t + 1) / 2);
}

// Keys on the line of a row and head.  A row of one tile takes whole units, so that a
// batch of them is cut between units.
template <bool kSeen>
__device__ inline int64_t row_keys(const Attend &a, const Row &r) {
    const int64_t all = (int64_t)max(r.base, 0) + r.n + a.extra;
    if (r.n <= a.tq) return r.n ? (all + a.unit - 1) & -(int64_t)a.unit : 0;
    return keys_before<kSeen>(a, r, (r.n - 1) / a.tq) + all;
}

// A place on the line.
struct Place {
    int64_t row, total;   // the row; keys on the whole line
    int64_t rest;         // keys of the row before this place
    Row r;                // what the row is
};

// Where piece number `share` (this block's) begins, and the keys of a piece.  All threads of
// the block call it; row < 0 past the line's end.
template <bool kSeen, int kBlock = kThreads>
__device__ inline Place find(const Attend &a, int64_t share, int64_t *piece) {
    __shared__ int64_t sums[kBlock / kWave];
    __shared__ int64_t found[2];
    __shared__ Row found_row;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t per = (a.rows + kBlock - 1) / kBlock, lo = threadIdx.x * per, hi = min(lo + per, a.rows);
    const int64_t heads = (int64_t)a.kv_heads * a.parts;
    int64_t mine = 0;
    Row r{};
    for (int64_t i = lo; i < hi; ++i) {
        r = row_at(a, i);
        mine += heads * row_keys<kSeen>(a, r);
    }
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
    for (int w = 0; w < kBlock / kWave; ++w) {
        if (w < wave) upto += sums[w];
        p.total += sums[w];
    }
    p.total = uniform(p.total);
    const int shift = __builtin_ctz((uint32_t)a.blocks * (uint32_t)a.unit);  // (both are powers of two)
    *piece = max((int64_t)1, (p.total + (1ll << shift) - 1) >> shift) * a.unit;
    const int64_t at = share * *piece;
    if (at >= upto - mine && at < upto) {  // one thread: walk its rows
        int64_t rest = at - (upto - mine);
        int64_t i = lo;
        if (per > 1) {
            for (; i < hi; ++i) {
                r = row_at(a, i);
                const int64_t u = heads * row_keys<kSeen>(a, r);
                if (rest < u) break;
                rest -= u;
            }
        }
        found[0] = i;
        found[1] = rest;
        found_row = r;
    }
    __syncthreads();
    p.row = uniform(found[0]);
    p.rest = uniform(found[1]);
    p.r = uniform(found_row);
    return p;
}

// A tile, and the place in it.
struct Tile {
    int32_t head, part, tile;     // K/V head and part of its group; number in the row
    int32_t first, n;             // its first token in the chunk, and its tokens
    int32_t heads;                // query heads of the part
    int64_t rest, keys;           // keys of it on the line before the place, and all of them
};

template <bool kSeen>
__device__ inline Tile tile_at(const Attend &a, const Row &r, int64_t rest) {
    const int64_t u = row_keys<kSeen>(a, r);
    const int32_t vh = (int32_t)(rest / u);
    rest -= vh * u;
    int32_t lo = 0, hi = (r.n + a.tq - 1) / a.tq;  // keys_before(lo) <= rest < keys_before(hi)
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (keys_before<kSeen>(a, r, mid) <= rest) lo = mid;
        else hi = mid;
    }
    Tile t;
    t.head = vh / a.parts;
    t.part = vh - t.head * a.parts;
    t.tile = lo;
    t.first = lo * a.tq;
    t.n = min(a.tq, r.n - t.first);
    t.heads = min(a.group, a.per_kv - t.part * a.group);
    t.rest = rest - keys_before<kSeen>(a, r, lo);
    t.keys = r.n <= a.tq ? u : (int64_t)max(r.base, 0) + (kSeen ? r.n : t.first + t.n) + a.extra;
    return t;
}

// The units of a tile that are a block's: from .. to of all.
struct Share {
    int32_t from, to, all;
};

template <int kKeys>
__device__ inline Share share_of(const Attend &a, const Tile &t, int64_t left) {
    auto unit = [&](int64_t at) { return (int32_t)(max(at - a.extra, (int64_t)0) / kKeys); };
    Share s;
    s.all = unit(t.keys + kKeys - 1);
    s.from = unit(t.rest);
    s.to = left >= t.keys - t.rest ? s.all : unit(t.rest + left);
    return s;
}

// What the block's piece begins with, for k_join.
template <int kKeys>
__device__ inline void note(const Attend &a, int64_t block, const Row &r, const Tile &t, int64_t piece) {
    if (threadIdx.x != 0) return;
    // (a tile has fewer than 2^31 keys)
    const uint32_t keys = (uint32_t)min(piece, (int64_t)INT32_MAX), rest = (uint32_t)(t.keys - t.rest - 1);
    const int32_t behind = (int32_t)(t.rest - a.extra - kKeys);
    a.cuts[block] = Cut{behind >= 0, behind >= 0 ? (int32_t)((uint32_t)behind / keys) : 0, (int32_t)(rest / keys),
                        r.first + t.first, t.n, t.head * a.per_kv + t.part * a.group, t.heads};
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

// Where the weights lie, in powers of two: m is put kRaise under the highest score, and may lag until a
// weight passes 2^kMost.  bf16 has fp32's range.  In fp16 what lies under 2^-24 is lost, and a long row of small
// weights with it, so the highest weight is kept as high as the type allows, 2^7 to 2^15.
template <bool kHalf>
struct Range {
    static constexpr float kRaise = kHalf ? 7.f : 0.f, kMost = kRaise + 8.f;
    // where m goes for a highest score x
    static __device__ float follow(float m, float x, float c) {
        return fmaxf(m, kHalf ? x - fminf(kRaise / c, 1e38f) : x);  // (a tiny scale: no infinite step)
    }
};

// In both kernels below, kRuns: 16 keys from a multiple of 16 lie side by side in one page (pages of 16
// tokens or more, strides of 32 bits), so that its number and where they begin are the same for all lanes.

// Where place `in` of a page (kRuns: its run of 16) begins, in bytes.
template <bool kRuns>
__device__ inline uint64_t place_in(const Attend &a, uint32_t page, uint32_t in) {
    if constexpr (kRuns)
        return (uint64_t)page * (uint32_t)(2 * a.page_stride) + (in & ~15u) * (uint32_t)(2 * a.token_stride);
    else
        return (uint64_t)page * (uint64_t)(2 * a.page_stride) + in * (uint64_t)(2 * a.token_stride);
}

// V of a key that some of a tile's queries see and others do not must be finite in the products, where what a query does not see
// has the weight 0.  So what is not finite there becomes 0 (`only_finite`), and is added to the queries that see it
// when the tile's sums are done (`not_finite`); a tile looks at its last tokens' keys for such, and hardly ever finds one.

// Bits 15 and 31 of it, over all words of `of`: some half is not finite.
template <bool kHalf>
__device__ inline uint32_t exponents(uint32_t of, uint32_t before) {
    constexpr uint32_t kAll = kHalf ? 0x7C007C00u : 0x7F807F80u, kOne = kHalf ? 0x04000400u : 0x00800080u;
    return before | ((of & kAll) + kOne);
}

template <bool kHalf>
__device__ inline uint32_t only_finite(uint32_t x) {
    constexpr uint32_t kAll = kHalf ? 0x7C00u : 0x7F80u;
    if ((x & kAll) == kAll) x &= 0xFFFF0000u;
    if ((x >> 16 & kAll) == kAll) x &= 0xFFFFu;
    return x;
}

template <bool kHalf>
__device__ inline float to_float(uint16_t x) {
    if constexpr (kHalf) return (float)__builtin_bit_cast(_Float16, x);
    else return __uint_as_float((uint32_t)x << 16);
}

// x if that is not finite, else 0
template <bool kHalf>
__device__ inline float not_finite(uint16_t x) {
    constexpr uint32_t kAll = kHalf ? 0x7C00u : 0x7F80u;
    return (x & kAll) == kAll ? to_float<kHalf>(x) : 0.f;
}

// kSeen: bit i says whether a token (of the call's) sees key k0 + i of its sequence; 32 keys, of which those past the row's
// tokens are not seen.
__device__ inline uint32_t seen_of(const Attend &a, const Row &r, int64_t token, int32_t k0) {
    const int32_t at = k0 - r.base, end = r.n - at;  // k0 among the row's tokens; bits from `end` on are past them
    if (at <= -32) return 0xFFFFFFFFu;
    if (end <= 0) return 0;
    const uint64_t *const row = a.seen + token * a.seen_stride;
    const int32_t w = max(at, 0) >> 6, in = max(at, 0) & 63;
    uint64_t x = w < a.seen_words ? row[w] >> in : 0;
    if (in > 32 && w + 1 < a.seen_words) x |= row[w + 1] << (64 - in);
    uint32_t y = (uint32_t)x;
    if (at < 0) y = y << -at | ((1u << -at) - 1);
    return end < 32 ? y & ((1u << end) - 1) : y;
}

// V of a key, of a head of which `v` is the first element, or null where the key lies in no page.
__device__ inline const uint16_t *v_of(const Attend &a, const uint16_t *v, const int32_t *pages, int32_t key) {
    const int32_t id = pages[(uint32_t)key >> a.shift];
    if ((uint32_t)id >= (uint32_t)a.pages) return nullptr;
    return v + id * a.page_stride + (key & ((1 << a.shift) - 1)) * a.token_stride;
}

// What lane `of` holds of x, for all lanes.
__device__ inline uint64_t lane_of(uint64_t x, int of) {
    return (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, of) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), of) << 32;
}

// A tile of at most 16 rows by all its keys, 32 keys per wave and step.  The bytes of
// K and V bound it, so the fragments come straight from memory into registers, the next
// step's while this one is computed, and LDS only joins the waves' sums at the end.
// S^T = K Q^T leaves each lane the weights of one query, for the same eight keys that it
// then holds as the second factor of O^T = V^T P^T: no weight changes lanes.  V's columns
// are paired in registers (v_perm).  64 rows of up to 8,192 tokens, 8 K/V heads of 128: 225 us,
// 5.7 TB/s of K and V.  One row of 700 tokens: 7 to 8 us, of which 2 find the cut and 3 more pass
// until the first keys are there.
constexpr int kNarrowKeys = 128;

template <int DP, bool kHalf, bool kRuns, bool kSeen>
__global__ void __launch_bounds__(kThreads, 2) k_attend_narrow(Attend a) {
    constexpr int kKeys = kNarrowKeys;
    constexpr int kSteps = DP / 32;  // products of 32 dimensions
    constexpr int kCols = DP / 16;   // dimensions per lane of 16: adjacent ones
    constexpr int kRows = 16;
    __shared__ float joint[4][16][DP + 4];
    __shared__ float tops[4][16], weights[4][16];
    __shared__ int32_t odd[4];  // the wave has put zeros in the place of values that are not finite
    const int lane = threadIdx.x % kWave, wave = uniform((int32_t)threadIdx.x / kWave);
    const int col = lane % 16, grp = lane / 16;
    const uint32_t place = (1u << a.shift) - 1;
    // where a lane's parts of K and V lie in their vectors, in bytes (kRuns: from their run's first); lanes past the
    // last dimension read others of the vector
    uint32_t k_in[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
        k_in[s] = 2 * ((32 * s + 8 * grp < a.dim ? 32 * s + 8 * grp : 0) + (kRuns ? (uint32_t)col * (uint32_t)a.token_stride : 0));
    const uint32_t v_in = 2 * ((kCols * col < a.dim ? kCols * col : 0) + (kRuns ? (uint32_t)(4 * grp) * (uint32_t)a.token_stride : 0));
    int64_t piece;
    Place p = find<kSeen>(a, blockIdx.x, &piece);
    if (p.row < 0) {
        if (threadIdx.x == 0) a.cuts[blockIdx.x].is = 0;
        return;
    }
    const int64_t from = blockIdx.x * piece;
    const int64_t whole_piece = min(piece, p.total - from);
    int64_t left = whole_piece;
    const float c = a.scale * kLog2e;
    while (left > 0) {
        const Row r = p.r;
        if (p.rest >= row_keys<kSeen>(a, r) * a.kv_heads * a.parts) {
            p.r = uniform(row_at(a, ++p.row));
            p.rest = 0;
            continue;
        }
        const Tile t = tile_at<kSeen>(a, r, p.rest);
        const Share share = share_of<kKeys>(a, t, left);
        if (left == whole_piece) note<kKeys>(a, blockIdx.x, r, t, piece);
        p.rest += t.keys - t.rest;
        left -= t.keys - t.rest;
        if (share.from == share.to) continue;  // (the piece ends before the next unit)
        // queries, one per lane of 16; rows past the tile's see no key.  Lanes past the last
        // dimension read others of the vector (queries: zero).
        u32x4 q[kSteps];
        const int32_t all = max(0, r.base + r.n);  // tokens of the sequence, chunk included
        const int32_t most = kSeen ? all : max(0, min(r.base + t.first + t.n, all));
        const int32_t least = max(0, min(kSeen ? r.base : r.base + t.first + 1, all));
        const int row = col, tok = row / t.heads, h = row - tok * t.heads;
        const bool is = tok < t.n;
        const int32_t seen = !is ? 0 : kSeen ? all : max(0, min(r.base + t.first + tok + 1, all));  // keys that the query sees
        const uint16_t *src = a.q + (int64_t)(r.first + t.first + tok) * a.q_token +
                              (int64_t)(t.head * a.per_kv + t.part * a.group + h) * a.q_head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 32 * s + 8 * grp;
            q[s] = is && d < a.dim ? *reinterpret_cast<const u32x4 *>(src + d) : u32x4{0, 0, 0, 0};
        }
        f32x4 o[kCols];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int j = 0; j < kCols; ++j) o[j] = f32x4{0, 0, 0, 0};
        global_u8 *const kh = (global_u8 *)(a.k + (int64_t)t.head * a.head_stride);
        global_u8 *const vh = (global_u8 *)(a.v + (int64_t)t.head * a.head_stride);
        const int32_t *const pages = a.table + r.slot * a.table_stride;
        int32_t clear = least;  // keys that need no look at the mask; 0 once a page number is bad
        int32_t zeros = 0;

        // A step's keys, one per lane of 32; those past the last one that the tile sees stand for it.  `id`:
        // the pages they lie in.
        auto key_of = [&](int32_t k0) { return min(k0 + lane % 32, most - 1); };
        auto page_of = [&](int32_t k0) { return pages[(uint32_t)key_of(k0) >> a.shift]; };
        auto place_of = [&](int32_t k0, int32_t id) -> uint64_t {
            const bool ok = (uint32_t)id < (uint32_t)a.pages;
            if (!__all(ok)) clear = 0;
            const uint32_t in = (uint32_t)key_of(k0) & place;
            return place_in<kRuns>(a, ok ? id : 0, in);
        };
        struct Step {
            u32x4 k[2][kSteps];
            u32x4 v[8];  // kCols * 2 bytes of each are used
        };
        // the fragments: K of key 16 i + col; V of the keys 16 i + 4 grp + (0..3)
        auto load = [&](uint64_t at, Step &x) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint64_t begin = kRuns ? lane_of(at, 16 * i) : __shfl(at, 16 * i + col);
#pragma unroll
                for (int s = 0; s < kSteps; ++s) x.k[i][s] = *(global_u32x4 *)(kh + begin + k_in[s]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint64_t begin = kRuns ? lane_of(at, 16 * (j / 4)) + (uint32_t)(j % 4) * (uint32_t)(2 * a.token_stride)
                                             : __shfl(at, 16 * (j / 4) + 4 * grp + j % 4);
                global_u8 *src = vh + begin + v_in;
                if constexpr (kCols == 8) {
                    x.v[j] = *(global_u32x4 *)src;
                } else {
                    const u32x2 y = *(global_u32x2 *)src;
                    x.v[j] = u32x4{y[0], y[1], 0, 0};
                }
            }
        };
        auto compute = [&](int32_t k0, int32_t id, Step &x) {
            uint32_t have = 0xFFFFFFFFu;  // keys of the step that lie in a page
            if (__builtin_expect(k0 + 32 > clear, 0)) {
                asm volatile("");
                have = (uint32_t)__ballot((uint32_t)id < (uint32_t)a.pages);
                // V of keys that no query sees or that lie in no page: zeros (their weights are zero, and
                // what lies there may be anything)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = 16 * (j / 4) + 4 * grp + j % 4;
                    if (k0 + key >= most || !(have >> key & 1)) x.v[j] = u32x4{0, 0, 0, 0};
                }
                if (least < most) {
                    uint32_t top = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int i = 0; i < kCols / 2; ++i) top = exponents<kHalf>(x.v[j][i], top);
                    if (__any((top & 0x80008000u) != 0)) {
                        zeros = 1;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (k0 + 16 * (j / 4) + 4 * grp + j % 4 >= least)
#pragma unroll
                                for (int i = 0; i < kCols / 2; ++i) x.v[j][i] = only_finite<kHalf>(x.v[j][i]);
                    }
                }
            }
            if (__builtin_expect(a.dim < DP, 0)) {  // K past the last dimension: the queries' zeros there would make an infinity NaN
                asm volatile("");
#pragma unroll
                for (int d = 0; d < kSteps; ++d)
                    if (32 * d + 8 * grp >= a.dim) x.k[0][d] = x.k[1][d] = u32x4{0, 0, 0, 0};
            }
            f32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < kSteps; ++d) s[i] = mfma16<kHalf>(x.k[i][d], q[d], s[i]);
            if (__builtin_expect(k0 + 32 > clear, 0)) {
                asm volatile("");
                if constexpr (kSeen) have &= is ? seen_of(a, r, r.first + t.first + tok, k0) : 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = 16 * (j / 4) + 4 * grp + j % 4;
                    if (k0 + key >= seen || !(have >> key & 1)) s[j / 4][j % 4] = -INFINITY;
                }
            }
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, s[j / 4][j % 4]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__any((top - m) * c > Range<kHalf>::kMost)) {  // NaN (both -inf): no
                const float now = Range<kHalf>::follow(m, top, c);
                const float keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - now) * c);
                m = now;
                l *= keep;
#pragma unroll
                for (int j = 0; j < kCols; ++j) o[j] *= keep;
            }
            const float mc = m == -INFINITY ? 0.f : m * c;
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j / 4][j % 4], c, -mc));
                l += w[j];
            }
            u32x4 pw;
#pragma unroll
            for (int i = 0; i < 4; ++i) pw[i] = pack<kHalf>(w[2 * i], w[2 * i + 1]);
            __builtin_amdgcn_sched_barrier(0);  // the columns of V are paired late, into K's registers
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
                u32x4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = __builtin_amdgcn_perm(x.v[2 * i + 1][j / 2], x.v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
                o[j] = mfma16<kHalf>(v, pw, o[j]);
            }
        };
        const int32_t k_end = min(share.to * kKeys, most);
        int32_t k0 = share.from * kKeys + 32 * wave;
        if (k0 < k_end) {
            // pages two steps ahead, so that no load waits for one that was asked for after the last loads
            Step x, y;
            int32_t id0 = page_of(k0), id1 = page_of(k0 + kKeys);
            load(place_of(k0, id0), x);
            while (true) {
                const int32_t id2 = page_of(k0 + 2 * kKeys);
                if (k0 + kKeys < k_end) load(place_of(k0 + kKeys, id1), y);
                compute(k0, id0, x);
                if ((k0 += kKeys) >= k_end) break;
                id0 = page_of(k0 + 2 * kKeys);
                if (k0 + kKeys < k_end) load(place_of(k0 + kKeys, id2), x);
                compute(k0, id1, y);
                if ((k0 += kKeys) >= k_end) break;
                id1 = id0;
                id0 = id2;
            }
        }
        // join the waves: the largest m, then the sums under it
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (grp == 0) {
            tops[wave][col] = m;
            weights[wave][col] = l;
        }
        if (lane == 0) odd[wave] = zeros;
        __syncthreads();
        const bool whole = share.to - share.from == share.all;
        const int64_t at = 2 * (int64_t)blockIdx.x + (share.from == 0);  // a cut tile's partial sums
        const float high = fmaxf(fmaxf(tops[0][col], tops[1][col]), fmaxf(tops[2][col], tops[3][col]));
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - high) * c);
        // o[j][i] is dimension kCols (4 grp + i) + j of query `col`
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kCols; j += 4)
                *reinterpret_cast<f32x4 *>(&joint[wave][col][kCols * (4 * grp + i) + j]) =
                    f32x4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]} * keep;
        __syncthreads();
        // a thread takes a query and kCols dimensions
        const int out_row = threadIdx.x / 16, d0 = kCols * (threadIdx.x % 16);
        const int out_tok = out_row / t.heads, out_h = out_row - out_tok * t.heads;
        if (out_tok < t.n) {
            float sum[kCols] = {}, lsum = 0.f, mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w) mx = fmaxf(mx, tops[w][out_row]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float mw = tops[w][out_row];
                lsum += weights[w][out_row] * (mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - mx) * c));  // (NaN stays)
#pragma unroll
                for (int j = 0; j < kCols; ++j) sum[j] += joint[w][out_row][d0 + j];
            }
            if (least < most && __builtin_expect(odd[0] | odd[1] | odd[2] | odd[3], 0) && d0 < a.dim) {
                const int32_t end = min(kSeen ? most : min(r.base + t.first + out_tok + 1, most), share.to * kKeys);
                for (int32_t k = max(least, share.from * kKeys); k < end; ++k) {
                    if (kSeen && !(seen_of(a, r, r.first + t.first + out_tok, k) & 1)) continue;
                    const uint16_t *v = v_of(a, a.v + (int64_t)t.head * a.head_stride + d0, pages, k);
                    if (!v) continue;
#pragma unroll
                    for (int j = 0; j < kCols; ++j) sum[j] += not_finite<kHalf>(v[j]);
                }
            }
            if (whole) {
                const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
                const int64_t token = r.first + t.first + out_tok;
                const int64_t head = t.head * a.per_kv + t.part * a.group + out_h;
                uint16_t *dst = a.out + token * a.out_token + head * a.out_head + d0;
                if (d0 < a.dim) {
                    uint32_t y[kCols / 2];
#pragma unroll
                    for (int j = 0; j < kCols / 2; ++j) y[j] = pack<kHalf>(sum[2 * j] * inv, sum[2 * j + 1] * inv);
                    if constexpr (kCols == 8) *reinterpret_cast<u32x4 *>(dst) = u32x4{y[0], y[1], y[2], y[3]};
                    else *reinterpret_cast<u32x2 *>(dst) = u32x2{y[0], y[1]};
                }
                if (a.lse && d0 == 0) a.lse[token * a.heads + head] = lsum == 0.f ? -INFINITY : mx * a.scale + logf(lsum);
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
}

// -------------------------------------------------------------------- wide ---

// A tile of 32 kBlocks rows to each of kWaves waves, by 64 keys a unit: the matrix products bound it (256
// rows), or the bytes of K and V (128, for fewer rows).
// K and V go through LDS, two units of each; the next one's bytes are on their way in
// registers while this one is computed.  Keys lie apart in LDS by their bytes and 16 (K) or
// 32 (V) more, which leaves few banks asked twice (6 cycles of 100) and every read at a fixed distance from
// one address.  As above S^T = K Q^T, O^T = V^T P^T (V read from LDS by columns),
// so the weights stay in their lanes.  A wave has its matrix unit to itself, and 64 rows,
// since with 32 the reads of K and V from LDS take as long as the products.  So that the
// matrix unit does not wait for the softmax, a half unit (32 keys) is in three stages at
// once: the products of the next half's scores and of the last half's weights with V run
// beside this half's exponentials.  4,096 tokens over 16,384 keys, 32 heads of 128: 905 to 980 us
// by the card, not traced, 16 of k_join among them, 0.98 to 1.06 PFLOP/s (a bf16 product of 8,192^3 by the library: 1.23), the matrix units
// busy in 47 cycles of 100 at the 2.1 GHz that the power leaves.  Where K and V's bytes bound it a unit takes 2.1
// us, 4 TB/s (32 trees of up to 32 tokens over 158,700, kSeen: 658 MB in 135 to 147 us, 4.5 to 4.9 TB/s, with one block to a CU, on some
// cards 150 to 170; two to four units of each on their way in registers: 138 to 144).
// kSeen in tiles of 256 rows, heads of 128: 16 trees of up to 64 over 74,600 tokens, 32 and 8 heads, 52 GFLOP and 316 MB in 103 to 120 us
// (matrix units 33 cycles of 100, vector issue 31); four of up to 250 over 134,800, 345 GFLOP in 440 to 520 (44 and 40), 0.66 to 0.78 PFLOP/s.
// In heads of up to 64 there are more exponentials and sums to a product, and a second wave beside the first fills its gaps: 256 rows
// in eight waves of 32 (kSeen; four trees of up to 250 tokens over 116,700, 56 GFLOP: 92 us, in four waves of 64 108, in two blocks of 128
// rows 100, whose join takes 5 more).  Neither unit is full (vector issue 55 cycles of 100, matrix units 31): a wave issues in 45 of its
// cycles, waits in 32, for its turn in 23.
constexpr int kWideKeys = 64;

// What is not finite in V of the keys from .. to - 1, added to the sums or outputs that this lane has written (lanes and rows as
// below).  Apart from these, and from the thread's number on, so that it takes none of their registers.
template <int DP, int kWaves, int kBlocks, bool kHalf, bool kSeen>
__device__ inline void add_values(const Attend &a, const Row &r, const Tile &t, int32_t from, int32_t to, bool whole, int64_t at) {
    constexpr int kWaveRows = 32 * kBlocks, kRows = kWaves * kWaveRows;
    int32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int32_t *const pages = a.table + r.slot * a.table_stride;
#pragma unroll 1
    for (int b = 0; b < kBlocks; ++b) {
        const int row = thread / kWave * kWaveRows + 32 * b + thread % 32, tok = row / t.heads, h = row - tok * t.heads;
        if (tok >= t.n) return;
        const int64_t token = r.first + t.first + tok, head = t.head * a.per_kv + t.part * a.group + h;
        uint16_t *const out = a.out + token * a.out_token + head * a.out_head;
        float *const sum = a.sums + (at * kRows + row) * DP;
        const int32_t end = kSeen ? to : min(to, r.base + t.first + tok + 1);
#pragma unroll 1
        for (int32_t key = from; key < end; ++key) {
            if (kSeen && !(seen_of(a, r, token, key) & 1)) continue;
            const uint16_t *const v = v_of(a, a.v + (int64_t)t.head * a.head_stride, pages, key);
            if (!v) continue;
#pragma unroll 1
            for (int d = thread / 8 & 4; d < a.dim; d = d % 4 == 3 ? d + 5 : d + 1) {
                const float x = not_finite<kHalf>(v[d]);
                if (x == 0.f) continue;
                if (whole) out[d] = (uint16_t)pack<kHalf>(to_float<kHalf>(out[d]) + x, 0.f);
                else sum[d] += x;
            }
        }
    }
}

template <int DP, int kWaves, int kBlocks, bool kHalf, bool kRuns, bool kSeen>
__global__ void __launch_bounds__(kWave * kWaves, kWaves == 4 && kBlocks == 1 && DP == 64 ? 2 : 1) k_attend_wide(Attend a) {
    constexpr int kThreads = kWave * kWaves, kWaveRows = 32 * kBlocks, kRows = kWaves * kWaveRows;
    constexpr int kPieces = DP / 8;            // 16-byte pieces of a key
    constexpr int kSteps = DP / 16;            // products over 16 dimensions
    constexpr int kCols = DP / 32;             // blocks of 32 output dimensions
    constexpr int kLoads = kPieces * kWideKeys / kThreads;
    constexpr int kKStride = DP + 8, kVStride = DP + 16;
    constexpr uint32_t kKUnit = kWideKeys * kKStride, kVUnit = kWideKeys * kVStride;
    extern __shared__ __align__(16) uint16_t bufs[];  // two units of K, two of V
    uint16_t *const kbuf = bufs, *const vbuf = bufs + 2 * kKUnit;
    const int lane = threadIdx.x % kWave, wave = uniform((int32_t)threadIdx.x / kWave);
    const int col = lane % 32, half = lane / 32;
    // blocks go to the eight dies in turn: neighbouring pieces, which share K and V, to one die
    const int64_t block = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    // the number, among the block's, of the last tile in which zeros were put in the place of values that are not finite
    __shared__ int32_t odd;
    int32_t number = 0;
    if (threadIdx.x == 0) odd = 0;
    int64_t piece;
    Place p = find<kSeen, kThreads>(a, block, &piece);
    if (p.row < 0) {
        if (threadIdx.x == 0) a.cuts[block].is = 0;
        return;
    }
    const int64_t whole_piece = min(piece, p.total - block * piece);
    int64_t left = whole_piece;
    const float c = a.scale * kLog2e;
    const uint32_t place = (1u << a.shift) - 1;

    // this lane's reads: K rows as the first factor; V by columns: four keys of one dimension
    const uint16_t *const k_read = kbuf + col * kKStride + 8 * half;
    const uint16_t *const v_read = vbuf + (4 * half + (lane % 16) / 4) * kVStride + 16 * (lane / 16 % 2) + 4 * (lane % 4);
    // and its writes: piece `mine` of keys `key`, `key` + kApart, ...
    constexpr int kApart = kThreads / kPieces;
    const int key = threadIdx.x / kPieces, mine = threadIdx.x % kPieces;
    // (K past the last dimension: zeros from here on, since the queries' zeros there would make an infinity NaN; these lanes write
    // into the gap between two keys)
    const bool in_dim = 8 * mine < a.dim;
    uint16_t *const k_write = kbuf + key * kKStride + (in_dim ? 8 * mine : DP), *const v_write = vbuf + key * kVStride + 8 * mine;
    if (!in_dim)
#pragma unroll
        for (int i = 0; i < 2 * kLoads; ++i) *reinterpret_cast<u32x4 *>(kbuf + (key + i * kApart) * kKStride + 8 * mine) = u32x4{0, 0, 0, 0};
    const uint32_t in_run = 2 * ((kRuns ? (uint32_t)(key % 16) * (uint32_t)a.token_stride : 0) + (in_dim ? 8 * mine : 0));

    while (left > 0) {
        const Row r = p.r;
        if (p.rest >= row_keys<kSeen>(a, r) * a.kv_heads * a.parts) {
            p.r = uniform(row_at(a, ++p.row));
            p.rest = 0;
            continue;
        }
        const Tile t = tile_at<kSeen>(a, r, p.rest);
        const Share share = share_of<kWideKeys>(a, t, left);
        if (left == whole_piece) note<kWideKeys>(a, block, r, t, piece);
        p.rest += t.keys - t.rest;
        left -= t.keys - t.rest;
        if (share.from == share.to) continue;  // (the piece ends before the next unit)
        const int32_t all = max(0, r.base + r.n);
        const int32_t most = kSeen ? all : max(0, min(r.base + t.first + t.n, all));
        const int32_t shared_keys = max(0, min(kSeen ? r.base : r.base + t.first + 1, all));  // that every query of the tile's sees
        ++number;
        u32x4 q[kBlocks][kSteps];
        int32_t seen[kBlocks];
        const int half_q = here(half);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int row = kWaveRows * wave + 32 * b + col, tok = row / t.heads, h = row - tok * t.heads;
            const bool is = tok < t.n;
            // (kSeen: the token)
            seen[b] = kSeen ? (is ? r.first + t.first + tok : -1) : is ? max(0, min(r.base + t.first + tok + 1, all)) : 0;
            const uint16_t *src = a.q + (int64_t)(r.first + t.first + tok) * a.q_token +
                                  (int64_t)(t.head * a.per_kv + t.part * a.group + h) * a.q_head;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int d = 16 * s + 8 * half_q;
                q[b][s] = is && d < a.dim ? *reinterpret_cast<const u32x4 *>(src + d) : u32x4{0, 0, 0, 0};
            }
        }
        // keys that every query of the wave's sees (what rows past the tile's come to is written nowhere)
        const int32_t least = kWaveRows * wave / t.heads < t.n
                                  ? (kSeen ? shared_keys : max(0, min(r.base + t.first + kWaveRows * wave / t.heads + 1, all))) : INT_MAX;
        f32x16 o[kBlocks][kCols], sa[kBlocks], sb[kBlocks];
        u32x4 pa[kBlocks][2], pb[kBlocks][2];
        // m and m c; the score above which m follows; sums of weights; the highest of the last scores (this lane's)
        float m[kBlocks], mc[kBlocks], bound[kBlocks], l[kBlocks], top[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            m[b] = bound[b] = -INFINITY;
            mc[b] = l[b] = 0.f;
#pragma unroll
            for (int d = 0; d < kCols; ++d) o[b][d] = f32x16{};
#pragma unroll
            for (int i = 0; i < 2; ++i) pa[b][i] = u32x4{0, 0, 0, 0};
        }
        global_u8 *const kh = (global_u8 *)(a.k + (int64_t)t.head * a.head_stride);
        global_u8 *const vh = (global_u8 *)(a.v + (int64_t)t.head * a.head_stride);
        const int32_t *const pages = a.table + r.slot * a.table_stride;
        int32_t clear = least;  // keys that need no look at the mask; 0 once a page number is bad

        // A unit's keys, one per lane; those past the last one that the tile sees stand for it.  `id`: the
        // pages they lie in.
        auto key_of = [&](int32_t k0) { return min(k0 + lane, most - 1); };
        auto page_of = [&](int32_t k0) { return pages[(uint32_t)key_of(k0) >> a.shift]; };
        // where the keys lie
        auto place_of = [&](int32_t k0, int32_t id) -> uint64_t {
            const bool is = (uint32_t)id < (uint32_t)a.pages;
            if (!__all(is)) clear = 0;
            const uint32_t in = (uint32_t)key_of(k0) & place;
            return place_in<kRuns>(a, is ? id : 0, in);
        };
        u32x4 k_in[kLoads], v_in[kLoads];
        // piece i of this lane's share of a unit's K (or V)
        auto load = [&](global_u8 *from, uint64_t at, int i) -> u32x4 {
            const int j = kApart * i + (kApart > 16 ? wave / 2 * 16 : 0);  // the 16 keys' first
            return *(global_u32x4 *)(from + (kRuns ? lane_of(at, j) : __shfl(at, kApart * i + key)) + in_run);
        };
        auto store_k = [&](int buf, int i) {
            *reinterpret_cast<u32x4 *>(k_write + buf * kKUnit + i * kApart * kKStride) = k_in[i];
        };
        auto store_v = [&](int buf, int i) {
            *reinterpret_cast<u32x4 *>(v_write + buf * kVUnit + i * kApart * kVStride) = v_in[i];
        };
        // V of keys that no query sees or that lie in no page: zeros (their weights are zero, and what
        // lies there may be anything)
        auto clean = [&](int32_t k0, int32_t id) {
            if (__builtin_expect(k0 + kWideKeys > shared_keys || clear == 0, 0)) {
                asm volatile("");
                const uint64_t ok = __ballot((uint32_t)id < (uint32_t)a.pages);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int j = kApart * i + key;
                    if (k0 + j >= most || !(ok >> j & 1)) v_in[i] = u32x4{0, 0, 0, 0};
                }
                if (shared_keys < most) {
                    uint32_t high = 0;
#pragma unroll
                    for (int i = 0; i < kLoads; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) high = exponents<kHalf>(v_in[i][j], high);
                    if (__any((high & 0x80008000u) != 0)) {
                        odd = number;
#pragma unroll
                        for (int i = 0; i < kLoads; ++i)
                            if (k0 + kApart * i + key >= shared_keys)
#pragma unroll
                                for (int j = 0; j < 4; ++j) v_in[i][j] = only_finite<kHalf>(v_in[i][j]);
                    }
                }
            }
        };
        auto read_k = [&](const uint16_t *at, int s) { return *reinterpret_cast<const u32x4 *>(at + 16 * s); };
        auto read_v = [&](const uint16_t *at, int d, int i) -> u32x4 {  // keys 16 i + 4 half + (0..3, 8..11)
            typedef __attribute__((address_space(3))) i16x4 lds;
            const uint16_t *from = at + 32 * d + 16 * i * kVStride;
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds *)from));
            const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds *)(from + 8 * kVStride)));
            return u32x4{x[0], x[1], y[0], y[1]};
        };
        auto k_half = [&](int buf, int h) { return k_read + buf * kKUnit + h * 32 * kKStride; };
        auto v_half = [&](int buf, int h) { return v_read + buf * kVUnit + h * 32 * kVStride; };
        auto highest = [&](const f32x16 &s) {
            float x = s[0];
#pragma unroll
            for (int i = 1; i < 15; i += 2) x = fmaxf(fmaxf(x, s[i]), s[i + 1]);
            return fmaxf(x, s[15]);
        };
        auto gather = [&](const uint16_t *at, const u32x4 (&w)[kBlocks][2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < kCols; ++d) {
                    const u32x4 v = read_v(at, d, i);
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) o[b][d] = mfma32<kHalf>(v, w[b][i], o[b][d]);
                }
        };
        // scores of the half unit h at key k0, of a unit in pages `id`: those not seen are -inf
        auto settle = [&](int32_t k0, int h, int32_t id, f32x16 (&s)[kBlocks]) {
            if (__builtin_expect(k0 + 32 > clear, 0)) {
                asm volatile("");  // a branch, not selections in every turn
                const uint32_t ok = (uint32_t)(__ballot((uint32_t)id < (uint32_t)a.pages) >> 32 * h);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const int32_t rest = kSeen ? 32 : seen[b] - k0 - 4 * half;
                    const uint32_t have = (kSeen ? ok & (seen[b] < 0 ? 0 : seen_of(a, r, seen[b], k0)) : ok) >> 4 * half;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int x = 8 * (i / 4) + i % 4;
                        if (x >= rest || !(have >> x & 1)) s[b][i] = -INFINITY;
                    }
                    top[b] = highest(s[b]);
                }
            }
        };
        // m follows when it lags too far; sums, and the weights w on their way to V, go along.  After the first time it moves
        // by whole powers of two in the weights, so that these, in 16 bits, keep their digits.
        auto follow = [&](u32x4 (&w)[kBlocks][2]) {
            if (__builtin_expect(__any(top[0] > bound[0] || top[kBlocks - 1] > bound[kBlocks - 1]), 0)) {
                asm volatile("");
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(top[b]), __float_as_uint(top[b]), false, false);
                    const float now = Range<kHalf>::follow(m[b], fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])), c);
                    float keep = 1.f;
                    if (m[b] == -INFINITY) {  // nothing has a weight yet
                        if (now != -INFINITY) {
                            keep = 0.f;
                            m[b] = now;
                            mc[b] = now * c;
                        }
                    } else {
                        const float by = ceilf((m[b] - now) * c);
                        keep = ldexpf(1.f, (int)fmaxf(by, -512.f));
                        mc[b] -= by;
                        m[b] = mc[b] / c;
                    }
                    bound[b] = m[b] + Range<kHalf>::kMost / c;
                    l[b] *= keep;
#pragma unroll
                    for (int d = 0; d < kCols; ++d) o[b][d] *= keep;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t x = w[b][i][j];
                            w[b][i][j] = pack<kHalf>(to_float<kHalf>((uint16_t)x) * keep, to_float<kHalf>((uint16_t)(x >> 16)) * keep);
                        }
                }
            }
        };
        // One half unit: its weights from s into w, the next scores into s1, the last weights w0 into O.
        // A step is the two products with one fragment of K or V, the reads of a fragment further on, and
        // a share of the softmax and of `more`; the compiler keeps to the steps' order, which feeds the matrix
        // unit.
        auto stage = [&](const f32x16 (&s)[kBlocks], u32x4 (&w)[kBlocks][2], const uint16_t *k, f32x16 (&s1)[kBlocks], const uint16_t *v,
                         const u32x4 (&w0)[kBlocks][2], auto more) {
            constexpr int kFrags = kSteps + 2 * kCols, kAhead = 2, kWeights = 16 * kBlocks, kEach = kWeights / kFrags;
            constexpr int kTop = (16 + kFrags - kSteps - 2) / (kFrags - kSteps - 1);  // scores looked at in a step
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
                    asm volatile("" : "+v"(y), "+v"(l[b]));  // here, not where they are first used
                    w[b][i / 8][i % 8 / 2] = y;
                }
            };
#pragma unroll
            for (int f = 0; f < kAhead; ++f) fetch(f);
#pragma unroll
            for (int f = 0; f < kFrags; ++f) {
                if (f + kAhead < kFrags) fetch(f + kAhead);
                multiply(f, 0);
#pragma unroll
                for (int e = 0; e < kEach; ++e) weigh(kEach * f + e);
                if constexpr (kBlocks == 2) multiply(f, 1);
                more(f);
                if (f > kSteps) {
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                        for (int i = kTop * (f - kSteps - 1); i < min(16, kTop * (f - kSteps)); ++i)
                            top[b] = i ? fmaxf(top[b], s1[b][i]) : s1[b][0];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };

        const int32_t k0 = share.from * kWideKeys, k1 = share.to * kWideKeys;
        if (k0 < most) {
            // the pages of the unit at hand and of those after it
            int32_t id0 = page_of(k0), id1 = page_of(k0 + kWideKeys), id2 = page_of(k0 + 2 * kWideKeys), id3 = 0;
            const uint64_t at0 = place_of(k0, id0);
            uint64_t at1 = place_of(k0 + kWideKeys, id1);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) k_in[i] = load(kh, at0, i);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) v_in[i] = load(vh, at0, i);  // (with K's, or behind it: takes as long)
            __syncthreads();  // the last tile is done with the buffers
#pragma unroll
            for (int i = 0; i < kLoads; ++i) store_k(0, i);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) k_in[i] = load(kh, at1, i);
            // the half unit before the first has weights of zero and a V of zeros
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                *reinterpret_cast<u32x4 *>(v_write + kVUnit + i * kApart * kVStride) = u32x4{0, 0, 0, 0};
            __syncthreads();
#pragma unroll
            for (int f = 0; f < kSteps; ++f) {
                const u32x4 x = read_k(k_half(0, 0), f);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) sa[b] = mfma32<kHalf>(x, q[b][f], f == 0 ? f32x16{} : sa[b]);
            }
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) top[b] = highest(sa[b]);
            settle(k0, 0, id0, sa);
            follow(pa);
            int x = 0;  // the unit's buffers
            for (int32_t k = k0; k < k1; k += kWideKeys) {
                // This unit's V and the next one's K have been loaded, and go to LDS; the next V and the K of
                // the unit after it set out.
                const uint64_t at2 = place_of(k + 2 * kWideKeys, id2);
                id3 = page_of(k + 3 * kWideKeys);
                clean(k, id0);
                stage(sa, pb, k_half(x, 1), sb, v_half(x ^ 1, 1), pa, [&](int f) {
                    const int i = f / 4;
                    if (i >= kLoads) return;
                    if (f % 4 == 0) {
                        store_k(x ^ 1, i);
                        k_in[i] = load(kh, at2, i);
                    } else if (f % 4 == 2) {
                        store_v(x, i);
                        v_in[i] = load(vh, at1, i);
                    }
                });
                settle(k + 32, 1, id0, sb);
                __syncthreads();
                follow(pb);
                stage(sb, pa, k_half(x ^ 1, 0), sa, v_half(x, 0), pb, [](int) {});
                settle(k + 64, 0, id1, sa);
                if (k + kWideKeys < k1) follow(pa);
                id0 = id1;
                id1 = id2;
                id2 = id3;
                at1 = at2;
                x ^= 1;
            }
            gather(v_half(x ^ 1, 1), pa);
        }
        // o[b][d][i] is dimension 32 d + 8 (i / 4) + 4 half + i % 4 of query `col`
        const bool whole = share.to - share.from == share.all;
        const int64_t at = 2 * block + (share.from == 0);
        const int half_o = here(half);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[b]), __float_as_uint(l[b]), false, false);
            const float sum = __uint_as_float(y[0]) + __uint_as_float(y[1]);
            const int row = kWaveRows * wave + 32 * b + col, tok = row / t.heads, h = row - tok * t.heads;
            if (tok >= t.n) continue;
            if (whole) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                const int64_t token = r.first + t.first + tok, head = t.head * a.per_kv + t.part * a.group + h;
                uint16_t *dst = a.out + token * a.out_token + head * a.out_head;
#pragma unroll
                for (int d = 0; d < kCols; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int dim = 32 * d + 2 * i + 4 * half_o;
                        if (dim < a.dim)
                            *reinterpret_cast<u32x2 *>(dst + dim) =
                                u32x2{pack<kHalf>(o[b][d][i] * inv, o[b][d][i + 1] * inv),
                                      pack<kHalf>(o[b][d][i + 2] * inv, o[b][d][i + 3] * inv)};
                    }
                if (a.lse && half_o == 0)
                    a.lse[token * a.heads + head] = sum == 0.f ? -INFINITY : m[b] * a.scale + logf(sum);
            } else {
                float *dst = a.sums + (at * kRows + row) * DP;
#pragma unroll
                for (int d = 0; d < kCols; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *reinterpret_cast<f32x4 *>(dst + 32 * d + 2 * i + 4 * half_o) =
                            f32x4{o[b][d][i], o[b][d][i + 1], o[b][d][i + 2], o[b][d][i + 3]};
                if (half_o == 0) {
                    float *ml = a.sums + 2 * (int64_t)a.blocks * kRows * DP + (at * kRows + row) * 2;
                    ml[0] = m[b];
                    ml[1] = sum;
                }
            }
        }
        // (`odd` was written before the last barrier, and the next tile writes it after one)
        if (__builtin_expect(k1 > shared_keys && shared_keys < most && odd == number, 0))
            add_values<DP, kWaves, kBlocks, kHalf, kSeen>(a, r, t, max(k0, shared_keys), min(k1, most), whole, at);
    }
}

// ---------------------------------------------------------------------- join ---

// Partial sums of the tiles that a cut goes through.  blockIdx.x is the cut after
// block x; the blocks of a tile's first cut share its rows, a group of threads to a row.
// Where the tile is in many pieces the blocks of all its cuts do, and the groups of one share
// a row's pieces, whose sums meet in LDS.  Where there are few tiles the chain of reads bounds
// it, else the partial sums' bytes.
// us per call: 3.9 for one row of 700 tokens, 7.7 for 4 tiles in 512 pieces (12 with the first
// cut's blocks alone), 15.5 for 255 cuts of 256 rows of 128 (70 MB).
// kSeen: rows of up to 16 pieces take a group each in tiles of 256 too, as their blocks would take several in turn (14.7 -> 10.7
// us for four trees over 116,700 tokens; without a mask the order of the sums stays what it was).
template <int DP, int kRows, bool kHalf, bool kSeen>
__global__ void __launch_bounds__(kThreads) k_join(Attend a) {
    constexpr int kMost = kSeen && kRows == 256 ? 16 : 5;  // pieces of a row that a group takes alone
    constexpr int kLanes = DP / 4, kGroups = kThreads / kLanes;
    __shared__ float part[kGroups][DP];
    __shared__ float part_l[kGroups];
    const Cut t = a.cuts[blockIdx.x + 1];
    const bool many = t.back + t.more >= 4;  // six pieces or more
    if (!t.is || (!many && t.back)) return;
    const int64_t cut = blockIdx.x + 1 - t.back, last = blockIdx.x + 1 + t.more;  // the tile's first cut, and its last
    const int rows = t.n * t.heads, shares = (many ? t.back + t.more + 1 : 1) * gridDim.y;
    const int each = rows <= shares ? 1 : (rows + shares - 1) / shares;
    const int row0 = min((t.back * (int)gridDim.y + (int)blockIdx.y) * each, rows), row1 = min(row0 + each, rows);
    if (row0 == row1) return;
    const float c = a.scale * kLog2e;
    const float *ml = a.sums + 2 * (int64_t)a.blocks * kRows * DP;
    const int lane = threadIdx.x % kLanes, g = threadIdx.x / kLanes;
    // the first piece begins the tile, the others go on with it
    auto slot_of = [&](int64_t i) { return i < cut ? 2 * i + 1 : 2 * i; };
    auto write = [&](int row, f32x4 x, float l, float mx) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int tok = row / t.heads, h = row - tok * t.heads;
        const int64_t token = t.token + tok, head = t.head + h;
        if (4 * lane < a.dim)
            *reinterpret_cast<u32x2 *>(a.out + token * a.out_token + head * a.out_head + 4 * lane) =
                u32x2{pack<kHalf>(x[0] * inv, x[1] * inv), pack<kHalf>(x[2] * inv, x[3] * inv)};
        if (a.lse && lane == 0) a.lse[token * a.heads + head] = l == 0.f ? -INFINITY : mx * a.scale + logf(l);
    };
    const int pieces = t.back + t.more + 2;
    if (!many || (kMost > 5 && pieces <= kMost && row1 - row0 > 1)) {  // a group to a row; five pieces are asked for together
        for (int row = row0 + g; row < row1; row += kGroups) {
            f32x4 x[5], sum{0, 0, 0, 0};
            float mi[5], li[5], mx = -INFINITY, l = 0.f;
            auto fetch = [&](int p0) {
#pragma unroll
                for (int i = 0; i < 5; ++i) {
                    mi[i] = -INFINITY;
                    if (p0 + i >= pieces) continue;
                    const int64_t at = slot_of(cut - 1 + p0 + i) * kRows + row;
                    mi[i] = ml[at * 2];
                    li[i] = ml[at * 2 + 1];
                    x[i] = *reinterpret_cast<const f32x4 *>(a.sums + at * DP + 4 * lane);
                }
            };
            fetch(0);
#pragma unroll
            for (int i = 5; i < kMost; ++i)
                if (i < pieces) mx = fmaxf(mx, ml[(slot_of(cut - 1 + i) * kRows + row) * 2]);
#pragma unroll
            for (int i = 0; i < 5; ++i) mx = fmaxf(mx, mi[i]);
            for (int p = 0;;) {
#pragma unroll
                for (int i = 0; i < 5; ++i) {
                    if (p + i >= pieces) break;
                    const float keep = mi[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mi[i] - mx) * c);
                    sum += x[i] * keep;
                    l += li[i] * keep;
                }
                if (kMost == 5 || (p += 5) >= pieces) break;
                fetch(p);
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
    int rows, keys;   // of a tile, of a unit
    int grid, extra;  // blocks of the launch; keys that stand for a tile's own cost
};

// `seen`: with a mask among the new tokens.
Shape shape_of(const tam_chunk &c, int64_t heads, bool seen) {
    const int64_t longest = c.longest ? std::min(c.longest, c.tokens) : c.tokens;
    const int64_t rows = longest * (heads / c.kv_heads);
    if (rows <= 16) return Shape{16, kNarrowKeys, 512, kNarrowKeys};
    // a batch of mostly short rows fills tiles of 128 rows better (us per call with 128 and 256: 40 chunks of up to
    // 200 tokens, 74 rows on average, 50 and 63; 24 of 265 rows on average, heads of 64, 46 and 41)
    // With a mask one block to a CU: half the cuts, whose sums cost more than a second block's loads bring (us per call in a graph
    // with 256 blocks and 512, 16 tokens of 32 and 8 heads of 128 over 700, 3,000 and 12,000, one request: 15.2, 17.7 and 23.2; 17.5, 20.4
    // and 29.5; four: 18.8, 24.4 and 45.4; 22.8, 29.6 and 52.9; 16: 24.1, 46.5 and 175; 26.4, 51.2 and 181); and a tile's own cost is
    // higher.  (In tiles of 16 rows, which read K and V four times, one request takes 14.7, 20.7 and 34.)
    const bool small = rows <= 128 || c.tokens * (heads / c.kv_heads) <= 128 * c.rows;
    if (seen) return small ? Shape{128, kWideKeys, 256, 4 * kWideKeys} : Shape{256, kWideKeys, 256, 8 * kWideKeys};
    return small ? Shape{128, kWideKeys, 512, 2 * kWideKeys} : Shape{256, kWideKeys, 256, 5 * kWideKeys};
}

int padded(int64_t dim) { return dim <= 64 ? 64 : 128; }

template <int DP, int kRows, bool kHalf, bool kSeen>
hipError_t launch_join(const Attend &a, hipStream_t s) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_join<DP, kRows, kHalf, kSeen>), dim3((unsigned)a.blocks - 1, kRows == 16 ? 4 : 16), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

// whether kRuns holds
bool runs(const Attend &a) {
    return a.shift >= 4 && a.page_stride <= INT32_MAX && a.token_stride <= (INT32_MAX / 2) >> a.shift;
}

template <int DP, int kWaves, int kBlocks, bool kHalf, bool kSeen>
hipError_t launch_wide(const Attend &a, hipStream_t s) {
    constexpr size_t kLds = 2 * kWideKeys * (DP + 8 + DP + 16) * sizeof(uint16_t);
    if (runs(a))
        hipLaunchKernelGGL((k_attend_wide<DP, kWaves, kBlocks, kHalf, true, kSeen>), dim3((unsigned)a.blocks), dim3(kWave * kWaves), kLds, s, a);
    else
        hipLaunchKernelGGL((k_attend_wide<DP, kWaves, kBlocks, kHalf, false, kSeen>), dim3((unsigned)a.blocks), dim3(kWave * kWaves), kLds, s, a);
    return launch_join<DP, 32 * kWaves * kBlocks, kHalf, kSeen>(a, s);
}

template <int DP, bool kHalf, bool kSeen>
hipError_t launch(const Attend &a, const Shape &sh, hipStream_t s) {
    if (sh.rows == 256) {
        if constexpr (DP == 64 && kSeen) return launch_wide<DP, 8, 1, kHalf, kSeen>(a, s);
        else return launch_wide<DP, 4, 2, kHalf, kSeen>(a, s);
    }
    if (sh.rows == 128) return launch_wide<DP, 4, 1, kHalf, kSeen>(a, s);
    if (runs(a))
        hipLaunchKernelGGL((k_attend_narrow<DP, kHalf, true, kSeen>), dim3((unsigned)a.blocks), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((k_attend_narrow<DP, kHalf, false, kSeen>), dim3((unsigned)a.blocks), dim3(kThreads), 0, s, a);
    return launch_join<DP, 16, kHalf, kSeen>(a, s);
}

template <int DP, bool kHalf>
hipError_t launch(const Attend &a, const Shape &sh, hipStream_t s) {
    return a.seen ? launch<DP, kHalf, true>(a, sh, s) : launch<DP, kHalf, false>(a, sh, s);
}

}  // namespace

int64_t attend_work_bytes(const tam_chunk &c, int64_t heads) {
    auto bytes = [&](const Shape &sh) {
        return 2 * (int64_t)sh.grid * sh.rows * (padded(c.head_dim) + 2) * 4 + sh.grid * (int64_t)sizeof(Cut);
    };
    return std::max(bytes(shape_of(c, heads, false)), bytes(shape_of(c, heads, true)));
}

hipError_t launch_attend(const tam_chunk &c, const Queries &q, const Seen &seen, void *work, hipStream_t s) {
    const Shape sh = shape_of(c, q.heads, seen.bits != nullptr);
    const int64_t group = q.heads / c.kv_heads;
    Attend a{static_cast<const uint16_t *>(c.k), static_cast<const uint16_t *>(c.v),
             static_cast<const uint16_t *>(q.q), static_cast<uint16_t *>(q.out), q.lse, c.page_stride,
             c.head_stride, c.token_stride, q.q_token, q.q_head, q.out_token, q.out_head, c.table, c.length,
             c.offsets, c.slot_ids, c.table_stride, c.slots, c.max_pages, c.rows, c.tokens, (int32_t)c.num_pages,
             __builtin_ctzll((unsigned long long)c.page_tokens), (int32_t)q.heads, (int32_t)c.kv_heads,
             (int32_t)group, (int32_t)c.head_dim, q.scale, 0, 0, 0, 0, 0, 0, nullptr, nullptr, seen.bits, seen.stride, seen.words};
    a.group = (int32_t)std::min<int64_t>(group, sh.rows);
    a.parts = (int32_t)((group + a.group - 1) / a.group);
    a.tq = sh.rows / a.group;
    a.blocks = sh.grid;
    a.unit = sh.keys;
    a.extra = sh.extra;
    a.sums = static_cast<float *>(work);
    a.cuts = reinterpret_cast<Cut *>(a.sums + 2 * (int64_t)sh.grid * sh.rows * (padded(c.head_dim) + 2));
    const bool half = c.dtype == TAM_DTYPE_FP16;
    if (padded(c.head_dim) == 64) return half ? launch<64, true>(a, sh, s) : launch<64, false>(a, sh, s);
    return half ? launch<128, true>(a, sh, s) : launch<128, false>(a, sh, s);
}

}  // namespace tam
