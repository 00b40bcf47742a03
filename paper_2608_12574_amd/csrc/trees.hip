// Trees of drafted tokens: which tokens each one sees, and the path that the model's choices follow.
//
// A row's tokens are a forest: token j of the row follows token p = parents[j] if 0 <= p < j, else the text
// before the row.  Parents come before their children, so every walk up or down ends.
//
// k_tree: seen(j) = {j} + seen(p), depth(j) = depth(p) + 1.  A chain of LDS reads per token: 1.9 us for one tree of 16, 4.4 for 256 of
// up to 256 tokens (31,000, 1.2 MB), where a block takes as long as its deepest token's chain.
// k_walk: from token 0 on to the first child that the choice made after a token names (below 0: none); a token that stays at depth d moves to
// place d of the row, the row's other tokens are cut off, and pages past the new length are given back.
// k_shift: the moves themselves, in every plane.  path[d] >= d grows with d, so a place moved to is never one that
// a later token is still to be moved from, and a thread may move its piece of the tokens in their order.  The walk is a trip to
// memory per step of the path, the moves are bound by their bytes where there are many: 128 trees of up to 64 tokens in 8 layers 11.6 to
// 13.6 us (8 MB, in one launch, on half of the CUs; a wave waits in 89 cycles of 100), 128 of 32 tokens in 32 layers 16 to 18 (45 MB), of
// which the walk takes 6 and the moves 10.5 to 12 (3.7 to 4.3 TB/s; waits in 73).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"

namespace tam {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;

// The tokens of row i among all of a call's.
struct Span {
    int64_t lo;
    int32_t n;
};

__device__ inline Span span_of(const int32_t *offsets, int64_t i, int64_t tokens) {
    if (!offsets) return Span{i, i < tokens};
    const int64_t lo = max((int64_t)offsets[i], (int64_t)0), hi = min((int64_t)offsets[i + 1], tokens);
    return Span{lo, (int32_t)max(hi - lo, (int64_t)0)};
}

// ------------------------------------------------------------------- masks ---

// A block takes a row, a thread a token: once up the chain of parents, in LDS where the row fits (the ancestors' numbers fall, so
// that a word's are a run of the chain, and it is written where they end).
constexpr int kTreeThreads = 256, kHeld = 4096;

__global__ void __launch_bounds__(kTreeThreads) k_tree(const int32_t *__restrict__ parents, const int32_t *__restrict__ offsets,
                                                       int64_t tokens, uint64_t *__restrict__ seen, int64_t words,
                                                       int32_t *__restrict__ depth) {
    __shared__ int32_t held[kHeld];
    const Span s = span_of(offsets, blockIdx.x, tokens);
    const int32_t *up = parents + s.lo;
    const bool in_lds = s.n <= kHeld;
    if (in_lds) {
        for (int j = threadIdx.x; j < s.n; j += kTreeThreads) held[j] = up[j];
        __syncthreads();
    }
    auto parent = [&](int32_t j) {
        const int32_t p = in_lds ? held[j] : up[j];
        return p < j ? p : -1;
    };
    for (int64_t i = threadIdx.x; i < s.n; i += kTreeThreads) {
        const int32_t j = (int32_t)i;
        uint64_t *row = seen + (s.lo + j) * words;
        int64_t w = words;  // the words from here on are written
        uint64_t bits = 0;
        int32_t deep = -1;
        for (int32_t at = j; at >= 0; at = parent(at), ++deep) {
            const int64_t of = at >> 6;
            if (of < w) {
                if (w < words) row[w] = bits;
                while (--w > of) row[w] = 0;
                bits = 0;
            }
            if (of == w) bits |= 1ull << (at & 63);
        }
        if (w < words) row[w] = bits;
        while (--w >= 0) row[w] = 0;
        depth[s.lo + j] = deep;
    }
}

// -------------------------------------------------------------------- path ---

struct Walk {
    const int32_t *tokens, *picks, *parents, *offsets, *slot_ids;
    int64_t rows, total;
    int32_t *table, *length, *refs;
    int64_t slots, max_pages, table_stride;
    int32_t pages, shift;
    int64_t page_stride, token_stride;  // bytes
    int32_t *path, *count, *last;
    int64_t *src, *dst;  // [total] where the token at each depth lies, and goes, in a plane; -1: nowhere
    int32_t *first;      // [rows] the first depth that moves
};

// A wave takes a row.  The children of a token come after it, so that a step looks at the tokens from there on, 64 at a time.
// (With the lists in registers a call takes as long.)
__device__ inline void walk(const Walk &a, int64_t i, int lane) {
    const Span s = span_of(a.offsets, i, a.total);
    const int64_t slot = a.slot_ids ? a.slot_ids[i] : i;
    const bool is = slot >= 0 && slot < a.slots;
    const int32_t most = (int32_t)(a.max_pages << a.shift);
    const int32_t len = is ? min(max(a.length[slot], 0), most) : 0;
    if (!is || s.n == 0) {  // nothing stays, nothing changes
        for (int64_t d = lane; d < s.n; d += kWave) a.path[s.lo + d] = -1;
        if (lane == 0) {
            a.count[i] = a.first[i] = 0;
            a.last[i] = -1;
        }
        return;
    }
    const int32_t base = len - s.n;
    int32_t *const row = a.table + slot * a.table_stride;
    auto place = [&](int32_t p) -> int64_t {  // of a position, in a plane
        if (p < 0 || p >= most) return -1;
        const int32_t page = row[p >> a.shift];
        if ((uint32_t)page >= (uint32_t)a.pages) return -1;
        return page * a.page_stride + (p & ((1 << a.shift) - 1)) * a.token_stride;
    };
    int32_t here = 0, d = 0, mine = -1, from = INT_MAX;
    int32_t want = a.picks[s.lo];
    auto write = [&](int32_t d0, int32_t stay) {  // depths d0 + lane, of which `stay` stay
        if (lane >= stay) return;
        a.path[s.lo + d0 + lane] = mine;
        const bool moves = mine != d0 + lane;
        a.src[s.lo + d0 + lane] = moves ? place(base + mine) : -1;
        a.dst[s.lo + d0 + lane] = moves ? place(base + d0 + lane) : -1;
    };
    while (true) {
        if (lane == d % kWave) mine = here;
        if (here != d) from = min(from, d);
        if (d % kWave == kWave - 1) write(d - (kWave - 1), kWave);
        ++d;
        int32_t then = -1;
        for (int64_t j0 = here + 1; want >= 0 && j0 < s.n; j0 += kWave) {
            const int64_t j = j0 + lane;
            const uint64_t some = __ballot(j < s.n && a.parents[s.lo + j] == here && a.tokens[s.lo + j] == want);
            if (some) {
                then = (int32_t)j0 + __builtin_ctzll(some);
                break;
            }
        }
        if (then < 0) break;
        here = then;
        want = a.picks[s.lo + here];
    }
    if (d % kWave) write(d / kWave * kWave, d % kWave);
    for (int64_t j = (int64_t)d + lane; j < s.n; j += kWave) a.path[s.lo + j] = -1;
    const int32_t now = max(base + d, 0);
    if (lane == 0) {
        a.count[i] = d;
        a.last[i] = want;
        a.first[i] = min(from, d);
        a.length[slot] = now;
    }
    // (the places above have been read: the stores before this one needed them)
    const int32_t held = (len + (1 << a.shift) - 1) >> a.shift, keep = (now + (1 << a.shift) - 1) >> a.shift;
    for (int32_t j = keep + lane; j < held; j += kWave) {
        const int32_t page = row[j];
        if ((uint32_t)page < (uint32_t)a.pages) atomicSub(&a.refs[page], 1);
        row[j] = -1;
    }
}

__global__ void __launch_bounds__(kWave) k_walk(Walk a) { walk(a, blockIdx.x, threadIdx.x); }

struct Shift {
    uint8_t *data;
    int64_t plane_stride, head_stride;  // bytes
    const int32_t *offsets, *count, *first;
    const int64_t *src, *dst;
    int64_t total;
    int32_t heads, pieces;  // of 16 bytes, of a vector
    int64_t items;          // planes * heads * pieces
};

constexpr int kShiftThreads = 256, kTogether = 4;

// A thread takes 16 bytes of a plane and head (items x, x + step, ...), of all the tokens of row i that move.
__device__ inline void shift(const Shift &a, int64_t i, int64_t x, int64_t step) {
    const int32_t from = a.first[i], to = a.count[i];
    if (from >= to) return;
    const int64_t lo = span_of(a.offsets, i, a.total).lo;
    for (; x < a.items; x += step) {
        const int64_t vector = x / a.pieces, plane = vector / a.heads;
        uint8_t *const at = a.data + plane * a.plane_stride + (vector - plane * a.heads) * a.head_stride + (x - vector * a.pieces) * 16;
        for (int32_t d = from; d < to; d += kTogether) {
            u32x4 v[kTogether];
            int64_t src[kTogether], dst[kTogether];
#pragma unroll
            for (int e = 0; e < kTogether; ++e) {
                src[e] = d + e < to ? a.src[lo + d + e] : -1;
                dst[e] = d + e < to ? a.dst[lo + d + e] : -1;
                if (src[e] >= 0 && dst[e] >= 0) v[e] = *reinterpret_cast<const u32x4 *>(at + src[e]);
            }
#pragma unroll
            for (int e = 0; e < kTogether; ++e)
                if (src[e] >= 0 && dst[e] >= 0) *reinterpret_cast<u32x4 *>(at + dst[e]) = v[e];
        }
    }
}

__global__ void __launch_bounds__(kShiftThreads) k_shift(Shift a) {
    shift(a, blockIdx.x, blockIdx.y * (int64_t)kShiftThreads + threadIdx.x, (int64_t)gridDim.y * kShiftThreads);
}

// Both for a row in one block.
constexpr int kBothThreads = 1024;

__global__ void __launch_bounds__(kBothThreads) k_walk_shift(Walk w, Shift a) {
    if (threadIdx.x < kWave) walk(w, blockIdx.x, threadIdx.x);
    __syncthreads();
    shift(a, blockIdx.x, threadIdx.x, kBothThreads);
}

}  // namespace

hipError_t launch_tree_masks(const int32_t *parents, const int32_t *offsets, int64_t rows, int64_t tokens, uint64_t *seen,
                             int64_t words, int32_t *depth, hipStream_t s) {
    hipLaunchKernelGGL(k_tree, dim3((unsigned)rows), dim3(kTreeThreads), 0, s, parents, offsets, tokens, seen, words, depth);
    return hipGetLastError();
}

// Up to this many pieces of 16 bytes to a token (8 layers of 8 heads of 128) one launch does both, which costs the host 2.5 us
// less.  us on the device per call of 1 and 128 trees of 32 tokens, 4 layers: 2.6 and 7.0, in two launches 3.9 and 7.4; 8 layers:
// 5.3 and 10.4, 5.5 and 9.4; 16 layers: 7.3 and 13.5, 5.8 and 11.5.  (The rows are not asked: many of them in 5 to 8 layers lose up to
// 1 us by it where a graph has spared the host its part.)
constexpr int64_t kBothItems = 2048;
constexpr int64_t kBothRows = ((1ll << 32) - 1) / kBothThreads;  // a launch has fewer than 2^32 threads

// places from and to of each token, and each row's first move
int64_t accept_work_bytes(const tam_chunk &n) { return 16 * n.tokens + 4 * n.rows; }

hipError_t launch_pages_accept(const tam_pages &c, const tam_chunk &n, const int32_t *tokens, const int32_t *picks,
                               const int32_t *parents, int32_t *path, int32_t *count, int32_t *last, void *work, hipStream_t s) {
    int64_t *src = static_cast<int64_t *>(work), *dst = src + n.tokens;
    int32_t *first = reinterpret_cast<int32_t *>(dst + n.tokens);
    const Walk a{tokens, picks, parents, n.offsets, n.slot_ids, n.rows, n.tokens, c.table, c.length, c.refs, c.slots, c.max_pages,
                 c.table_stride, (int32_t)c.num_pages, __builtin_ctzll((unsigned long long)c.page_tokens), c.page_stride,
                 2 * n.token_stride, path, count, last, src, dst, first};
    const int64_t pieces = n.head_dim / 8, items = c.planes * n.kv_heads * pieces;
    const Shift m{static_cast<uint8_t *>(c.data), c.plane_stride, 2 * n.head_stride, n.offsets, count, first, src, dst, n.tokens,
                  (int32_t)n.kv_heads, (int32_t)pieces, items};
    if (items <= kBothItems && n.rows <= kBothRows) {
        hipLaunchKernelGGL(k_walk_shift, dim3((unsigned)n.rows), dim3(kBothThreads), 0, s, a, m);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(k_walk, dim3((unsigned)n.rows), dim3(kWave), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t blocks = std::min<int64_t>((items + kShiftThreads - 1) / kShiftThreads, 1024);
    hipLaunchKernelGGL(k_shift, dim3((unsigned)n.rows, (unsigned)blocks), dim3(kShiftThreads), 0, s, m);
    return hipGetLastError();
}

}  // namespace tam
