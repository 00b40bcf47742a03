// The pages of a K/V cache: fork, extend, compact and store.
//
// Which pages a call gives, copies and moves is decided on the device, from the
// tables that lie there, so a decode step needs no answer from the host.  A page
// is free when its count is 0; there is no list of free pages to keep in step.  A
// call that takes pages finds the lowest free ones by a pass over the counts
// (4 bytes per page).  The decisions are one block's work (k_extend, 6.0 us for 4 rows and
// 7.4 for 256; k_plan, 6.7 us for 2,048 pages): a few dependent trips to memory and
// prefix sums over the rows or the pages bound them.  The page contents are moved by a
// launch of their own over the whole chip, which its bytes bound (k_copy: 126 MB read and
// written in 27 us, k_move: 537 MB in 113 us, 4.7 TB/s; a large copy reaches 5.1).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "step.hpp"

namespace tam {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;
constexpr int kPlan = 1024;  // threads of the deciding blocks
constexpr int kBlock = 256;

// Sequences and counts of a call; pages of a slot by its length.
struct Tables {
    int32_t *table, *length, *refs;
    int64_t slots, max_pages, stride;
    int32_t pages, shift;  // tokens of a page: 1 << shift

    __device__ bool slot_ok(int64_t s) const { return s >= 0 && s < slots; }
    // a length the table can hold
    __device__ int64_t tokens(int64_t s) const { return min(max((int64_t)length[s], (int64_t)0), max_pages << shift); }
    __device__ int64_t held(int64_t t) const { return (t + (1 << shift) - 1) >> shift; }
    __device__ bool page_ok(int32_t p) const { return (uint32_t)p < (uint32_t)pages; }
};

Tables tables_of(const tam_pages &c) {
    return Tables{c.table, c.length, c.refs, c.slots, c.max_pages, c.table_stride, (int32_t)c.num_pages,
                  __builtin_ctzll((unsigned long long)c.page_tokens)};
}

// Sum over the threads before this one, and over all of them (kPlan threads).
__device__ int64_t scan(int64_t x, int64_t *total) {
    __shared__ int64_t sums[kPlan / kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int64_t y = x;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int64_t up = __shfl_up(y, d);
        if (lane >= d) y += up;
    }
    __syncthreads();  // the last call's sums have been read
    if (lane == kWave - 1) sums[wave] = y;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlan / kWave; ++w) {
        const int64_t v = sums[w];
        before += w < wave ? v : 0;
        all += v;
    }
    *total = all;
    return before + y - x;
}

// ------------------------------------------------------------------- fork ---

// The new rows into `rows` ([n][max_pages]) and their lengths into `lens`, and the
// counts: the tables still hold the old rows, which are every row's parents.
__device__ void fork_read(const Tables &t, const int32_t *slots, const int32_t *parents, const int32_t *lengths,
                          int64_t i, int32_t *rows, int32_t *lens, int first, int step) {
    const int64_t slot = slots[i], parent = parents[i];
    if (!t.slot_ok(slot)) return;
    const bool from = t.slot_ok(parent);
    int64_t len = from ? t.tokens(parent) : 0;
    if (from && lengths) len = min(len, max((int64_t)lengths[i], (int64_t)0));
    const int64_t old = t.held(t.tokens(slot)), now = t.held(len);
    for (int64_t j = first; j < t.max_pages; j += step) {
        const int32_t was = j < old ? t.table[slot * t.stride + j] : -1;
        const int32_t is = j < now ? t.table[parent * t.stride + j] : -1;
        if (is != was) {
            if (t.page_ok(is)) atomicAdd(&t.refs[is], 1);
            if (t.page_ok(was)) atomicSub(&t.refs[was], 1);
        }
        rows[i * t.max_pages + j] = is;
    }
    if (first == 0) lens[i] = (int32_t)len;
}

__device__ void fork_write(const Tables &t, const int32_t *slots, int64_t i, const int32_t *rows, const int32_t *lens,
                           int first, int step) {
    const int64_t slot = slots[i];
    if (!t.slot_ok(slot)) return;
    for (int64_t j = first; j < t.max_pages; j += step) t.table[slot * t.stride + j] = rows[i * t.max_pages + j];
    if (first == 0) t.length[slot] = lens[i];
}

__global__ void __launch_bounds__(kBlock) k_fork_read(Tables t, const int32_t *slots, const int32_t *parents,
                                                      const int32_t *lengths, int32_t *rows, int32_t *lens) {
    fork_read(t, slots, parents, lengths, blockIdx.x, rows, lens, threadIdx.x, kBlock);
}

__global__ void __launch_bounds__(kBlock) k_fork_write(Tables t, const int32_t *slots, const int32_t *rows,
                                                       const int32_t *lens) {
    fork_write(t, slots, blockIdx.x, rows, lens, threadIdx.x, kBlock);
}

// A few rows: one block does both, a wave per row.
__global__ void __launch_bounds__(kPlan) k_fork_few(Tables t, const int32_t *slots, const int32_t *parents,
                                                    const int32_t *lengths, int64_t n, int32_t *rows, int32_t *lens) {
    const int lane = threadIdx.x % kWave;
    for (int64_t i = threadIdx.x / kWave; i < n; i += kPlan / kWave)
        fork_read(t, slots, parents, lengths, i, rows, lens, lane, kWave);
    __syncthreads();
    for (int64_t i = threadIdx.x / kWave; i < n; i += kPlan / kWave) fork_write(t, slots, i, rows, lens, lane, kWave);
}

// ----------------------------------------------------------------- extend ---

// A call's scratch: per row the pages it needs (exclusive sum) and its copy; per
// page what the rows say of it; the free pages taken.
struct ExtendWork {
    int32_t *start;   // [n] pages needed by the rows before
    int32_t *last;    // [n] the partly filled last page, or -1; then the row's tokens
    int32_t *src;     // [n] the page copied, or -1
    int32_t *dst;     // [n] to where
    int32_t *sharers; // [pages] rows that write on in the page
    int32_t *final_;  // [pages] the last such row
    int32_t *got;     // [pages] free pages, ascending
};

// kOne: a row per thread (at most kPlan of them), which keeps it in registers, and the rows of a page are
// found in a hash table in LDS instead of the scratch (us of a step of 4 and of 256 beams: 12.3 and 41.6, with
// !kOne 14.2 and 44).
template <bool kOne>
__global__ void __launch_bounds__(kPlan) k_extend(Tables t, const int32_t *__restrict__ slots,
                                                  const int32_t *__restrict__ counts, int64_t n, int32_t *info,
                                                  ExtendWork w) {
    const int64_t mask = ((int64_t)1 << t.shift) - 1;
    constexpr int kPlaces = kOne ? 2 * kPlan : 1;
    __shared__ int32_t page_of[kPlaces], sharers_of[kPlaces], final_of[kPlaces];
    // A row, and the pages it needs.
    struct Row {
        int64_t slot, len, count;  // slot < 0: nothing to do
        int32_t page, start, copy;  // the partly filled last page or -1; pages needed by the rows before; copied
    };
    auto row_at = [&](int64_t i) {
        Row r{-1, 0, 0, -1, 0, 0};
        if (i >= n) return r;
        const int64_t slot = slots[i], count = counts[i];
        if (!t.slot_ok(slot) || count <= 0) return r;
        r.slot = slot;
        r.count = count;
        r.len = t.tokens(slot);
        if (r.len & mask) r.page = t.table[slot * t.stride + (r.len >> t.shift)];
        if (!t.page_ok(r.page)) r.page = -1;
        return r;
    };
    // the first counts of the search for free pages, which wait for nothing
    int32_t refs0[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t p = 4 * (int64_t)threadIdx.x + j;
        refs0[j] = p < t.pages ? t.refs[p] : 1;
    }
    // rows that write on in a page
    Row mine{-1, 0, 0, -1, 0, 0};
    if (kOne) mine = row_at(threadIdx.x);
    int32_t holders = 0, at_place = 0;
    if constexpr (kOne) {
        if (mine.page >= 0) holders = t.refs[mine.page];
        for (int i = threadIdx.x; i < kPlaces; i += kPlan) page_of[i] = final_of[i] = -1, sharers_of[i] = 0;
        __syncthreads();
        if (mine.page >= 0) {
            uint32_t at = ((uint32_t)mine.page * 0x9E3779B1u) >> 21;  // (there are twice as many places as rows)
            while (true) {
                const int32_t was = atomicCAS(&page_of[at], -1, mine.page);
                if (was == -1 || was == mine.page) break;
                at = (at + 1) % kPlaces;
            }
            atomicAdd(&sharers_of[at], 1);
            atomicMax(&final_of[at], (int32_t)threadIdx.x);
            at_place = (int32_t)at;
        }
        __syncthreads();
    } else {
        for (int64_t i = threadIdx.x; i < n; i += kPlan) {
            const int32_t page = row_at(i).page;
            w.last[i] = page;
            if (page >= 0) w.sharers[page] = 0, w.final_[page] = -1;
        }
        __syncthreads();
        for (int64_t i = threadIdx.x; i < n; i += kPlan) {
            const int32_t page = w.last[i];
            if (page >= 0) {
                atomicAdd(&w.sharers[page], 1);
                atomicMax(&w.final_[page], (int32_t)i);
            }
        }
        __syncthreads();
    }
    // pages needed, row after row; rows too long for the table in the sum's upper bits
    constexpr int kWide = 48;
    int64_t need = 0, narrow = 0;
    for (int64_t i0 = 0; i0 < n; i0 += kPlan) {
        const int64_t i = i0 + threadIdx.x;
        Row r = kOne ? mine : row_at(i);
        int64_t pages = 0;
        bool wide = false;
        if (r.slot >= 0) {
            if (kOne && r.page >= 0)
                r.copy = holders != sharers_of[at_place] || final_of[at_place] != (int32_t)i;
            if (!kOne && r.page >= 0)  // device-scope reads: the block's own atomics wrote these words
                r.copy = t.refs[r.page] != __hip_atomic_load(&w.sharers[r.page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ||
                         __hip_atomic_load(&w.final_[r.page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != (int32_t)i;
            const int64_t total = t.held(r.len + r.count);
            wide = total > t.max_pages;
            pages = r.copy + total - t.held(r.len);
        }
        int64_t sum;
        const int64_t before = scan(pages | (int64_t)wide << kWide, &sum) & ((1ll << kWide) - 1);
        r.start = (int32_t)min(need + before, (int64_t)INT_MAX);
        need += sum & ((1ll << kWide) - 1);
        narrow += sum >> kWide;
        if (kOne) {
            mine = r;
        } else if (i < n) {
            w.start[i] = r.start;
            w.src[i] = r.copy ? r.page : -1;
            w.last[i] = (int32_t)r.len;
        }
    }
    // the free pages, in order
    int64_t nfree = 0;
    for (int64_t p0 = 0; p0 < t.pages; p0 += 4 * kPlan) {
        const int64_t p = p0 + 4 * (int64_t)threadIdx.x;
        bool is[4];
        int64_t own = 0, sum;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            is[j] = p + j < t.pages && (p0 ? t.refs[p + j] : refs0[j]) <= 0;
            own += is[j];
        }
        int64_t at = nfree + scan(own, &sum);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (is[j]) {
                if (at < need) w.got[at] = (int32_t)(p + j);
                ++at;
            }
        nfree += sum;
    }
    const bool done = need <= nfree && narrow == 0;
    if (threadIdx.x == 0) {
        info[0] = done;
        info[1] = (int32_t)min(need, (int64_t)INT_MAX);
        info[2] = (int32_t)nfree;
        info[3] = (int32_t)narrow;
    }
    __syncthreads();
    if (!done) {
        for (int64_t i = threadIdx.x; i < n; i += kPlan) w.src[i] = -1;
        return;
    }
    // The pages are handed out: a thread takes a row, and the rows that get many pages go to the whole wave.
    constexpr int kAlone = 4;
    const int lane = threadIdx.x % kWave;
    for (int64_t i0 = 0; i0 < n; i0 += kPlan) {
        const int64_t i = i0 + threadIdx.x;
        Row r = mine;
        if (kOne && i < n) w.src[i] = r.copy ? r.page : -1;
        if (!kOne) {  // as it was counted above
            r = Row{-1, 0, 0, -1, 0, 0};
            if (i < n && t.slot_ok(slots[i]) && counts[i] > 0)
                r = Row{slots[i], w.last[i], counts[i], w.src[i], w.start[i], w.src[i] >= 0};
        }
        int64_t first = 0, total = 0;
        if (r.slot >= 0) {
            total = t.held(r.len + r.count);
            first = t.held(r.len) - r.copy;
            if (r.copy) {
                w.dst[i] = w.got[r.start];
                atomicSub(&t.refs[r.page], 1);
            }
            t.length[r.slot] = (int32_t)(r.len + r.count);
            for (int64_t j = first; j < min(total, first + kAlone); ++j) {
                const int32_t page = w.got[r.start + (j - first)];
                t.table[r.slot * t.stride + j] = page;
                t.refs[page] = 1;
            }
        }
        for (uint64_t rest = __ballot(total - first > kAlone); rest; rest &= rest - 1) {
            const int of = __ffsll((unsigned long long)rest) - 1;
            const int64_t s = __shfl(r.slot, of), f = __shfl(first, of), m = __shfl(total, of);
            const int32_t at = __shfl(r.start, of);
            for (int64_t j = f + kAlone + lane; j < m; j += kWave) {
                const int32_t page = w.got[at + (j - f)];
                t.table[s * t.stride + j] = page;
                t.refs[page] = 1;
            }
        }
    }
}

// ------------------------------------------------------------------- copy ---

struct Pool {
    uint8_t *data;
    int64_t planes, plane_stride, page_stride, page_bytes;
};

// Item k is plane k % planes of pair k / planes; a block per item, `blocks` of them, grid-stride.  The
// number of pairs is n, or *count where that is smaller.
template <typename V>
__device__ void copy_pages(const Pool &p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int64_t n,
                           const int32_t *count, int64_t block, int64_t blocks) {
    if (count) n = min(n, (int64_t)*count);
    const int64_t items = n * p.planes, words = p.page_bytes / (int64_t)sizeof(V);
    for (int64_t k = block; k < items; k += blocks) {
        const int64_t pair = k / p.planes, plane = k - pair * p.planes;
        if (src[pair] < 0) continue;
        const V *from = reinterpret_cast<const V *>(p.data + plane * p.plane_stride + src[pair] * p.page_stride);
        V *to = reinterpret_cast<V *>(p.data + plane * p.plane_stride + dst[pair] * p.page_stride);
        for (int64_t i = threadIdx.x; i < words; i += kBlock) to[i] = from[i];
    }
}

template <typename V>
__global__ void __launch_bounds__(kBlock) k_copy(Pool p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                 int64_t n) {
    copy_pages<V>(p, src, dst, n, nullptr, blockIdx.x, gridDim.x);
}

constexpr int64_t kCopyBlocks = 256 * 16;

Pool pool_of(const tam_pages &c) {
    return Pool{static_cast<uint8_t *>(c.data), c.planes, c.plane_stride, c.page_stride, c.page_bytes};
}

// whether pages can be moved in pieces of 16 bytes
bool in_pieces(const tam_pages &c) {
    return (reinterpret_cast<uintptr_t>(c.data) | (uint64_t)c.plane_stride | (uint64_t)c.page_stride | (uint64_t)c.page_bytes) % 16 == 0;
}

// blocks for up to n pages
int64_t copy_blocks(const tam_pages &c, int64_t n) {
    if (c.planes == 0 || c.page_bytes == 0) return 0;
    return n > kCopyBlocks ? kCopyBlocks : std::min(n * c.planes, kCopyBlocks);
}

hipError_t launch_copy(const tam_pages &c, const int32_t *src, const int32_t *dst, int64_t n, hipStream_t s) {
    const int64_t blocks = copy_blocks(c, n);
    if (!blocks) return hipSuccess;
    hipLaunchKernelGGL(in_pieces(c) ? k_copy<u32x4> : k_copy<uint8_t>, dim3((unsigned)blocks), dim3(kBlock), 0, s, pool_of(c), src,
                       dst, n);
    return hipGetLastError();
}

// ---------------------------------------------------------------- compact ---

// Pages in use at or above the number of them (`src`) and free pages below it
// (`dst`), both ascending; the new numbers and counts.
__global__ void __launch_bounds__(kPlan) k_plan(Tables t, int32_t *info, int32_t *__restrict__ moved, int32_t *src,
                                                int32_t *dst) {
    int64_t sum, used = 0;
    {
        int64_t mine = 0;
        for (int64_t p = threadIdx.x; p < t.pages; p += kPlan) mine += t.refs[p] > 0;
        scan(mine, &used);
    }
    int64_t out = 0, hole = 0;
    for (int64_t p0 = 0; p0 < t.pages; p0 += kPlan) {
        const int64_t p = p0 + threadIdx.x;
        const bool in = p < t.pages, is = in && t.refs[p] > 0;
        const bool goes = is && p >= used, gap = in && !is && p < used;
        // both sums in one scan
        const int64_t at = scan(((int64_t)goes << 32) | (int64_t)gap, &sum);
        if (goes) src[out + (at >> 32)] = (int32_t)p;
        if (gap) dst[hole + (at & 0xFFFFFFFF)] = (int32_t)p;
        if (in) moved[p] = is ? (int32_t)p : -1;
        out += sum >> 32;
        hole += sum & 0xFFFFFFFF;
    }
    __syncthreads();
    for (int64_t k = threadIdx.x; k < out; k += kPlan) {
        const int32_t a = src[k], b = dst[k];
        moved[a] = b;
        t.refs[b] = t.refs[a];
        t.refs[a] = 0;
    }
    if (threadIdx.x == 0) {
        info[0] = (int32_t)used;
        info[1] = (int32_t)out;
    }
}

// The tables' new numbers, a block per slot, and beside them the pages' contents (one launch: 2 us less than two).
template <typename V>
__global__ void __launch_bounds__(kBlock) k_move(Tables t, const int32_t *__restrict__ moved, Pool p,
                                                 const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int64_t n,
                                                 const int32_t *count) {
    const int64_t slot = blockIdx.x;
    if (slot >= t.slots) return copy_pages<V>(p, src, dst, n, count, slot - t.slots, gridDim.x - t.slots);
    const int64_t held = t.held(t.tokens(slot));
    for (int64_t j = threadIdx.x; j < t.max_pages; j += kBlock) {
        int32_t *at = t.table + slot * t.stride + j;
        const int32_t p = j < held ? *at : -1;
        *at = t.page_ok(p) ? moved[p] : -1;
    }
}

// ------------------------------------------------------------------ store ---

struct Store {
    uint16_t *k, *v;
    int64_t page_stride, head_stride, token_stride;
    const uint16_t *k_new, *v_new;
    int64_t k_token, k_head, v_token, v_head;
    const int32_t *table, *length, *offsets, *slot_ids;
    int64_t table_stride, slots, max_pages, pages, rows, tokens;
    int32_t shift, heads, chunks;  // chunks: 16-byte pieces of a head's vector
};

// The row of a token: the last one that starts at or before it.
__device__ int64_t row_of(const int32_t *offsets, int64_t rows, int64_t t) {
    int64_t lo = 0, hi = rows;  // offsets[lo] <= t < offsets[hi]
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A block per token: 16 bytes of K and of V per thread and turn.  The bytes bound it: 3,074 tokens of 8 heads of
// 128, 25 MB read and written, in 7.1 us (3.5 TB/s).
__global__ void __launch_bounds__(kBlock) k_store(Store a) {
    const int64_t t = blockIdx.x;
    int64_t row = t, j = 0, n = 1;
    if (a.offsets) {
        if (t < a.offsets[0] || t >= a.offsets[a.rows]) return;
        row = row_of(a.offsets, a.rows, t);
        j = t - a.offsets[row];
        n = (int64_t)a.offsets[row + 1] - a.offsets[row];
    } else if (t >= a.rows) {
        return;
    }
    const int64_t slot = a.slot_ids ? a.slot_ids[row] : row;
    if (slot < 0 || slot >= a.slots) return;
    const int64_t pos = (int64_t)a.length[slot] - n + j;
    if (pos < 0 || (pos >> a.shift) >= a.max_pages) return;
    const int64_t page = a.table[slot * a.table_stride + (pos >> a.shift)];
    if (page < 0 || page >= a.pages) return;
    const int64_t to = page * a.page_stride + (pos & ((1ll << a.shift) - 1)) * a.token_stride;
    for (int i = threadIdx.x; i < a.heads * a.chunks; i += kBlock) {
        const int h = i / a.chunks, d = 8 * (i - h * a.chunks);
        *reinterpret_cast<u32x4 *>(a.k + to + h * a.head_stride + d) =
            *reinterpret_cast<const u32x4 *>(a.k_new + t * a.k_token + h * a.k_head + d);
        *reinterpret_cast<u32x4 *>(a.v + to + h * a.head_stride + d) =
            *reinterpret_cast<const u32x4 *>(a.v_new + t * a.v_token + h * a.v_head + d);
    }
}

// Rows that one block forks: a row's trips to memory follow one another, so a wave takes one row (us per
// call, one launch and two: 4 rows 2.6 and 4.6, 256 rows 38 and 8.7).
constexpr int64_t kFew = kPlan / kWave;

}  // namespace

// fork: [n][max_pages] rows and [n] lengths; extend: 4 words per row and 3 per
// page; compact: 2 per page
int64_t pages_work_bytes(const tam_pages &c, int64_t n) {
    return 4 * std::max(n * (c.max_pages + 1), 4 * n + 3 * c.num_pages);
}

hipError_t launch_pages_fork(const tam_pages &c, const int32_t *slots, const int32_t *parents, const int32_t *lengths,
                             int64_t n, void *work, hipStream_t s) {
    const Tables t = tables_of(c);
    int32_t *rows = static_cast<int32_t *>(work), *lens = rows + n * c.max_pages;
    if (n <= kFew) {
        hipLaunchKernelGGL(k_fork_few, dim3(1), dim3(kPlan), 0, s, t, slots, parents, lengths, n, rows, lens);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(k_fork_read, dim3((unsigned)n), dim3(kBlock), 0, s, t, slots, parents, lengths, rows, lens);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_fork_write, dim3((unsigned)n), dim3(kBlock), 0, s, t, slots, rows, lens);
    return hipGetLastError();
}

hipError_t launch_pages_extend(const tam_pages &c, const int32_t *slots, const int32_t *counts, int64_t n,
                               int32_t *info, void *work, hipStream_t s) {
    int32_t *p = static_cast<int32_t *>(work);
    const ExtendWork w{p, p + n, p + 2 * n, p + 3 * n, p + 4 * n, p + 4 * n + c.num_pages, p + 4 * n + 2 * c.num_pages};
    hipLaunchKernelGGL(n <= kPlan ? k_extend<true> : k_extend<false>, dim3(1), dim3(kPlan), 0, s, tables_of(c), slots, counts,
                       n, info, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.page_tokens == 1) return e;  // pages of one token are never partly filled
    return launch_copy(c, w.src, w.dst, n, s);
}

hipError_t launch_pages_compact(const tam_pages &c, int32_t *info, int32_t *moved, void *work, hipStream_t s) {
    int32_t *src = static_cast<int32_t *>(work), *dst = src + c.num_pages;
    hipLaunchKernelGGL(k_plan, dim3(1), dim3(kPlan), 0, s, tables_of(c), info, moved, src, dst);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t blocks = c.slots + copy_blocks(c, c.num_pages / 2);
    if (!blocks) return hipSuccess;
    hipLaunchKernelGGL(in_pieces(c) ? k_move<u32x4> : k_move<uint8_t>, dim3((unsigned)blocks), dim3(kBlock), 0, s, tables_of(c), moved,
                       pool_of(c), src, dst, c.num_pages / 2, info + 1);
    return hipGetLastError();
}

hipError_t launch_pages_store(const tam_chunk &c, const void *k_new, int64_t k_token, int64_t k_head,
                              const void *v_new, int64_t v_token, int64_t v_head, hipStream_t s) {
    const Store a{static_cast<uint16_t *>(c.k), static_cast<uint16_t *>(c.v), c.page_stride, c.head_stride,
                  c.token_stride, static_cast<const uint16_t *>(k_new), static_cast<const uint16_t *>(v_new),
                  k_token, k_head, v_token, v_head, c.table, c.length, c.offsets, c.slot_ids, c.table_stride, c.slots,
                  c.max_pages, c.num_pages, c.rows, c.tokens, __builtin_ctzll((unsigned long long)c.page_tokens),
                  (int32_t)c.kv_heads, (int32_t)(c.head_dim / 8)};
    hipLaunchKernelGGL(k_store, dim3((unsigned)c.tokens), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace tam
