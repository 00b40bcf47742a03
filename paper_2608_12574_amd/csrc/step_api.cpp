// C entry points of the decode step's operators beside the mask: argument checks
// and launches.  (tam_adjust_logits, which takes a handle, is in tam_api.cpp.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <array>
#include <climits>
#include <cstdint>

#include "step.hpp"

namespace {

using tam::api_fail;

#define STEP_HIP(expr)                                                                                    \
    do {                                                                                                  \
        const hipError_t e_ = (expr);                                                                     \
        if (e_ != hipSuccess) return api_fail(TAM_E_DEVICE, std::string(#expr) + ": " + hipGetErrorString(e_)); \
    } while (0)

bool power_of_two(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }
bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A launch has fewer than 2^32 threads along an axis: blocks of 256.
constexpr int64_t kMostBlocks = (1 << 24) - 1;

struct Axis {
    int64_t count, stride;
};

// Whether vectors of `size` lie apart: each axis, in the order of the strides, steps over all that those before it
// span.  (What a launch writes, it must not write twice.)
template <size_t N>
bool apart(int64_t size, std::array<Axis, N> axes) {
    for (Axis &x : axes) x.stride = x.stride < 0 ? (x.stride == INT64_MIN ? INT64_MAX : -x.stride) : x.stride;
    std::sort(axes.begin(), axes.end(), [](const Axis &x, const Axis &y) { return x.stride < y.stride; });
    __int128 span = size;
    for (const Axis &x : axes) {
        if (x.count < 2) continue;
        if (x.stride < span) return false;
        span += (__int128)(x.count - 1) * x.stride;
    }
    return true;
}

// null: fine, else what is wrong
const char *tables_wrong(const void *table, const void *length, int64_t slots, int64_t max_pages, int64_t stride,
                         int64_t pages, int64_t page_tokens) {
    if (slots < 0 || slots >= INT32_MAX) return "slots must be in 0 .. 2^31 - 2";
    if (pages < 1 || pages >= INT32_MAX) return "num_pages must be in 1 .. 2^31 - 2";
    if (!power_of_two(page_tokens) || page_tokens > 65536) return "page_tokens must be a power of two, at most 65536";
    if (max_pages < 0 || max_pages > (1 << 30) / page_tokens)
        return "max_pages must be >= 0, and max_pages * page_tokens at most 2^30";
    if (stride < max_pages) return "table_stride must be >= max_pages";
    if (slots > 0 && (!length || (max_pages > 0 && !table))) return "null table or length";
    if (!aligned(table, 4) || !aligned(length, 4)) return "table and length must be 4-byte aligned";
    return nullptr;
}

const char *pages_wrong(const tam_pages *c) {
    if (!c) return "null cache";
    if (const char *w = tables_wrong(c->table, c->length, c->slots, c->max_pages, c->table_stride, c->num_pages,
                                     c->page_tokens))
        return w;
    if (!c->refs || !aligned(c->refs, 4)) return "refs is null or not 4-byte aligned";
    if (c->planes < 0 || c->planes > 65536 || c->page_bytes < 0) return "planes must be in 0 .. 65536, page_bytes >= 0";
    if (c->planes > 0 && c->page_bytes > 0) {
        if (!c->data) return "null data";
        if (c->page_stride < c->page_bytes || c->plane_stride < 0)
            return "page_stride must be >= page_bytes and plane_stride >= 0";
        if (!apart<2>(c->page_bytes, {{{c->planes, c->plane_stride}, {c->num_pages, c->page_stride}}})) return "pages overlap";
    }
    return nullptr;
}

const char *rows_wrong(const tam_pages *c, int64_t n) {
    if (n < 0 || n > c->slots) return "n must be in 0 .. slots";
    return nullptr;
}

// `plane`: the call reads or writes k and v
const char *chunk_wrong(const tam_chunk *c, bool plane = true) {
    if (!c) return "null chunk";
    if (const char *w = tables_wrong(c->table, c->length, c->slots, c->max_pages, c->table_stride, c->num_pages,
                                     c->page_tokens))
        return w;
    if (c->dtype != TAM_DTYPE_BF16 && c->dtype != TAM_DTYPE_FP16) return "dtype must be BF16 or FP16";
    if (c->kv_heads < 1 || c->kv_heads > 65535) return "kv_heads must be in 1 .. 65535";
    if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return "head_dim must be a multiple of 8 in 8 .. 128";
    if (c->rows < 0 || c->rows >= INT32_MAX || c->tokens < 0 || c->tokens >= INT32_MAX)
        return "rows and tokens must be in 0 .. 2^31 - 2";
    if (!c->slot_ids && c->rows > c->slots) return "rows must be <= slots without slot_ids";
    if (c->longest < 0) return "longest must be >= 0";
    if (plane && (!c->k || !c->v)) return "null k or v";
    if ((plane && (!aligned(c->k, 16) || !aligned(c->v, 16))) || c->page_stride % 8 || c->head_stride % 8 || c->token_stride % 8)
        return "k and v must be 16-byte aligned and their strides multiples of 8";
    if (c->page_stride < 0 || c->head_stride < 0 || c->token_stride < 0) return "strides must be >= 0";
    if (!aligned(c->offsets, 4) || !aligned(c->slot_ids, 4)) return "offsets and slot_ids must be 4-byte aligned";
    return nullptr;
}

const char *store_wrong(const tam_chunk *c, const void *k_new, int64_t k_token, int64_t k_head, const void *v_new,
                        int64_t v_token, int64_t v_head) {
    if (const char *w = chunk_wrong(c)) return w;
    if (c->tokens > kMostBlocks) return "tokens must be below 2^24";
    if (c->tokens > 0 && (!k_new || !v_new)) return "null device pointer";
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || k_token % 8 || k_head % 8 || v_token % 8 || v_head % 8)
        return "k_new and v_new must be 16-byte aligned and their strides multiples of 8";
    if (!apart<3>(c->head_dim, {{{c->num_pages, c->page_stride}, {c->kv_heads, c->head_stride}, {c->page_tokens, c->token_stride}}}))
        return "the pool's vectors overlap";
    return nullptr;
}

const char *top_wrong(int dtype, int64_t B, int64_t V, int64_t k) {
    if (dtype != TAM_DTYPE_FP32 && dtype != TAM_DTYPE_BF16) return "dtype must be FP32 or BF16";
    if (B < 0 || B > TAM_MAX_TOP_ROWS) return "B must be in 0 .. TAM_MAX_TOP_ROWS";
    if (V < 1 || V > TAM_MAX_TOP_COLUMNS) return "V must be in 1 .. TAM_MAX_TOP_COLUMNS";
    if (k < 1 || k > TAM_MAX_TOP) return "k must be in 1 .. TAM_MAX_TOP";
    return nullptr;
}

tam_status attend(const tam_chunk *c, const tam::Queries &x, const tam::Seen &seen, void *work, void *stream) {
    const char *w = chunk_wrong(c);
    if (!w && (x.heads < 1 || x.heads > 65535 || x.heads % c->kv_heads)) w = "heads must be a multiple of kv_heads, at most 65535";
    if (!w && !(x.scale > 0.f && x.scale < 1e30f)) w = "scale must be positive and finite";
    if (!w && c->tokens > 0 && (!x.q || !x.out)) w = "null device pointer";
    if (!w && c->tokens > 0 && !work && tam::attend_work_bytes(*c, x.heads) > 0) w = "null work";
    if (!w && (!aligned(x.q, 16) || !aligned(x.out, 16) || x.q_token % 8 || x.q_head % 8 || x.out_token % 8 || x.out_head % 8))
        w = "q and out must be 16-byte aligned and their strides multiples of 8";
    if (!w && !apart<2>(c->head_dim, {{{c->tokens, x.out_token}, {x.heads, x.out_head}}})) w = "out's vectors overlap";
    if (!w && (!aligned(x.lse, 4) || !aligned(work, 16))) w = "lse must be 4-byte and work 16-byte aligned";
    if (w) return api_fail(TAM_E_INVAL, w);
    if (c->tokens == 0 || c->rows == 0) return TAM_OK;
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_attend(*c, x, seen, work, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

}  // namespace

extern "C" {

int64_t tam_pages_work(const tam_pages *c, int64_t n) {
    tam::api_begin();
    const char *w = pages_wrong(c);
    if (!w) w = rows_wrong(c, n);
    if (w) return api_fail(TAM_E_INVAL, w), -1;
    return tam::pages_work_bytes(*c, n);
}

tam_status tam_pages_fork(const tam_pages *c, const int32_t *slots, const int32_t *parents, const int32_t *lengths,
                          int64_t n, void *work, void *stream) {
    tam::api_begin();
    const char *w = pages_wrong(c);
    if (!w) w = rows_wrong(c, n);
    if (!w && n > kMostBlocks) w = "n must be below 2^24";
    if (!w && n > 0 && (!slots || !parents || !work)) w = "null device pointer";
    if (!w && !aligned(work, 16)) w = "work must be 16-byte aligned";
    if (w) return api_fail(TAM_E_INVAL, w);
    if (n == 0) return TAM_OK;
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_pages_fork(*c, slots, parents, lengths, n, work, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

tam_status tam_pages_extend(const tam_pages *c, const int32_t *slots, const int32_t *counts, int64_t n, int32_t *info,
                            void *work, void *stream) {
    tam::api_begin();
    const char *w = pages_wrong(c);
    if (!w) w = rows_wrong(c, n);
    if (!w && ((n > 0 && (!slots || !counts)) || !info || !work)) w = "null device pointer";
    if (!w && !aligned(work, 16)) w = "work must be 16-byte aligned";
    if (w) return api_fail(TAM_E_INVAL, w);
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_pages_extend(*c, slots, counts, n, info, work, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

tam_status tam_pages_compact(const tam_pages *c, int32_t *info, int32_t *moved, void *work, void *stream) {
    tam::api_begin();
    const char *w = pages_wrong(c);
    if (!w && c->slots > kMostBlocks - 4096) w = "slots must be below 2^24 - 4096";  // a block each, beside those that copy pages
    if (!w && (!info || !moved || !work)) w = "null device pointer";
    if (!w && !aligned(work, 16)) w = "work must be 16-byte aligned";
    if (w) return api_fail(TAM_E_INVAL, w);
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_pages_compact(*c, info, moved, work, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

tam_status tam_pages_store(const tam_chunk *c, const void *k_new, int64_t k_token, int64_t k_head, const void *v_new,
                           int64_t v_token, int64_t v_head, void *stream) {
    tam::api_begin();
    const char *w = store_wrong(c, k_new, k_token, k_head, v_new, v_token, v_head);
    if (w) return api_fail(TAM_E_INVAL, w);
    if (c->tokens == 0 || c->rows == 0) return TAM_OK;
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_pages_store(*c, k_new, k_token, k_head, v_new, v_token, v_head,
                                     static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

int64_t tam_attend_work(const tam_chunk *c, int64_t heads) {
    tam::api_begin();
    const char *w = chunk_wrong(c);
    if (!w && (heads < 1 || heads > 65535 || heads % c->kv_heads)) w = "heads must be a multiple of kv_heads, at most 65535";
    if (w) return api_fail(TAM_E_INVAL, w), -1;
    return tam::attend_work_bytes(*c, heads);
}

tam_status tam_attend(const tam_chunk *c, const void *q, int64_t q_token, int64_t q_head, int64_t heads, float scale,
                      void *out, int64_t out_token, int64_t out_head, float *lse, void *work, void *stream) {
    tam::api_begin();
    const tam::Queries queries{q, q_token, q_head, out, out_token, out_head, lse, heads, scale};
    return attend(c, queries, tam::Seen{nullptr, 0, 0}, work, stream);
}

tam_status tam_attend_seen(const tam_chunk *c, const void *q, int64_t q_token, int64_t q_head, int64_t heads, float scale,
                           const uint64_t *seen, int64_t words, int64_t seen_stride, void *out, int64_t out_token,
                           int64_t out_head, float *lse, void *work, void *stream) {
    tam::api_begin();
    if ((c && c->tokens > 0 && !seen) || !aligned(seen, 8)) return api_fail(TAM_E_INVAL, "seen is null or not 8-byte aligned");
    if (words < 1 || words > INT32_MAX || seen_stride < words) return api_fail(TAM_E_INVAL, "words must be in 1 .. 2^31 - 1 and seen_stride >= words");
    const tam::Queries queries{q, q_token, q_head, out, out_token, out_head, lse, heads, scale};
    return attend(c, queries, tam::Seen{seen, words, seen_stride}, work, stream);
}

tam_status tam_tree_masks(const int32_t *parents, const int32_t *offsets, int64_t rows, int64_t tokens, uint64_t *seen,
                          int64_t words, int32_t *depth, void *stream) {
    tam::api_begin();
    if (rows < 0 || rows > (1 << 23) || tokens < 0 || tokens >= INT32_MAX)
        return api_fail(TAM_E_INVAL, "rows must be in 0 .. 2^23, tokens in 0 .. 2^31 - 2");
    if (words < 1 || words > (1 << 25)) return api_fail(TAM_E_INVAL, "words must be in 1 .. 2^25");
    if (tokens > 0 && (!parents || !seen || !depth)) return api_fail(TAM_E_INVAL, "null device pointer");
    if (!aligned(parents, 4) || !aligned(offsets, 4) || !aligned(depth, 4) || !aligned(seen, 8))
        return api_fail(TAM_E_INVAL, "parents, offsets and depth must be 4-byte and seen 8-byte aligned");
    if (tokens == 0 || rows == 0) return TAM_OK;
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_tree_masks(parents, offsets, rows, tokens, seen, words, depth, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

tam_status tam_pages_append(const tam_chunk *c, const tam_rotation *r, const void *k_new, int64_t k_token, int64_t k_head,
                            const void *v_new, int64_t v_token, int64_t v_head, const void *q, int64_t q_token, int64_t q_head,
                            int64_t heads, void *out, int64_t out_token, int64_t out_head, void *stream) {
    tam::api_begin();
    const char *w = store_wrong(c, k_new, k_token, k_head, v_new, v_token, v_head);
    if (!w && !r) w = "null rotation";
    if (!w && (r->pairs < 0 || r->pairs > c->head_dim / 2 || r->pairs % 4)) w = "pairs must be a multiple of 4, at most head_dim / 2";
    if (!w && r->adjacent != 0 && r->adjacent != 1) w = "adjacent must be 0 or 1";
    if (!w && r->pairs > 0 && !r->frequencies) w = "null frequencies";
    if (!w && (!aligned(r->frequencies, 4) || !aligned(r->depth, 4))) w = "frequencies and depth must be 4-byte aligned";
    if (!w && (heads < 0 || heads > 65535)) w = "heads must be in 0 .. 65535";
    if (!w && heads > 0) {
        if (c->tokens > 0 && (!q || !out)) w = "null device pointer";
        if (!w && (!aligned(q, 16) || !aligned(out, 16) || q_token % 8 || q_head % 8 || out_token % 8 || out_head % 8))
            w = "q and out must be 16-byte aligned and their strides multiples of 8";
        if (!w && !apart<2>(c->head_dim, {{{c->tokens, out_token}, {heads, out_head}}})) w = "out's vectors overlap";
    }
    if (w) return api_fail(TAM_E_INVAL, w);
    if (c->tokens == 0 || c->rows == 0) return TAM_OK;
    STEP_HIP(hipGetLastError());
    const tam::Fresh fresh{k_new, k_token, k_head, v_new, v_token, v_head, q, q_token, q_head, heads, out, out_token, out_head};
    STEP_HIP(tam::launch_pages_append(*c, *r, fresh, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

int64_t tam_pages_accept_work(const tam_chunk *n) {
    tam::api_begin();
    if (const char *w = chunk_wrong(n, false)) return api_fail(TAM_E_INVAL, w), -1;
    return tam::accept_work_bytes(*n);
}

tam_status tam_pages_accept(const tam_pages *c, const tam_chunk *n, const int32_t *tokens, const int32_t *picks,
                            const int32_t *parents, int32_t *path, int32_t *count, int32_t *last, void *work, void *stream) {
    tam::api_begin();
    const char *w = pages_wrong(c);
    if (!w) w = chunk_wrong(n, false);
    if (!w && (n->table != c->table || n->length != c->length || n->slots != c->slots || n->max_pages != c->max_pages ||
               n->table_stride != c->table_stride || n->num_pages != c->num_pages || n->page_tokens != c->page_tokens))
        w = "the chunk's tables are not the cache's";
    if (!w && n->rows > c->slots) w = "rows must be <= slots";
    if (!w && n->rows > kMostBlocks) w = "rows must be below 2^24";
    if (!w && !apart<2>(n->head_dim, {{{n->kv_heads, n->head_stride}, {n->page_tokens, n->token_stride}}})) w = "a page's vectors overlap";
    if (!w && c->planes > 0) {
        // (strides of 2^62 and more would wrap below; a page cannot be that large)
        if (c->page_bytes == 0 || (__int128)(n->kv_heads - 1) * n->head_stride + (__int128)(n->page_tokens - 1) * n->token_stride + n->head_dim > c->page_bytes / 2)
            w = "the chunk's vectors do not fit the cache's pages";
        if (!w && (!aligned(c->data, 16) || c->plane_stride % 16 || c->page_stride % 16)) w = "data must be 16-byte aligned and its strides multiples of 16";
    }
    if (!w && n->tokens > 0 && (!tokens || !picks || !parents || !path || !work)) w = "null device pointer";
    if (!w && n->rows > 0 && (!count || !last || !work)) w = "null device pointer";
    if (!w && (!aligned(tokens, 4) || !aligned(picks, 4) || !aligned(parents, 4) || !aligned(path, 4) || !aligned(count, 4) || !aligned(last, 4) || !aligned(work, 16)))
        w = "the lists must be 4-byte and work 16-byte aligned";
    if (w) return api_fail(TAM_E_INVAL, w);
    if (n->rows == 0) return TAM_OK;
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_pages_accept(*c, *n, tokens, picks, parents, path, count, last, work, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

int64_t tam_top_tokens_work(int64_t B, int64_t V, int64_t k, int dtype) {
    tam::api_begin();
    if (const char *w = top_wrong(dtype, B, V, k)) return api_fail(TAM_E_INVAL, w), -1;
    return tam::top_work_bytes(B, V, (int)k, dtype);
}

tam_status tam_top_tokens(const void *logits, int dtype, int64_t B, int64_t V, int64_t row_stride, int64_t k, int32_t *tokens,
                          float *logprobs, float *lse, void *work, void *stream) {
    tam::api_begin();
    const char *w = top_wrong(dtype, B, V, k);
    if (!w && row_stride < 0) w = "row_stride must be >= 0";
    if (!w && B > 0 && (!logits || !tokens || !logprobs)) w = "null device pointer";
    if (!w && B > 0 && !work && tam::top_work_bytes(B, V, (int)k, dtype) > 0) w = "null work";
    if (!w && (!aligned(logits, dtype == TAM_DTYPE_FP32 ? 4 : 2) || !aligned(tokens, 4) || !aligned(logprobs, 4) || !aligned(lse, 4) || !aligned(work, 16)))
        w = "logits, tokens, logprobs and lse must be aligned to their elements, work to 16 bytes";
    if (w) return api_fail(TAM_E_INVAL, w);
    if (B == 0) return TAM_OK;
    STEP_HIP(hipGetLastError());
    STEP_HIP(tam::launch_top_tokens(logits, dtype, B, V, row_stride, (int)k, tokens, logprobs, lse, work, static_cast<hipStream_t>(stream)));
    return TAM_OK;
}

}  // extern "C"
