// Launchers of the decode step's operators beside the mask (adjust.hip, append.hip,
// attend.hip, pages.hip, top.hip, trees.hip) and what their C entry points (step_api.cpp) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "tam.h"

namespace tam {

void api_begin();                                           // clears the thread's message
tam_status api_fail(tam_status st, const std::string &msg);  // sets it

// edits and mask rows; rows null: every token valid
hipError_t launch_adjust(const uint64_t *rows, int64_t num_rows, int64_t rows_stride, const int32_t *ids,
                         const tam_edits &e, int64_t B, int64_t V, void *logits, int dtype, int64_t row_stride,
                         hipStream_t s);

hipError_t launch_pages_fork(const tam_pages &c, const int32_t *slots, const int32_t *parents, const int32_t *lengths,
                             int64_t n, void *work, hipStream_t s);
hipError_t launch_pages_extend(const tam_pages &c, const int32_t *slots, const int32_t *counts, int64_t n,
                               int32_t *info, void *work, hipStream_t s);
hipError_t launch_pages_compact(const tam_pages &c, int32_t *info, int32_t *moved, void *work, hipStream_t s);
int64_t pages_work_bytes(const tam_pages &c, int64_t n);

hipError_t launch_pages_store(const tam_chunk &c, const void *k_new, int64_t k_token, int64_t k_head,
                              const void *v_new, int64_t v_token, int64_t v_head, hipStream_t s);

// what tam_attend is called with beside the chunk
struct Queries {
    const void *q;
    int64_t q_token, q_head;
    void *out;
    int64_t out_token, out_head;
    float *lse;
    int64_t heads;
    float scale;
};
// which of its row's tokens each one sees (tam_attend_seen); bits null: those up to itself
struct Seen {
    const uint64_t *bits;
    int64_t words, stride;
};
hipError_t launch_attend(const tam_chunk &c, const Queries &q, const Seen &seen, void *work, hipStream_t s);
int64_t attend_work_bytes(const tam_chunk &c, int64_t heads);

// what tam_pages_append is called with beside the chunk and the rotation
struct Fresh {
    const void *k;
    int64_t k_token, k_head;
    const void *v;
    int64_t v_token, v_head;
    const void *q;
    int64_t q_token, q_head, heads;
    void *out;
    int64_t out_token, out_head;
};
hipError_t launch_pages_append(const tam_chunk &c, const tam_rotation &r, const Fresh &x, hipStream_t s);

hipError_t launch_tree_masks(const int32_t *parents, const int32_t *offsets, int64_t rows, int64_t tokens, uint64_t *seen,
                             int64_t words, int32_t *depth, hipStream_t s);
hipError_t launch_pages_accept(const tam_pages &c, const tam_chunk &n, const int32_t *tokens, const int32_t *picks,
                               const int32_t *parents, int32_t *path, int32_t *count, int32_t *last, void *work, hipStream_t s);
int64_t accept_work_bytes(const tam_chunk &n);

hipError_t launch_top_tokens(const void *logits, int dtype, int64_t B, int64_t V, int64_t row_stride, int k, int32_t *tokens,
                             float *logprobs, float *lse, void *work, hipStream_t s);
int64_t top_work_bytes(int64_t B, int64_t V, int k, int dtype);

}  // namespace tam
