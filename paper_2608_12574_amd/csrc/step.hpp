// Launchers of the decode step's operators beside the mask (adjust.hip,
// attend.hip, pages.hip) and what their C entry points (step_api.cpp) share.
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
hipError_t launch_attend(const tam_chunk &c, const Queries &q, void *work, hipStream_t s);
int64_t attend_work_bytes(const tam_chunk &c, int64_t heads);

}  // namespace tam
