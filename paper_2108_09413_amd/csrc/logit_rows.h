// Operators on rows of class logits: what their entry points (logit_api.cpp) hand to their kernels (logit_rows.hip).
#pragma once
#include "isr_internal.h"

namespace isr {

struct LogitRows {
    const void *x;
    int32_t type;
    uint32_t classes;
    uint64_t rows, stride;
    float scale;
};

// How rows are cut into chunks of a workgroup each (cut_rows), and what the chunks need of the workspace.
struct RowCut {
    uint32_t nv;           // vectors of 16 bytes a thread
    uint32_t chunks;       // of a row
    uint32_t chunk_vecs;   // vectors of a chunk, the last one's may be fewer
    uint32_t list_cap;     // room for candidates of the top alternatives, of a chunk
    uint32_t rows;         // of a launch
    size_t parts_bytes, lists_bytes;
};
RowCut cut_rows(int type, uint32_t classes, uint64_t rows, uint32_t top);

struct Part;
struct LogprobsParams {
    LogitRows l;
    const int32_t *given;
    uint32_t n_given, top;
    float *logprob, *entropy;
    int32_t *top_class;
    float *top_logprob, *stats;
    // set by the launcher
    uint64_t row0;
    uint32_t chunks, chunk_vecs, list_cap;
    Part *parts;
    uint2 *lists;
};

struct LogprobsGradParams {
    LogitRows l;
    const int32_t *given;
    uint32_t n_given;
    const float *up_logprob, *entropy, *up_entropy, *stats;
    void *grad;
    uint64_t grad_stride;
    // set by the launcher
    uint64_t row0;
    uint32_t chunks, chunk_vecs;
};

struct DistillParams {
    LogitRows l;
    const int32_t *entry;
    const void *value;
    int32_t value_type;
    uint32_t top;
    float value_scale;
    int32_t rest;
    const float *weight;
    float *loss, *stats;      // stats: [rows][8], DistillStat
    void *grad;
    uint64_t grad_stride;
    // set by the launcher
    uint64_t row0;
    uint32_t chunks, chunk_vecs;
    Part *parts;
};

hipError_t launch_logprobs(LogprobsParams p, const RowCut &cut, void *workspace, hipStream_t st);
hipError_t launch_logprobs_grad(LogprobsGradParams p, hipStream_t st);
hipError_t launch_distill(DistillParams p, RowCut cut, void *workspace, hipStream_t st);   // and the gradient, if p.grad
hipError_t launch_distill_grad(DistillParams p, hipStream_t st);

}  // namespace isr
