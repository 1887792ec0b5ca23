// Operators on rows of class logits: what their entry points (logit_api.cpp) hand to their kernels (logprobs.hip, distill.hip).
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

// How rows go, and how they are cut into chunks of a workgroup each and what those need of the workspace.
enum class Way {
    sixteen,   // 16 lanes a row
    wave,      // a wave a row
    chunks,    // a workgroup a chunk
    row,       // a workgroup a row, chunk by chunk
    alone      // a workgroup of ALONE threads a row
};
constexpr uint32_t WAVE_VECS = 256;   // of a row that a wave holds by vectors
constexpr int ALONE = 1024;
struct RowCut {
    Way way;
    uint32_t nv;           // vectors of 16 bytes a thread of a chunk
    uint32_t chunks;       // of a row
    uint32_t chunk_vecs;   // vectors of a chunk, the last one's may be fewer
    uint32_t list_cap;     // room for candidates of the top alternatives, of a chunk
    uint32_t rows;         // of a launch
    size_t parts_bytes, lists_bytes;
};
RowCut cut_logprobs(int type, uint32_t classes, uint64_t rows, uint32_t top);
size_t logprobs_workspace(int type, uint32_t classes, uint64_t rows, uint32_t top);   // bytes
RowCut cut_distill(int type, uint32_t classes, uint64_t rows, uint32_t top, bool rest);
RowCut cut_gradient(const LogitRows &l);

struct Part;
// row0 to lists: set by the launcher, for each launch
struct LogprobsParams {
    LogitRows l;
    const int32_t *given;
    uint32_t n_given, top;
    float *logprob, *entropy;
    int32_t *top_class;
    float *top_logprob, *stats;
    uint64_t row0;
    uint32_t run;             // rows
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
    uint64_t row0;
    uint32_t run, chunks, chunk_vecs;
};

// Statistics of a row between the loss and its gradient.  logs == -infinity: the gradient is zero.
struct DistillStat {
    float m, logs;               // of all classes; m: as the logits' type holds it
    float rest_m, rest_logs;     // of those that are no entry (rest), else as m and logs
    float value_m, value_logs;   // q = exp(value_scale (value - value_m) - value_logs)
    float total, left;           // sum of q and q_rest; q_rest, 0 where only rounding leaves one and there is no class for it
};
static_assert(sizeof(DistillStat) == 32, "eight words a row");

struct DistillParams {
    LogitRows l;
    const int32_t *entry;
    const void *value;
    int32_t value_type;
    uint32_t top;
    float value_scale;
    int32_t rest;
    const float *weight;
    float *loss;
    DistillStat *stats;
    void *grad;
    uint64_t grad_stride;
    uint64_t row0;
    uint32_t run, chunks, chunk_vecs;
    Part *parts;
};

hipError_t launch_logprobs(LogprobsParams p, const RowCut &cut, void *workspace, hipStream_t st);
hipError_t launch_logprobs_grad(LogprobsGradParams p, hipStream_t st);

// Whether loss and gradient of rows of this shape are one launch, which needs neither a workspace nor the statistics.
bool distill_in_one(int type, uint32_t classes);
hipError_t launch_distill(DistillParams p, const RowCut &cut, void *workspace, hipStream_t st);   // the gradient too, if p.grad
hipError_t launch_distill_grad(DistillParams p, hipStream_t st);

}  // namespace isr
