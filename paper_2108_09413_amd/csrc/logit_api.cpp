// Entry points of the operators on rows of class logits: arguments are checked here, on the host, and the kernels
// rely on it.  Nothing is allocated, copied or waited for.
#include <initializer_list>

#include "logit_rows.h"

namespace {

using namespace isr;

constexpr uint32_t MAX_CLASSES = 1u << 24;

size_t element_bytes(int type) { return type == ISR_F32 || type == ISR_I32 ? 4 : 2; }
bool aligned(const void *p, size_t n) { return (uintptr_t)p % n == 0; }
bool usable_scale(float s) { return s >= 1e-30f && s <= 1e30f; }   // its product with log2 e too is a normal number; not NaN

// shapes and type, what the size of a workspace depends on
bool valid_shape(const isr_logits *l) {
    return l && l->type >= ISR_F32 && l->type <= ISR_I32 && l->classes >= 1 && l->classes <= MAX_CLASSES && l->rows <= 0x7FFFFFFF;
}

// elements that rows of a stride span, 0 where that passes 2^60
uint64_t span(uint64_t rows, uint64_t stride, uint32_t classes) {
    if (rows == 0) return 0;
    if (rows > 1 && stride > ((1ull << 60) - classes) / (rows - 1)) return 0;
    return (rows - 1) * stride + classes;
}

bool valid_logits(const isr_logits *l) {
    if (!valid_shape(l) || !usable_scale(l->scale) || l->row_stride < l->classes) return false;
    return l->rows == 0 || (l->data_device && aligned(l->data_device, element_bytes(l->type)) && span(l->rows, l->row_stride, l->classes));
}

bool valid_teacher(const isr_teacher *t) {
    return t && t->type >= ISR_F32 && t->type <= ISR_F16 && t->top >= 1 && t->top <= ISR_MAX_GIVEN && usable_scale(t->scale) &&
           (t->rest == 0 || t->rest == 1);
}

bool teacher_data(const isr_teacher *t) {
    return t->class_device && t->logit_device && aligned(t->class_device, 4) && aligned(t->logit_device, element_bytes(t->type));
}

// a gradient's rows: their own memory, or the logits' with the logits' type and stride
bool valid_grad(const isr_logits *l, const void *grad, uint64_t stride) {
    const size_t bytes = l->type == ISR_I32 ? 4 : element_bytes(l->type);
    if (!grad || !aligned(grad, bytes) || stride < l->classes || !span(l->rows, stride, l->classes)) return false;
    if (grad == l->data_device) return stride == l->row_stride && l->type != ISR_I32;
    const uintptr_t g = (uintptr_t)grad, x = (uintptr_t)l->data_device;
    const uint64_t gb = span(l->rows, stride, l->classes) * bytes, xb = span(l->rows, l->row_stride, l->classes) * element_bytes(l->type);
    return g >= x ? g - x >= xb : x - g >= gb;
}

bool all_aligned(std::initializer_list<const void *> words) {
    for (const void *p : words)
        if (!aligned(p, 4)) return false;
    return true;
}

LogitRows rows_of(const isr_logits *l) { return {l->data_device, l->type, l->classes, l->rows, l->row_stride, l->scale}; }

DistillParams distill_params(const isr_logits *l, const isr_teacher *t, const float *weight, float *loss, const void *stats, void *grad,
                             uint64_t grad_stride) {
    DistillParams p{};
    p.l = rows_of(l);
    p.entry = t->class_device; p.value = t->logit_device; p.value_type = t->type; p.top = t->top; p.value_scale = t->scale; p.rest = t->rest;
    p.weight = weight; p.loss = loss; p.stats = (DistillStat *)stats; p.grad = grad; p.grad_stride = grad_stride;
    return p;
}

int status(hipError_t e) {
    if (e == hipSuccess) return ISR_OK;
    set_last_device_error((int)e);
    return ISR_ERR_DEVICE;
}

}  // namespace

extern "C" {

size_t isr_logprobs_workspace_bytes(const isr_logits *l, uint32_t top) {
    if (!valid_shape(l) || l->rows == 0 || top > ISR_MAX_TOP) return 0;
    return logprobs_workspace(l->type, l->classes, l->rows, top);
}

int isr_logprobs(const isr_logits *l, const int32_t *given_device, uint32_t given, uint32_t top, float *logprob_device,
                 float *entropy_device, int32_t *top_class_device, float *top_logprob_device, float *stats_device,
                 void *workspace_device, size_t workspace_bytes, void *hip_stream) {
    if (!valid_logits(l) || given > ISR_MAX_GIVEN || top > ISR_MAX_TOP || top > l->classes) return ISR_ERR_ARG;
    if (!given && !top && !entropy_device && !stats_device) return ISR_ERR_ARG;
    if (l->rows == 0) return ISR_OK;
    if (given && (!given_device || !logprob_device)) return ISR_ERR_ARG;
    if (top && (!top_class_device || !top_logprob_device)) return ISR_ERR_ARG;
    if (!all_aligned({given_device, logprob_device, entropy_device, top_class_device, top_logprob_device, stats_device})) return ISR_ERR_ARG;
    const RowCut cut = cut_logprobs(l->type, l->classes, l->rows, top);
    const size_t need = cut.parts_bytes + cut.lists_bytes;
    if (need && (!workspace_device || workspace_bytes < need)) return ISR_ERR_WORKSPACE;
    if (need && !aligned(workspace_device, 16)) return ISR_ERR_ARG;
    LogprobsParams p{};
    p.l = rows_of(l);
    p.given = given_device; p.n_given = given; p.top = top;
    p.logprob = logprob_device; p.entropy = entropy_device; p.top_class = top_class_device; p.top_logprob = top_logprob_device; p.stats = stats_device;
    return status(launch_logprobs(p, cut, workspace_device, (hipStream_t)hip_stream));
}

int isr_logprobs_grad(const isr_logits *l, const int32_t *given_device, uint32_t given, const float *grad_logprob_device,
                      const float *entropy_device, const float *grad_entropy_device, const float *stats_device,
                      void *grad_logits_device, uint64_t grad_row_stride, void *hip_stream) {
    if (!valid_logits(l) || given > ISR_MAX_GIVEN) return ISR_ERR_ARG;
    if (!given && !grad_entropy_device) return ISR_ERR_ARG;
    if (!entropy_device != !grad_entropy_device) return ISR_ERR_ARG;
    if (l->rows == 0) return ISR_OK;
    if (given && (!given_device || !grad_logprob_device)) return ISR_ERR_ARG;
    if (!stats_device || !all_aligned({given_device, grad_logprob_device, entropy_device, grad_entropy_device, stats_device})) return ISR_ERR_ARG;
    if (!valid_grad(l, grad_logits_device, grad_row_stride)) return ISR_ERR_ARG;
    LogprobsGradParams p{};
    p.l = rows_of(l);
    p.given = given_device; p.n_given = given;
    p.up_logprob = grad_logprob_device; p.entropy = entropy_device; p.up_entropy = grad_entropy_device; p.stats = stats_device;
    p.grad = grad_logits_device; p.grad_stride = grad_row_stride;
    return status(launch_logprobs_grad(p, (hipStream_t)hip_stream));
}

// What the chunks of rows leave and, for a gradient behind them, the rows' statistics where the caller keeps none.
size_t isr_distill_workspace_bytes(const isr_logits *l, const isr_teacher *t) {
    if (!valid_shape(l) || !valid_teacher(t) || l->rows == 0) return 0;
    return cut_distill(l->type, l->classes, l->rows, t->top, t->rest != 0).parts_bytes + (distill_in_one(l->type, l->classes) ? 0 : l->rows * sizeof(DistillStat));
}

int isr_distill(const isr_logits *l, const isr_teacher *t, const float *row_weight_device, float *loss_device, float *stats_device,
                void *grad_logits_device, uint64_t grad_row_stride, void *workspace_device, size_t workspace_bytes, void *hip_stream) {
    if (!valid_logits(l) || !valid_teacher(t)) return ISR_ERR_ARG;
    if (l->rows == 0) return ISR_OK;
    if (!teacher_data(t) || !loss_device || !all_aligned({row_weight_device, loss_device, stats_device})) return ISR_ERR_ARG;
    if (grad_logits_device && !valid_grad(l, grad_logits_device, grad_row_stride)) return ISR_ERR_ARG;
    const size_t need = isr_distill_workspace_bytes(l, t);
    if (need && (!workspace_device || workspace_bytes < need)) return ISR_ERR_WORKSPACE;
    if (need && !aligned(workspace_device, 16)) return ISR_ERR_ARG;
    const RowCut cut = cut_distill(l->type, l->classes, l->rows, t->top, t->rest != 0);
    void *stats = stats_device;
    if (!stats && grad_logits_device && !distill_in_one(l->type, l->classes)) stats = (uint8_t *)workspace_device + cut.parts_bytes;
    const DistillParams p = distill_params(l, t, row_weight_device, loss_device, stats, grad_logits_device, grad_row_stride);
    return status(launch_distill(p, cut, workspace_device, (hipStream_t)hip_stream));
}

int isr_distill_grad(const isr_logits *l, const isr_teacher *t, const float *row_weight_device, const float *stats_device,
                     void *grad_logits_device, uint64_t grad_row_stride, void *hip_stream) {
    if (!valid_logits(l) || !valid_teacher(t)) return ISR_ERR_ARG;
    if (l->rows == 0) return ISR_OK;
    if (!teacher_data(t) || !stats_device || !all_aligned({row_weight_device, stats_device})) return ISR_ERR_ARG;
    if (!valid_grad(l, grad_logits_device, grad_row_stride)) return ISR_ERR_ARG;
    return status(launch_distill_grad(distill_params(l, t, row_weight_device, nullptr, stats_device, grad_logits_device, grad_row_stride),
                                      (hipStream_t)hip_stream));
}

}  // extern "C"
