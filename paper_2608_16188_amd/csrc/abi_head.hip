// extern "C" entry points of vmoe_head.h: argument validation, then launches.
#include <math.h>

#include "../../include/vmoe_head.h"
#include "common.h"

namespace vmoe {

// Launchers (head_loss.hip).
size_t head_saved_bytes(const vmoe_head_shape& s);
size_t head_fwd_workspace_bytes(const vmoe_head_shape& s);
size_t head_bwd_workspace_bytes(const vmoe_head_shape& s);
vmoe_status head_fwd_launch(const vmoe_head_shape& s, const void* x, const void* weight,
                            const void* bias, const int32_t* labels, const int32_t* teacher_idx,
                            const float* teacher_logits, const float* row_weight, float* losses,
                            float* row_losses, void* saved, void* ws, hipStream_t st);
vmoe_status head_bwd_launch(const vmoe_head_shape& s, const void* weight, const void* saved,
                            float w_label, float w_teacher, void* dx, void* dweight, void* dbias,
                            void* ws, hipStream_t st);

namespace {

constexpr int kMaxRowBytes = 1 << 22;  // N times an element's: a piece of 256 classes within 1 GiB
constexpr int kMaxClasses = 1 << 21, kMaxWidth = 1 << 16;
constexpr long long kMaxTokenBytes = 1LL << 31;  // N d: 32-bit offsets
constexpr long long kMaxLogits = 1LL << 36;   // N V: threads of one launch
constexpr float kMaxTemperature = 1024.0f;

vmoe_status check_shape(const vmoe_head_shape* s) {
    if (!s || s->n_rows < 0 || s->d_model < 8 || s->d_model % 8 != 0 || s->n_classes < 1)
        return VMOE_ERR_INVALID_ARG;
    if (s->n_teacher < 0 || s->n_teacher > VMOE_HEAD_MAX_TEACHER || s->reserved != 0)
        return VMOE_ERR_INVALID_ARG;
    if (s->dtype != VMOE_F32 && s->dtype != VMOE_BF16) return VMOE_ERR_INVALID_ARG;
    if (s->reduction != VMOE_REDUCE_MEAN && s->reduction != VMOE_REDUCE_SUM)
        return VMOE_ERR_INVALID_ARG;
    if (!(s->temperature >= 1.0f / kMaxTemperature && s->temperature <= kMaxTemperature))
        return VMOE_ERR_INVALID_ARG;
    const long long n = s->n_rows, size = s->dtype == VMOE_BF16 ? 2 : 4;
    if (n * size > kMaxRowBytes || s->n_classes > kMaxClasses || s->d_model > kMaxWidth ||
        n * s->d_model * size >= kMaxTokenBytes || n * s->n_classes >= kMaxLogits)
        return VMOE_ERR_UNSUPPORTED;
    return VMOE_OK;
}

bool dev(const void* p) { return p != nullptr && aligned16(p); }
bool opt(const void* p) { return p == nullptr || aligned16(p); }
vmoe_status need(bool ok) { return ok ? VMOE_OK : VMOE_ERR_INVALID_ARG; }

}  // namespace
}  // namespace vmoe

#define VMOE_TRY(expr)                \
    do {                              \
        vmoe_status _s = (expr);      \
        if (_s != VMOE_OK) return _s; \
    } while (0)

using namespace vmoe;

extern "C" {

size_t vmoe_head_loss_saved_bytes(const vmoe_head_shape* shape) {
    return check_shape(shape) == VMOE_OK ? head_saved_bytes(*shape) : 0;
}

size_t vmoe_head_loss_fwd_workspace_bytes(const vmoe_head_shape* shape) {
    return check_shape(shape) == VMOE_OK ? head_fwd_workspace_bytes(*shape) : 0;
}

size_t vmoe_head_loss_bwd_workspace_bytes(const vmoe_head_shape* shape) {
    return check_shape(shape) == VMOE_OK ? head_bwd_workspace_bytes(*shape) : 0;
}

vmoe_status vmoe_head_loss_fwd(const vmoe_head_shape* shape, const void* x, const void* weight,
                               const void* bias, const int32_t* labels,
                               const int32_t* teacher_idx, const float* teacher_logits,
                               const float* row_weight, float* losses, float* row_losses,
                               void* saved, void* workspace, size_t workspace_bytes,
                               void* stream) {
    VMOE_TRY(check_shape(shape));
    const bool teacher = shape->n_teacher > 0;
    VMOE_TRY(need(dev(x) && dev(weight) && opt(bias) && opt(labels) && opt(row_weight)));
    VMOE_TRY(need(teacher ? dev(teacher_idx) && dev(teacher_logits)
                          : !teacher_idx && !teacher_logits && labels));
    VMOE_TRY(need(dev(losses) && opt(row_losses) && dev(saved)));
    if (workspace_bytes < head_fwd_workspace_bytes(*shape) || !dev(workspace))
        return VMOE_ERR_WORKSPACE;
    return head_fwd_launch(*shape, x, weight, bias, labels, teacher_idx, teacher_logits,
                           row_weight, losses, row_losses, saved, workspace, as_stream(stream));
}

vmoe_status vmoe_head_loss_bwd(const vmoe_head_shape* shape, const void* weight,
                               const void* saved, float w_label, float w_teacher, void* dx,
                               void* dweight, void* dbias, void* workspace,
                               size_t workspace_bytes, void* stream) {
    VMOE_TRY(check_shape(shape));
    VMOE_TRY(need(dev(weight) && dev(saved) && opt(dx) && opt(dweight) && opt(dbias)));
    VMOE_TRY(need(isfinite(w_label) && isfinite(w_teacher * shape->temperature)));
    VMOE_TRY(need(dx || dweight || dbias));
    if (workspace_bytes < head_bwd_workspace_bytes(*shape) || !dev(workspace))
        return VMOE_ERR_WORKSPACE;
    return head_bwd_launch(*shape, weight, saved, w_label, w_teacher, dx, dweight, dbias,
                           workspace, as_stream(stream));
}

}  // extern "C"
