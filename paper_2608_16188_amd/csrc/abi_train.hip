// extern "C" entry points of vmoe_train.h: argument validation, then launches.
#include <float.h>
#include <math.h>

#include "common_train.h"

namespace vmoe {

// Launchers (one source file each).
size_t block_norm_bwd_workspace_bytes(const vmoe_norm_shape& s);
vmoe_status block_norm_fwd_launch(const vmoe_norm_shape& s, const void* x, const void* y,
                                  const void* post_w, const void* post_b, const void* gate,
                                  const float* row_scale, const void* pre_w, const void* pre_b,
                                  void* x_out, void* h, float* post_stats, float* pre_stats,
                                  hipStream_t st);
vmoe_status block_norm_bwd_launch(const vmoe_norm_shape& s, const void* dx_out, const void* dh,
                                  const void* x_out, const void* y, const void* post_w,
                                  const void* post_b, const void* gate, const float* row_scale,
                                  const void* pre_w, const float* post_stats,
                                  const float* pre_stats, void* dx, void* dy, float* dpost_w,
                                  float* dpost_b, float* dgate, float* dpre_w, float* dpre_b,
                                  void* ws, hipStream_t st);
size_t gate_loss_workspace_bytes(const Dims& D);
vmoe_status gate_loss_launch(const Dims& D, const float* logits, const float* bias,
                             const float* noise, const float* probs, const int32_t* idx,
                             const uint8_t* mask, float w_balance, float w_z, float* losses,
                             int32_t* demand, float* mean_probs, float* dlogits, void* ws,
                             hipStream_t st);
long long adamw_plan_chunks(const vmoe_adamw_tensor* tensors, int n_tensors);
void adamw_plan_write(const vmoe_adamw_tensor* tensors, int n_tensors, void* plan);
size_t grad_norm_workspace_bytes(long long n_chunks);
vmoe_status grad_norm_launch(const void* plan, long long n_chunks, double grad_scale,
                             double max_norm, float* clip, void* ws, hipStream_t st);
vmoe_status adamw_launch(const void* plan, long long n_chunks, const vmoe_adamw_hyper& hy,
                         const float* clip, hipStream_t st);
vmoe_status state_values_launch(const uint8_t* codes, const uint8_t* scale, bool is_signed,
                                long long n, void* out, int out_dtype, hipStream_t st);

namespace {

constexpr int kMaxNormWidth = 16384;
constexpr long long kMaxChunks = 0x7FFFFFFFLL;
constexpr long long kMaxValues = 1LL << 36;

bool known_dtype(int t) { return t == VMOE_F32 || t == VMOE_BF16; }
bool known_norm(int k) { return k >= VMOE_NORM_NONE && k <= VMOE_NORM_LAYER; }

vmoe_status check_norm_shape(const vmoe_norm_shape* s) {
    if (!s || s->n_tokens < 0 || s->n_groups < 1 || s->n_tokens % s->n_groups != 0)
        return VMOE_ERR_INVALID_ARG;
    if (s->d_model < 8 || s->d_model % 8 != 0 || s->reserved != 0) return VMOE_ERR_INVALID_ARG;
    if (!known_dtype(s->dtype) || !known_dtype(s->stream_dtype) || !known_dtype(s->dh_dtype))
        return VMOE_ERR_INVALID_ARG;
    if (s->dtype == VMOE_F32 && (s->stream_dtype != VMOE_F32 || s->dh_dtype != VMOE_F32))
        return VMOE_ERR_INVALID_ARG;
    if (!known_norm(s->pre_norm) || !known_norm(s->post_norm)) return VMOE_ERR_INVALID_ARG;
    if (!(s->eps > 0.0f) || !isfinite(s->eps) || !isfinite(s->residual_scale) ||
        !isfinite(s->branch_scale))
        return VMOE_ERR_INVALID_ARG;
    // a row lies in the registers of one block; token numbers keep room for a
    // grid's stride in 32 bits
    if (s->d_model > kMaxNormWidth || s->n_tokens > (1 << 30) || s->n_groups > (1 << 30))
        return VMOE_ERR_UNSUPPORTED;
    return VMOE_OK;
}

bool dev(const void* p) { return p != nullptr && aligned16(p); }
bool opt(const void* p) { return p == nullptr || aligned16(p); }

// What goes with a norm may be given only where there is one.
bool norm_args(int kind, const void* weight, const void* bias) {
    return kind != VMOE_NORM_NONE ? opt(weight) && opt(bias) : !weight && !bias;
}

}  // namespace
}  // namespace vmoe

#define VMOE_TRY(expr)                \
    do {                              \
        vmoe_status _s = (expr);      \
        if (_s != VMOE_OK) return _s; \
    } while (0)

using namespace vmoe;

static vmoe_status need(bool ok) { return ok ? VMOE_OK : VMOE_ERR_INVALID_ARG; }

extern "C" {

vmoe_status vmoe_block_norm_fwd(const vmoe_norm_shape* shape, const void* x, const void* y,
                                const void* post_weight, const void* post_bias, const void* gate,
                                const float* row_scale, const void* pre_weight,
                                const void* pre_bias, void* x_out, void* h, float* post_stats,
                                float* pre_stats, void* stream) {
    VMOE_TRY(check_norm_shape(shape));
    const bool pre = shape->pre_norm != VMOE_NORM_NONE, post = shape->post_norm != VMOE_NORM_NONE;
    VMOE_TRY(need(dev(x) && opt(y) && opt(gate) && opt(row_scale)));
    VMOE_TRY(need(norm_args(shape->pre_norm, pre_weight, pre_bias) &&
                  norm_args(shape->post_norm, post_weight, post_bias)));
    VMOE_TRY(need(y != nullptr ? dev(x_out) : pre && !post && !gate && !row_scale));
    VMOE_TRY(need(!pre || (dev(h) && dev(pre_stats))));
    VMOE_TRY(need(!post || dev(post_stats)));
    return block_norm_fwd_launch(*shape, x, y, post_weight, post_bias, gate, row_scale, pre_weight,
                                 pre_bias, x_out, h, post_stats, pre_stats, as_stream(stream));
}

size_t vmoe_block_norm_bwd_workspace_bytes(const vmoe_norm_shape* shape) {
    return check_norm_shape(shape) == VMOE_OK ? block_norm_bwd_workspace_bytes(*shape) : 0;
}

vmoe_status vmoe_block_norm_bwd(const vmoe_norm_shape* shape, const void* dx_out, const void* dh,
                                const void* x_out, const void* y, const void* post_weight,
                                const void* post_bias, const void* gate, const float* row_scale,
                                const void* pre_weight, const float* post_stats,
                                const float* pre_stats, void* dx, void* dy, float* dpost_weight,
                                float* dpost_bias, float* dgate, float* dpre_weight,
                                float* dpre_bias, void* workspace, size_t workspace_bytes,
                                void* stream) {
    VMOE_TRY(check_norm_shape(shape));
    const bool pre = shape->pre_norm != VMOE_NORM_NONE, post = shape->post_norm != VMOE_NORM_NONE;
    VMOE_TRY(need(opt(dx_out) && opt(y) && opt(gate) && opt(row_scale) && dev(dx)));
    VMOE_TRY(need(norm_args(shape->pre_norm, pre_weight, dpre_bias) &&
                  norm_args(shape->pre_norm, dpre_weight, nullptr) &&
                  norm_args(shape->post_norm, post_weight, post_bias) &&
                  norm_args(shape->post_norm, dpost_weight, dpost_bias) && opt(dgate)));
    VMOE_TRY(need(pre ? dev(dh) && dev(x_out) && dev(pre_stats) : !dh));
    VMOE_TRY(need(y != nullptr ? dev(dy) : pre && !post && !gate && !row_scale && !dgate));
    VMOE_TRY(need(!post || dev(post_stats)));
    const size_t need_ws = block_norm_bwd_workspace_bytes(*shape);
    if (workspace_bytes < need_ws || (need_ws > 0 && !dev(workspace))) return VMOE_ERR_WORKSPACE;
    return block_norm_bwd_launch(*shape, dx_out, dh, x_out, y, post_weight, post_bias, gate,
                                 row_scale, pre_weight, post_stats, pre_stats, dx, dy,
                                 dpost_weight, dpost_bias, dgate, dpre_weight, dpre_bias,
                                 workspace, as_stream(stream));
}

size_t vmoe_load_balance_loss_workspace_bytes(const vmoe_shape* shape) {
    Dims D;
    return make_dims(shape, &D) == VMOE_OK ? gate_loss_workspace_bytes(D) : 0;
}

vmoe_status vmoe_load_balance_loss(const vmoe_shape* shape, const float* logits,
                                   const float* logit_bias, const float* noise, const float* probs,
                                   const int32_t* expert_idx, const uint8_t* token_mask,
                                   float w_balance, float w_z, float* losses, int32_t* demand,
                                   float* mean_probs, float* dlogits, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    Dims D;
    VMOE_TRY(make_dims(shape, &D));
    VMOE_TRY(need(dev(logits) && dev(probs) && dev(expert_idx) && opt(logit_bias) && opt(noise) &&
                  opt(token_mask)));
    VMOE_TRY(need(dev(losses) && dev(demand) && opt(mean_probs) && dev(dlogits)));
    VMOE_TRY(need(isfinite(w_balance) && isfinite(w_z)));
    const size_t need_ws = gate_loss_workspace_bytes(D);
    if (workspace_bytes < need_ws || !dev(workspace)) return VMOE_ERR_WORKSPACE;
    return gate_loss_launch(D, logits, logit_bias, noise, probs, expert_idx, token_mask, w_balance,
                            w_z, losses, demand, mean_probs, dlogits, workspace,
                            as_stream(stream));
}

int64_t vmoe_adamw_plan_chunks(const vmoe_adamw_tensor* tensors, int32_t n_tensors) {
    if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return -1;
    const long long n = adamw_plan_chunks(tensors, n_tensors);
    return n < 0 ? -1 : n;
}

vmoe_status vmoe_adamw_plan(const vmoe_adamw_tensor* tensors, int32_t n_tensors, void* plan,
                            size_t plan_bytes) {
    VMOE_TRY(need(n_tensors >= 0 && (n_tensors == 0 || tensors)));
    const long long n = adamw_plan_chunks(tensors, n_tensors);
    if (n == -2) return VMOE_ERR_UNSUPPORTED;
    VMOE_TRY(need(n >= 0));
    if (plan_bytes / VMOE_ADAMW_PLAN_ENTRY_BYTES < static_cast<size_t>(n) ||
        (n > 0 && (!plan || (reinterpret_cast<uintptr_t>(plan) & 7u) != 0)))
        return VMOE_ERR_WORKSPACE;
    adamw_plan_write(tensors, n_tensors, plan);
    return VMOE_OK;
}

size_t vmoe_grad_norm_workspace_bytes(int64_t n_chunks) {
    return n_chunks < 0 || n_chunks > kMaxChunks ? 0 : grad_norm_workspace_bytes(n_chunks);
}

vmoe_status vmoe_grad_norm(const void* plan, int64_t n_chunks, double grad_scale, double max_norm,
                           float* clip, void* workspace, size_t workspace_bytes, void* stream) {
    VMOE_TRY(need(n_chunks >= 0 && n_chunks <= kMaxChunks && (n_chunks == 0 || dev(plan))));
    VMOE_TRY(need(isfinite(grad_scale) && max_norm > 0.0 && dev(clip)));
    if (workspace_bytes < grad_norm_workspace_bytes(n_chunks) || !dev(workspace))
        return VMOE_ERR_WORKSPACE;
    return grad_norm_launch(plan, n_chunks, grad_scale, max_norm, clip, workspace,
                            as_stream(stream));
}

vmoe_status vmoe_adamw(const void* plan, int64_t n_chunks, const vmoe_adamw_hyper* hyper,
                       const float* clip, void* stream) {
    VMOE_TRY(need(n_chunks >= 0 && n_chunks <= kMaxChunks && (n_chunks == 0 || dev(plan))));
    VMOE_TRY(need(hyper != nullptr && opt(clip)));
    VMOE_TRY(need(hyper->lr >= 0.0 && isfinite(hyper->lr) && isfinite(hyper->grad_scale)));
    VMOE_TRY(need(hyper->beta1 >= 0.0 && hyper->beta1 < 1.0 && hyper->beta2 >= 0.0 &&
                  hyper->beta2 < 1.0));
    VMOE_TRY(need(hyper->eps >= static_cast<double>(FLT_MIN) && isfinite(hyper->eps)));
    VMOE_TRY(need(hyper->step >= 1 && hyper->reserved == 0));
    return adamw_launch(plan, n_chunks, *hyper, clip, as_stream(stream));
}

vmoe_status vmoe_adamw_state_values(const uint8_t* codes, const uint8_t* scale, int32_t is_signed,
                                    int64_t n, void* out, int32_t out_dtype, void* stream) {
    VMOE_TRY(need(n >= 0 && (is_signed == 0 || is_signed == 1) && known_dtype(out_dtype)));
    VMOE_TRY(need(n == 0 || (codes && (reinterpret_cast<uintptr_t>(codes) & 3u) == 0 && scale &&
                             dev(out))));
    if (n >= kMaxValues) return VMOE_ERR_UNSUPPORTED;
    return state_values_launch(codes, scale, is_signed == 1, n, out, out_dtype, as_stream(stream));
}

}  // extern "C"
