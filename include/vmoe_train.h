/*
 * vmoe_train.h -- what a training step of one sparse block needs around the
 * layer of vmoe.h: the norms, gate and residual on either side of it, the
 * load-balance loss on its gate with the experts' demand, and the optimizer
 * that turns its gradients into new weights. Entry points of libvmoe.so.
 *
 * The conventions of vmoe.h hold: device pointers owned by the caller, 16-byte
 * aligned, row-major and contiguous; work enqueued on `stream` without
 * synchronising; no allocation; status codes, checked before anything is
 * enqueued; required pointers checked whatever the sizes. A workspace needs no
 * clearing and holds nothing between calls. Every sum is taken in a fixed
 * order (no float atomics): the same inputs give the same bits. Scalars that
 * are passed by value are recorded by a graph capture as they are then.
 */
#ifndef VMOE_TRAIN_H
#define VMOE_TRAIN_H

#include "vmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * Block norm
 * ------------------------------------------------------------------------- */

typedef enum { VMOE_NORM_NONE = 0, VMOE_NORM_RMS = 1, VMOE_NORM_LAYER = 2 } vmoe_norm_kind;

typedef struct vmoe_norm_shape {
    int32_t n_tokens;      /* N >= 0                                              */
    int32_t n_groups;      /* G >= 1, divides N: rows of `gate`                   */
    int32_t d_model;       /* d, multiple of 8, at most 16384 (else UNSUPPORTED)  */
    int32_t dtype;         /* y, h, dy and the weights (vmoe_dtype)               */
    int32_t stream_dtype;  /* x, x_out, dx_out, dx: F32, or BF16 with dtype BF16  */
    int32_t dh_dtype;      /* dh: F32 (as the layer's dx), or dtype               */
    int32_t pre_norm;      /* norm of x_out that gives h (vmoe_norm_kind)         */
    int32_t post_norm;     /* norm of the block's output y                        */
    float eps;             /* > 0                                                 */
    float residual_scale;  /* finite                                              */
    float branch_scale;    /* finite                                              */
    int32_t reserved;      /* must be 0                                           */
} vmoe_norm_shape;

/* What stands between two blocks, in one pass over the tokens: the norm after
 * a block, its gate, the residual add and the norm before the next block.
 *   q     = post(y)                                  y if post_norm is NONE
 *   x_out = residual_scale x + (branch_scale row_scale[t]) (gate[g,:] q)
 *   h     = pre(x_out)                               from x_out before it is rounded
 * with norm(v) = (v - mean) rstd weight + bias, rstd = 1/sqrt(var + eps)
 * (LAYER: population variance, taken about the mean) or
 * rstd = 1/sqrt(mean(v^2) + eps) and mean = 0 (RMS).
 *   x [N, d], x_out [N, d] (stream_dtype; may be the same), y [N, d], h [N, d] (dtype)
 *   post_weight, post_bias, pre_weight, pre_bias [d] (dtype): NULL weight = 1,
 *     NULL bias = 0; NULL where that norm is NONE
 *   gate [G, d] (dtype) or NULL = 1; tokens of group g are [g N/G, (g+1) N/G)
 *   row_scale [N] f32 or NULL = 1 (drop-path): a token whose row_scale is 0
 *     leaves the block out: its row of y is not read and may hold anything
 *   post_stats, pre_stats [N, 2] f32 out: mean and rstd, for the backward
 *     (0, 0 in post_stats of a token that leaves the block out)
 * y NULL: only h = pre(x) (x_out unused, may be NULL; post_norm NONE and gate, row_scale NULL).
 * pre_norm NONE: h and pre_stats unused, may be NULL. Not both.
 * All arithmetic is f32. */
vmoe_status vmoe_block_norm_fwd(const vmoe_norm_shape* shape, const void* x, const void* y,
                                const void* post_weight, const void* post_bias, const void* gate,
                                const float* row_scale, const void* pre_weight,
                                const void* pre_bias, void* x_out, void* h, float* post_stats,
                                float* pre_stats, void* stream);

/* Bytes of scratch that vmoe_block_norm_bwd needs (0 on an invalid shape). */
size_t vmoe_block_norm_bwd_workspace_bytes(const vmoe_norm_shape* shape);

/* Backward of vmoe_block_norm_fwd from dx_out [N, d] (gradient of x_out along
 * the stream, stream_dtype; NULL = 0) and dh [N, d] (dh_dtype; NULL exactly if
 * pre_norm is NONE), at the x_out that the forward stored (x where y was NULL):
 *   n = (x_out - mean) rstd, dn = dh pre_weight
 *   S = dx_out + rstd (dn - [LAYER: avg(dn)] - n avg(dn n))
 *   dx          = residual_scale S (or S where y is NULL)   [N, d] stream_dtype
 *   dpre_weight = sum_t dh n, dpre_bias = sum_t dh          [d] f32
 *   a = branch_scale row_scale[t], m = unit output of post (y if NONE)
 *   dgate[g]    = sum_{t in g} a S (post_weight m + post_bias)   [G, d] f32
 *   dpost_weight = sum_t a S gate m, dpost_bias = sum_t a S gate [d] f32
 *   dy          = gradient of post at y from a S gate       [N, d] dtype
 *                 (zeros for a token that leaves the block out; y not read there)
 * dx may be dx_out's buffer, dy may be y's. Parameter gradients that are NULL
 * are not formed. workspace: vmoe_block_norm_bwd_workspace_bytes(shape) bytes. */
vmoe_status vmoe_block_norm_bwd(const vmoe_norm_shape* shape, const void* dx_out, const void* dh,
                                const void* x_out, const void* y, const void* post_weight,
                                const void* post_bias, const void* gate, const float* row_scale,
                                const void* pre_weight, const float* post_stats,
                                const float* pre_stats, void* dx, void* dy, float* dpost_weight,
                                float* dpost_bias, float* dgate, float* dpre_weight,
                                float* dpre_bias, void* workspace, size_t workspace_bytes,
                                void* stream);

/* ---------------------------------------------------------------------------
 * Load-balance loss
 * ------------------------------------------------------------------------- */

/* Bytes of scratch that vmoe_load_balance_loss needs (0 on an invalid shape). */
size_t vmoe_load_balance_loss_workspace_bytes(const vmoe_shape* shape);

/* The experts' demand and two auxiliary losses on the gate, per routing group,
 * with their gradient with respect to the router logits. Over the n_g tokens of
 * group g that token_mask keeps:
 *   demand[g,e]     = number of (t, j) with expert_idx[t,j] = e (before capacity)
 *   f[g,e]          = demand[g,e] / (k n_g)
 *   mean_probs[g,e] = sum_t probs[t,e] / n_g
 *   losses[g,0]     = E sum_e f[g,e] mean_probs[g,e]       1 for an even load
 *   losses[g,1]     = sum_t lse_t^2 / n_g, lse_t = log sum_e exp z[t,e]
 *   dlogits[t,e]    = d/dlogits of sum_g w_balance losses[g,0] + w_z losses[g,1]
 *                   = p (w_balance E (f - <f, p>) + 2 w_z lse) / n_g
 * (demand is piecewise constant and passes no gradient); 0 for masked tokens.
 * n_g = 0 gives losses, demand and mean_probs of 0.
 *   logits, probs [N, E] f32, expert_idx [N, k] i32: vmoe_route's outputs;
 *     z = (logits + logit_bias) + noise as there, and lse_t = max z - log max p
 *     (the softmax's largest term), so no second exponential is taken
 *   logit_bias [E], noise [N, E] f32 or NULL, as given to vmoe_route
 *   token_mask [N] u8 or NULL: 0 = padding; its rows of logits, noise, probs and
 *     expert_idx may hold anything
 *   losses [G, 2] f32, demand [G, E] i32, dlogits [N, E] f32 out;
 *   mean_probs [G, E] f32 out or NULL
 * Indices outside [0, E) are not counted. Pass dlogits to
 * vmoe_dispatch_route_bwd_dlogits. Sums are f32 within a chunk of tokens and
 * double across chunks. VMOE_ERR_INVALID_ARG for non-finite weights. */
vmoe_status vmoe_load_balance_loss(const vmoe_shape* shape, const float* logits,
                                   const float* logit_bias, const float* noise, const float* probs,
                                   const int32_t* expert_idx, const uint8_t* token_mask,
                                   float w_balance, float w_z, float* losses, int32_t* demand,
                                   float* mean_probs, float* dlogits, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * AdamW over many tensors
 * ------------------------------------------------------------------------- */

/* States (first and second moment) of a tensor: f32, or 8 bits.
 * An 8-bit state keeps a byte per element and a scale byte s per block of 128
 * consecutive elements (the last one may be shorter): an element is
 * 2^(s - 127) u, u from its byte with 3 mantissa bits M and an exponent X:
 *   m: sign bit, 4-bit X, M;  u = +-2^(X - 15) (1 + M/8), +-2^-14 M/8 for X = 0
 *   v:           5-bit X, M;  u =   2^(X - 31) (1 + M/8),   2^-30 M/8 for X = 0
 * s is the f32 exponent field of the block's largest magnitude after rounding it
 * up to 3 mantissa bits (0 for a block of zeros or of values below 2^-126).
 * Where that overflows, or the block holds an infinity or NaN, s is 255 and the
 * whole block reads as infinite from then on.
 * Elements are rounded at random, up with the probability of what is cut off,
 * so a moment's expected value is its exact one however small a step's change
 * is (rounding to nearest would freeze v, which changes by a thousandth a step);
 * a positive v never becomes 0, so that no m is divided by an emptied v.
 * The random numbers are a function of seed, step and the element's number i
 * (index0 + its place) alone, in 32-bit arithmetic:
 *   mix(x): x ^= x >> 16; x *= 0x6A09E667; x ^= x >> 15; x *= 0xBB67AE85; x ^= x >> 16
 *   key = mix(seed ^ mix(step 0x9E3779B1)), and mix(key ^ (i >> 32)) where i >= 2^32
 *   bits = mix((i 0x9E3779B1) ^ key); its low 16 bits are m's, the high ones v's
 * and an element whose cut-off fraction is q of a step goes up where
 * q + (16 bits + 1/2) / 2^16 >= 1. */
typedef enum { VMOE_STATE_F32 = 0, VMOE_STATE_8BIT = 1 } vmoe_adamw_state;

typedef struct vmoe_adamw_tensor {
    void* param;          /* [n] param_dtype, updated                                 */
    float* master;        /* [n] f32 master weights, updated: required with a BF16
                             param (which becomes its rounding), NULL with an F32 one */
    const void* grad;     /* [n] grad_dtype                                           */
    void* m;              /* [n] first moment: f32, or u8                             */
    void* v;              /* [n] second moment                                        */
    uint8_t* m_scale;     /* [ceil(n / 128)] with 8-bit states, else NULL             */
    uint8_t* v_scale;
    int64_t n;            /* >= 0; with n = 0 no pointer is looked at                 */
    uint64_t index0;      /* number of the tensor's first element in the sequence of
                             random numbers, a multiple of 128                        */
    double lr_mult;       /* finite, >= 0: the tensor's learning rate is lr lr_mult   */
    double weight_decay;  /* finite, >= 0                                             */
    int32_t param_dtype;  /* vmoe_dtype                                               */
    int32_t grad_dtype;   /* vmoe_dtype                                               */
    int32_t state;        /* vmoe_adamw_state                                         */
    int32_t reserved;     /* must be 0                                                */
} vmoe_adamw_tensor;

typedef struct vmoe_adamw_hyper {
    double lr;          /* finite, >= 0                                               */
    double beta1;       /* in [0, 1)                                                  */
    double beta2;       /* in [0, 1)                                                  */
    double eps;         /* finite, at least 2^-126. Squares of gradients below some
                           2^-75 are 0 in f32: with an eps below them, grad_scale has
                           to bring gradients above that                              */
    double grad_scale;  /* finite: gradients are multiplied by it                     */
    int64_t step;       /* >= 1: this step's number, for the bias corrections         */
    uint32_t seed;      /* of the random numbers (with step and the element's number) */
    uint32_t reserved;  /* must be 0                                                  */
} vmoe_adamw_hyper;

/* A plan lists the tensors in chunks, VMOE_ADAMW_CHUNK elements each. It is made
 * once for a set of tensors (and again when one of them moves): vmoe_adamw_plan
 * writes it to host memory, the caller copies it to the GPU. Small pointers (the
 * scale bytes and 8-bit states) need only their own alignment: 4 bytes for u8
 * moments, 1 for scales; the others are 16-byte aligned. */
#define VMOE_ADAMW_CHUNK 8192
#define VMOE_ADAMW_PLAN_ENTRY_BYTES 80

/* Chunks of a plan (host): -1 on invalid arguments. A plan takes that many
 * times VMOE_ADAMW_PLAN_ENTRY_BYTES bytes. */
int64_t vmoe_adamw_plan_chunks(const vmoe_adamw_tensor* tensors, int32_t n_tensors);

/* Writes the plan to HOST memory of at least that size (8-byte aligned).
 * VMOE_ERR_INVALID_ARG: a NULL or misaligned pointer, n < 0, an unknown type,
 * a BF16 param without master weights or an F32 one with them, scales that are
 * missing (8 bits) or given (f32), index0 % 128 != 0, a negative or non-finite
 * rate; VMOE_ERR_UNSUPPORTED: 2^31 chunks or more; VMOE_ERR_WORKSPACE: too small. */
vmoe_status vmoe_adamw_plan(const vmoe_adamw_tensor* tensors, int32_t n_tensors, void* plan,
                            size_t plan_bytes);

/* Bytes of scratch that vmoe_grad_norm needs (0 for a negative n_chunks). */
size_t vmoe_grad_norm_workspace_bytes(int64_t n_chunks);

/* clip[0] = |grad_scale| times the 2-norm of all the plan's gradients together,
 * clip[1] = min(1, max_norm / (clip[0] + 1e-6)), or NaN where the norm is not
 * finite (a gradient is not, or its square leaves the range of f32): vmoe_adamw
 * given that clip changes nothing. max_norm > 0 (infinity: the norm alone).
 * plan: device copy of the plan, n_chunks as from vmoe_adamw_plan_chunks;
 * clip [2] f32, device, out. Squares are summed in f32 over a
 * thread's 32 elements of a chunk, in double beyond. */
vmoe_status vmoe_grad_norm(const void* plan, int64_t n_chunks, double grad_scale, double max_norm,
                           float* clip, void* workspace, size_t workspace_bytes, void* stream);

/* One AdamW step over every tensor of the plan:
 *   g = grad (grad_scale clip[1])                   clip NULL: 1
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   p = p - lr lr_mult (m c1 / (sqrt(v) c2 + eps) + weight_decay p)
 *   c1 = 1 / (1 - beta1^step),  c2 = 1 / sqrt(1 - beta2^step)
 * in f32, each product and sum of m and v rounded by itself (so that two
 * programs that follow this text get the same 8-bit states); p from the new
 * moments before they are rounded to 8 bits. p is master where there is one.
 * A clip[1] that is NaN leaves every tensor as it is; no step was taken then, and
 * the next call's step is to be the same number again, or its bias corrections
 * assume a gradient that the moments have not seen.
 * hyper is read by the call: a graph that captured it repeats that step's number on
 * every replay, so its rate and bias corrections stay and 8-bit states are rounded
 * with the same random numbers each time, no longer free of bias. A training step's
 * graph is to end before this call. */
vmoe_status vmoe_adamw(const void* plan, int64_t n_chunks, const vmoe_adamw_hyper* hyper,
                       const float* clip, void* stream);

/* The values of an 8-bit state (checkpoints, inspection): out [n] out_dtype; both
 * types hold them exactly unless they leave the normal range. is_signed: 1 for
 * m, 0 for v. codes [n] u8 4-byte aligned, scale [ceil(n / 128)] u8; n of 2^36
 * and more is VMOE_ERR_UNSUPPORTED. */
vmoe_status vmoe_adamw_state_values(const uint8_t* codes, const uint8_t* scale, int32_t is_signed,
                                    int64_t n, void* out, int32_t out_dtype, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* VMOE_TRAIN_H */
