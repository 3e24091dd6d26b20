/* inframind_learn.h -- C ABI of the learner's operators on MI355X.
 *
 * What follows a rollout when the executor policy is trained (Sec. 4.4): the
 * rollout (im_route_sample) gives actions, log-probabilities and entropies;
 * these operators compute the policy's layers and their gradients, the
 * log-probability and entropy of a linear softmax head with the gradient of
 * both, and the AdamW step of the parameters.
 *
 * Groups. Rows come in n_groups ranges, each with weights of its own: the
 * members of a population of policies (a tick's rows are env-major, so the
 * envs of a member are one range), or experts. offsets [n_groups + 1] (device
 * int32) is their CSR: group g has rows [offsets[g], offsets[g+1]),
 * offsets[0] = 0, offsets[n_groups] <= n_rows; a group may be empty. Rows
 * behind offsets[n_groups] are not read, and their outputs are left as they
 * were. offsets NULL: one group that holds every row (n_groups = 1). With n_rows = 0
 * offsets are not read.
 *
 * Conventions for every call:
 *   - Pointers are device memory of the current device unless marked "host";
 *     caller-owned buffers must stay valid until the stream work that uses
 *     them has finished. What a call writes (outputs, workspace, error) must not
 *     overlap what it reads or one another (refused); views of the same rows that
 *     take different columns do not overlap.
 *   - Matrices are row-major. ld_* are row strides in elements (at least the
 *     row's width, at most IM_MAX_LD); weights and their gradients are contiguous. 16-bit data
 *     needs 2-byte, 32-bit data 4-byte alignment, nothing more.
 *   - dtype IM_BF16: bf16 activations, weights and their gradients; IM_F32:
 *     fp32. Products are accumulated in fp32; biases, their gradients and the
 *     per-row statistics are fp32. A result is rounded once to its type.
 *   - `stream` is a hipStream_t (NULL = the default stream). Calls are
 *     stream-ordered and asynchronous, allocate nothing and may be captured
 *     into a graph. Results do not depend on timing: the same call on the same
 *     inputs gives the same bits.
 *   - `workspace`: workspace_bytes of device memory, 256-byte aligned, at least
 *     what the matching im_*_workspace reports; its contents need not be kept.
 *     Calls that may run at the same time need workspaces of their own.
 *   - `error`: a device int32 the call sets IM_ERR_* bits in, or NULL.
 *     IM_ERR_COUNT: offsets are not a CSR as above; nothing is computed.
 *   - Invalid arguments return IM_EINVAL synchronously and change nothing;
 *     im_learn_last_error describes the calling thread's last failed call.
 */
#ifndef INFRAMIND_LEARN_H
#define INFRAMIND_LEARN_H

#include "inframind.h"

#ifdef __cplusplus
extern "C" {
#endif

#define IM_MAX_GROUPS 1024        /* n_groups                                          */
#define IM_MAX_ROWS   (1 << 30)   /* n_rows                                            */
#define IM_MAX_DIM    65536       /* in_dim, out_dim, dim                              */
#define IM_MAX_LD     (1 << 22)   /* row strides (elements)                            */
#define IM_MAX_CLASSES (1 << 22)  /* n_classes                                         */
#define IM_MAX_TENSORS 65536      /* tensors of an im_adamw                            */
#define IM_MAX_ELEMENTS (1LL << 37)  /* elements of an im_adamw's tensors together      */
#define IM_STATE_BLOCK 256        /* elements of an 8-bit state that share a scale     */

/* ---- grouped layers -------------------------------------------------------
 * y_i = act(W_g x_i + b_g) for the rows i of group g.
 *   n_rows    rows of x and y, in [0, IM_MAX_ROWS]
 *   in_dim, out_dim   in [1, IM_MAX_DIM]
 *   dtype     im_dtype of x, W, y and of dy, dx, dW
 *   relu      forward: 1 = act is max(., 0), 0 = none
 *   relu_in   backward: 1 = x is itself a ReLU output, and dx is the gradient
 *             before that ReLU (zero where x <= 0); 0 = the gradient of x
 *   ld_x, ld_y, ld_dx   row strides of x, of y and dy, of dx */
typedef struct {
  int32_t n_groups, n_rows, in_dim, out_dim;
  int32_t dtype, relu, relu_in, reserved;
  int64_t ld_x, ld_y, ld_dx;
} im_linear_desc;

/* Bytes of workspace of im_linear_forward (backward = 0) or im_linear_backward
 * (backward = 1), in *bytes (host). */
im_status im_linear_workspace(const im_linear_desc* desc, int32_t backward, int64_t* bytes);

/*   x [n_rows x in_dim], W [n_groups x out_dim x in_dim], b fp32 [n_groups x
 *   out_dim] or NULL, y [n_rows x out_dim] out */
im_status im_linear_forward(const im_linear_desc* desc, const int32_t* offsets, const void* x,
                            const void* W, const float* b, void* y, void* workspace,
                            int64_t workspace_bytes, int32_t* error, void* stream);

/* Gradients from dy, the gradient of W_g x_i + b_g (that is, of y before its
 * activation: the layer above returns it so with relu_in).
 *   dx [n_rows x in_dim] = W_g^T dy_i; dW [n_groups x out_dim x in_dim] =
 *   sum_i dy_i x_i^T; db fp32 [n_groups x out_dim] = sum_i dy_i. Each may be
 *   NULL to skip it; those of an empty group are zero. W is read for dx only, x
 *   for dW and for dx with relu_in. */
im_status im_linear_backward(const im_linear_desc* desc, const int32_t* offsets, const void* dy,
                             const void* x, const void* W, void* dx, void* dW, float* db,
                             void* workspace, int64_t workspace_bytes, int32_t* error,
                             void* stream);

/* ---- softmax head -----------------------------------------------------------
 * z_i = W_g h_i + b_g, pi_i = softmax of z_i over the row's valid classes; the
 * logits are never kept. With target = the taken action, logp and entropy are
 * those that im_route_sample reports (Sec. 4.4, Eq. 5); -logp is the cross entropy.
 *   n_rows    in [0, IM_MAX_ROWS]; dim in [1, IM_MAX_DIM]; n_classes in [1, IM_MAX_CLASSES]
 *   dtype     im_dtype of h, W, dh, dW
 *   relu_in   backward: as in im_linear_desc, for h and dh
 *   ld_h, ld_dh   row strides
 * valid: uint32 [n_rows x ceil(n_classes / 32)], class j of a row is valid when
 * bit j % 32 of its word j / 32 is set, or NULL (every class is). A class whose
 * logit is -infinity is not valid either; any finite logit is one like others, the
 * lowest float too. A row without a valid class has logp, entropy and gradients 0
 * and lse -infinity. */
typedef struct {
  int32_t n_groups, n_rows, dim, n_classes;
  int32_t dtype, relu_in, reserved0, reserved1;
  int64_t ld_h, ld_dh;
} im_head_desc;

im_status im_head_workspace(const im_head_desc* desc, int32_t backward, int64_t* bytes);

/*   target   int32 [n_rows]: a class, or -1 (none: logp = 0). IM_ERR_ACTION: a
 *            target outside [-1, n_classes) or masked by `valid`; it counts as -1
 *   logp     fp32 [n_rows] out: ln pi(target) (-infinity where the target's logit is)
 *   entropy  fp32 [n_rows] out: -sum pi ln pi, or NULL
 *   lse      fp32 [n_rows] out: ln sum exp z over the valid classes (im_head_backward
 *            reads it), or NULL */
im_status im_head_forward(const im_head_desc* desc, const int32_t* offsets, const void* h,
                          const void* W, const float* b, const uint32_t* valid,
                          const int32_t* target, float* logp, float* entropy, float* lse,
                          void* workspace, int64_t workspace_bytes, int32_t* error, void* stream);

/* Gradients of sum_i (dlogp_i logp_i + dentropy_i entropy_i):
 *   dz_ij = dlogp_i ([j = target_i] - pi_ij) - dentropy_i pi_ij (ln pi_ij + entropy_i)
 *   dh_i = W_g^T dz_i, dW = sum_i dz_i h_i^T, db = sum_i dz_i
 * lse and entropy are the forward call's; dentropy NULL: no entropy term
 * (entropy may then be NULL); dlogp does not count where target is -1. pi is
 * formed from fp32 logits and the fp32 lse, off by |lse| 2^-23 of itself
 * (and is 1 at most), and a row whose lse is -1e30 or less, all of whose valid classes
 * are masked by their biases then, has gradients 0 as one without a valid class.
 * dz is formed in pieces of the classes and, for IM_BF16, rounded where it enters the
 * products of dh and dW: to two bf16 numbers (16 bits of mantissa) for heads of
 * up to 64 classes and 512 columns, to one above that (half a step, 2^-8 of each
 * dz, which dh's and dW's own rounding repeats); db sums it in fp32. A row whose
 * dlogp (or target) and dentropy are both none adds nothing to dW and db, and its
 * dh is zero, whatever its h holds; W must be finite. dh, dW and db may be NULL
 * to skip them; b may be NULL (no bias). */
im_status im_head_backward(const im_head_desc* desc, const int32_t* offsets, const void* h,
                           const void* W, const float* b, const uint32_t* valid,
                           const int32_t* target, const float* lse, const float* entropy,
                           const float* dlogp, const float* dentropy, void* dh, void* dW, float* db,
                           void* workspace, int64_t workspace_bytes, int32_t* error, void* stream);

/* ---- AdamW --------------------------------------------------------------------
 * One step over many tensors in one launch:
 *   g = scale grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *   param = (1 - lr weight_decay) param - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32 (root and quotient of the last line to 2 units, an eps above 0 is 2^-126 at
 * least); t is the step's number.
 *   param  fp32 [n]; grad fp32 or bf16 [n]; copy bf16 [n] (the parameters
 *          rounded for the bf16 products), or NULL
 *   state_bits 32: m, v fp32 [n]; m_scale, v_scale NULL
 *   state_bits 8: m and sqrt(v) as OCP e4m3 bytes [n], fp32 scales [ceil(n /
 *          IM_STATE_BLOCK)]: block k holds m_scale[k] * e4m3. scale = largest
 *          magnitude / 448 (at least 2^-126), codes rounded to nearest even; a
 *          sqrt(v) above zero gets the smallest code at least, so that its
 *          element's step stays bounded. The step itself uses m and v as
 *          computed, before they are rounded. One value that is not finite
 *          makes its block NaN.
 *   decay  1 = weight_decay applies to the tensor, 0 = it does not
 *   n >= 0. What is written must not overlap anything else of the list (refused);
 *          gradients may be shared. */
typedef struct {
  float* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  uint16_t* copy;
  int64_t n;
  int32_t decay, reserved;
} im_adamw_tensor;

typedef struct im_adamw im_adamw;

/* Plan of a list of tensors (host array, copied; the buffers are borrowed and
 * keep their places for the plan's life).
 *   state_bits 32 or 8; grad_dtype im_dtype of every grad
 * Allocates the plan's table on the current device; synchronises `stream`. */
im_status im_adamw_create(const im_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits,
                          int32_t grad_dtype, void* stream, im_adamw** out);

/* One step on the plan's device.
 *   step   device int64 [1], in/out: steps done; the call does step t = *step + 1
 *          and stores t (so a captured step may be replayed)
 *   scale  device fp32 [1] multiplied into the gradients (the inverse of a loss
 *          scale, a clipping coefficient), or NULL
 * IM_EINVAL unless lr, eps, weight_decay are finite and >= 0 and both betas are in [0, 1). Two
 * steps of one plan must not run at the same time. */
im_status im_adamw_step(im_adamw* opt, double lr, double beta1, double beta2, double eps,
                        double weight_decay, int64_t* step, const float* scale, void* stream);

/* Free the plan (synchronises the device, so not while a graph is captured; the
 * tensors stay). NULL is ignored. */
void im_adamw_destroy(im_adamw* opt);

/* ---- routing to experts ------------------------------------------------------
 * Each row chooses top_k of n_experts from its logits z (a layer's outputs):
 *   s_j = softmax of z over the row's valid experts, or sigmoid(z_j)
 *   choice by c_j = s_j + bias_j, or by z_j without bias (which orders as s_j does);
 *   with n_sets > 1 the experts are n_sets equal ranges, and only those of the
 *   top_sets best sets may be chosen: a set's value is its best c (set_best = 1)
 *   or the sum of its two best, of s + bias or of s (set_best = 2; a set with
 *   one valid expert has that one's)
 *   weight = scale s of the chosen experts, with renorm divided by the sum of theirs
 * c and the sets' values are compared as computed in 64 bits; of equal ones the lowest index is best, and what
 * lies nearer to one another than a 64-bit number's rounding may come in either order.
 * Experts come in the order of their c. An expert is valid where `valid` (uint32
 * [n_rows x ceil(n_experts / 32)], as for the softmax head, or NULL) has its bit and
 * its z is neither NaN nor -infinity; +infinity counts as the largest float. One
 * whose c is then NaN or -infinity cannot be chosen (a bias of -infinity shuts an
 * expert off; it stays part of the softmax). Where a row has fewer to choose, the
 * rest of its experts are -1, their weights 0.
 *   n_rows in [0, IM_MAX_ROWS]; n_experts in [1, IM_MAX_GROUPS]; top_k in [1,
 *   IM_MAX_TOP_K], at most the experts of top_sets sets; n_sets divides n_experts;
 *   top_sets in [1, n_sets]
 *   dtype  im_dtype of z and dz; score IM_SOFTMAX or IM_SIGMOID
 *   ld_z, ld_dz   row strides */
#define IM_MAX_TOP_K 32
#define IM_SOFTMAX 0
#define IM_SIGMOID 1
typedef struct {
  int32_t n_rows, n_experts, top_k, n_sets, top_sets, set_best;
  int32_t dtype, score, renorm;
  float scale;
  int64_t ld_z, ld_dz;
} im_router_desc;

/*   bias fp32 [n_experts] or NULL; expert int32 [n_rows x top_k] out; weight fp32
 *   [n_rows x top_k] out */
im_status im_router_forward(const im_router_desc* desc, const void* z, const float* bias, const uint32_t* valid,
                            int32_t* expert, float* weight, void* stream);

/* dz of sum weight dweight, for the experts as given (the choice has no gradient; the
 * sets and the bias do not count). Experts are those of the forward call, or any
 * others: one listed twice counts twice. IM_ERR_ACTION: an expert outside [-1,
 * n_experts) or not valid; it counts as -1, whose dweight does not count. dz is
 * zero for experts that are not valid. */
im_status im_router_backward(const im_router_desc* desc, const void* z, const uint32_t* valid,
                             const int32_t* expert, const float* dweight, void* dz, int32_t* error, void* stream);

/* ---- rows to experts and back --------------------------------------------------
 * The grouped layers take each expert's rows in one range. A pair is a row i and
 * its choice c; im_dispatch_plan orders the pairs by expert (those of one expert
 * by i, then c) and tells each its place:
 *   expert  int32 [n_rows x top_k]: -1 goes nowhere; the same expert may come twice
 *   offsets int32 [n_experts + 1] out: the groups' CSR
 *   slot    int32 [n_rows x top_k] out: place of the pair, or -1
 * IM_ERR_ACTION: an expert outside [-1, n_experts); it counts as -1.
 *   n_rows in [0, IM_MAX_ROWS], n_rows top_k at most IM_MAX_ROWS; top_k in [1,
 *   IM_MAX_TOP_K]; n_experts in [1, IM_MAX_GROUPS] (the plan's only); dim in [1, IM_MAX_DIM]
 *   dtype   of rows: IM_F32, IM_BF16, or IM_CODES for the int8 codes of packed
 *           rows (im_dispatch_forward only; their scales go as rows of one float)
 *   ld_row  row stride of what has n_rows rows (x, dx, y, dy)
 *   ld_slot row stride of what has n_slots rows (xs, dxs, ys), ld_dslot of dys
 *   n_slots rows of those, in [0, IM_MAX_ROWS]
 * In the other calls slots are the plan's: no place twice. IM_ERR_ACTION: a slot
 * outside [-1, n_slots); it counts as -1. Places that no slot names are neither read
 * nor written. Sums run over c in order, in fp32. */
#define IM_CODES 2
typedef struct {
  int32_t n_rows, top_k, n_experts, n_slots, dim, dtype;
  int64_t ld_row, ld_slot, ld_dslot;
} im_dispatch_desc;

im_status im_dispatch_workspace(const im_dispatch_desc* desc, int64_t* bytes);
im_status im_dispatch_plan(const im_dispatch_desc* desc, const int32_t* expert, int32_t* offsets, int32_t* slot,
                           void* workspace, int64_t workspace_bytes, int32_t* error, void* stream);
/* xs[slot_ic] = x_i */
im_status im_dispatch_forward(const im_dispatch_desc* desc, const void* x, const int32_t* slot, void* xs,
                              int32_t* error, void* stream);
/* dx_i = sum_c dxs[slot_ic] */
im_status im_dispatch_backward(const im_dispatch_desc* desc, const void* dxs, const int32_t* slot, void* dx,
                               int32_t* error, void* stream);
/* y_i = sum_c weight_ic ys[slot_ic] (a row with no slot: 0); weight fp32 [n_rows x top_k] */
im_status im_combine_forward(const im_dispatch_desc* desc, const void* ys, const int32_t* slot, const float* weight,
                             void* y, int32_t* error, void* stream);
/* dys[slot_ic] = weight_ic dy_i, dweight_ic = dy_i . ys[slot_ic] (0 without a slot);
 * dys or dweight may be NULL to skip it (ys is read for dweight only, weight for dys) */
im_status im_combine_backward(const im_dispatch_desc* desc, const void* dy, const void* ys, const int32_t* slot,
                              const float* weight, void* dys, float* dweight, int32_t* error, void* stream);

/* ---- rows in 8 bits -----------------------------------------------------------
 * A packed row is int8 codes in [-127, 127] and a scale: x_j = scale code_j.
 *   scale = max |x_j| / 127 (at least 2^-126), code = x_j (1 / scale), rounded to
 *   nearest even, every operation in fp32
 * so that |x_j - scale code_j| <= scale / 2 (and a few units of fp32; the largest float itself comes back as
 * infinity, which 127 scales are then). keep: what is not
 * zero gets the code 1 or -1 at least, so that a kept ReLU output says where it was above
 * zero (off by less than a scale there). A row with a value that is not finite has
 * the scale NaN and codes 0.
 * Weights are packed by their outputs: [n_groups out_dim] rows of in_dim.
 *   n_rows in [0, IM_MAX_ROWS]; dim in [1, IM_MAX_DIM]; dtype im_dtype of x
 *   ld_x, ld_codes   row strides (elements) */
typedef struct {
  int32_t n_rows, dim, dtype, keep;
  int64_t ld_x, ld_codes;
} im_rows_desc;

im_status im_rows_pack(const im_rows_desc* desc, const void* x, int8_t* codes, float* scale, void* stream);
/* x = scale code in fp32, rounded to its type */
im_status im_rows_unpack(const im_rows_desc* desc, const int8_t* codes, const float* scale, void* x, void* stream);

/* The grouped layers on packed rows. desc as for im_linear_*, with dtype that of what
 * is not packed (y; dy, W, dx, dW) and ld_x the row stride of the codes.
 * forward: y_i = act(x_scale_i W_scale_gj (sum_k x_ik W_gjk) + b_gj), a product of
 * 8-bit integers whose sum is exact; x and W are codes, W [n_groups x out_dim x in_dim]
 * contiguous, W_scale fp32 [n_groups x out_dim]. In fp32 the sum is multiplied by x_scale first: where that
 * passes the largest float, y is infinite however small W_scale is.
 * backward: the gradients of im_linear_backward with x in 8 bits, as it was kept
 * (IM_BF16: scale code is rounded to bf16 where it enters the product of dW, 2^-8 of it at
 * most, which rounding to the code left already of the largest); relu_in: dx is zero where the code is not above 0. */
im_status im_linear_workspace_packed(const im_linear_desc* desc, int32_t backward, int64_t* bytes);
im_status im_linear_forward_packed(const im_linear_desc* desc, const int32_t* offsets, const int8_t* x,
                                   const float* x_scale, const int8_t* W, const float* W_scale, const float* b,
                                   void* y, void* workspace, int64_t workspace_bytes, int32_t* error, void* stream);
im_status im_linear_backward_packed(const im_linear_desc* desc, const int32_t* offsets, const void* dy,
                                    const int8_t* x, const float* x_scale, const void* W, void* dx, void* dW,
                                    float* db, void* workspace, int64_t workspace_bytes, int32_t* error,
                                    void* stream);

/* Description of the calling thread's last failed call of this header. Never NULL. */
const char* im_learn_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* INFRAMIND_LEARN_H */
