/*
 * lrcnn.h -- row-centric CNN training (LR-CNN, arXiv 2401.11471) on one
 * AMD Instinct MI355X (gfx950).
 *
 * The paper re-orders the training of a convolution stack from layer order
 * ("column") to row order (Section III-A, Eqs. (4)-(5), Algorithm 1): the
 * input is split into horizontal row bands, every band is pushed through all
 * layers before the next one starts, and the feature maps of a band are
 * dropped as soon as the band is done. Backward propagation walks the bands
 * in reverse, recomputes each band's feature maps (Algorithm 1, BP loop) and
 * accumulates the weight gradients g^l over bands. Convolution windows that
 * straddle two bands (the "weak dependency", Section III-B) are handled in
 * one of two ways:
 *   LRCNN_CARRY      two-phase sharing (Section IV-A): rows of a feature map
 *                    that a later band still needs are kept when the band
 *                    that computed them finishes, and reused in FP and BP;
 *                    in BP the error that a band sends to rows owned by an
 *                    earlier band is carried to that band in float32.
 *   LRCNN_RECOMPUTE  overlapping partitioning (Section IV-B): the last layer
 *                    is split evenly and every band recomputes its whole
 *                    receptive cone; each band back-propagates only its own
 *                    rows of the upstream gradient and the partial gradients
 *                    are summed (exact, by linearity).
 * Padding is "semi-closed" (Section III-B): only the true image top and
 * bottom are padded; band edges always see real rows.
 *
 * Results equal ordinary layer-by-layer training up to float rounding.
 *
 * Conventions for every entry point:
 *  - Return value: LRCNN_OK (0) or a negative lrcnn_status; the message of the
 *    last error on the calling thread is returned by lrcnn_last_error().
 *  - Device pointers are caller-owned device memory (hipMalloc or a torch
 *    tensor); the library never allocates or frees device memory and never
 *    synchronises: all work is enqueued on `stream` (a hipStream_t; NULL is
 *    the default stream).
 *  - Tensors are dense NHWC: x is [B][H][W][C_in], y / dy are the last node's
 *    output [B][H_L][W_L][C_L]. Weights are [C_out][kh][kw][C_in].
 *    Storage type is the plan's dtype (float32 or bfloat16) for x, y, dy, dx
 *    and weights; affine scale/shift and weight gradients are float32.
 *  - Per-node arrays (w, aff_scale, aff_shift, dw, mask_out) are HOST arrays
 *    of n_nodes device pointers indexed by node id; entries of nodes they do
 *    not apply to are ignored and may be NULL.
 *  - Device pointers must be 16-byte aligned.
 *  - A plan must not be used from two streams or threads at once.
 */
#ifndef LRCNN_H
#define LRCNN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LRCNN_OK = 0,
  LRCNN_EINVAL = -1,      /* null pointer, bad enum, misaligned pointer      */
  LRCNN_ESHAPE = -2,      /* inconsistent graph or a layer with no output    */
  LRCNN_EPARTITION = -3,  /* band bounds not monotone / out of range         */
  LRCNN_EWORKSPACE = -4,  /* workspace smaller than the plan requires        */
  LRCNN_ESTATE = -5,      /* backward_rows without a matching forward_rows   */
  LRCNN_EDTYPE = -6,      /* unsupported dtype                               */
  LRCNN_EHIP = -7,        /* a HIP launch failed                             */
  LRCNN_EINFEASIBLE = -8  /* no band count fits the memory budget            */
} lrcnn_status;

/* Node kinds. Nodes are given in topological order; node 0 is the input. */
enum {
  LRCNN_OP_INPUT = 0,
  LRCNN_OP_CONV = 1,    /* bias-free cross-correlation, Eq. (1); optional  */
                        /* per-channel affine (fixed BatchNorm) and ReLU    */
  LRCNN_OP_MAXPOOL = 2, /* kh x kw window, stride, -inf padding             */
  LRCNN_OP_ADD = 3      /* elementwise in0 + in1 (residual), optional ReLU */
};

typedef struct {
  int32_t op;
  int32_t in0, in1;          /* producer node ids (in1 only for ADD), else -1 */
  int32_t c_out;             /* CONV output channels (ignored otherwise)      */
  int32_t kh, kw, sh, sw, ph, pw;
  int32_t affine;            /* CONV: out = scale[c] * conv + shift[c]       */
  int32_t relu;              /* CONV / ADD: ReLU after affine / sum           */
} lrcnn_node;

enum { LRCNN_F32 = 0, LRCNN_BF16 = 1 };
enum { LRCNN_CARRY = 0, LRCNN_RECOMPUTE = 1 };
/* Band placement. CARRY bands are ranges of input rows (Algorithm 1 splits
 * the input); RECOMPUTE bands are ranges of the last node's rows (the paper
 * divides the last layer evenly, Section IV-B).
 *   EVEN       r * H / N boundaries
 *   BALANCED   CARRY only: boundaries that minimise the peak workspace of
 *              the step (the skew of Section IV-A)
 *   EXPLICIT   the caller's `bounds` (n_bands + 1 non-decreasing values from
 *              0 to the partitioned height; empty bands are allowed)
 *   PAPER_2PS  CARRY only: the greedy partition of two-phase sharing
 *              (Section IV-A, Eqs. (11), (13), (14)). Band r must complete
 *              t_r rows of the last node: t_1 = first_rows (H_1^L; 0 reads
 *              as ceil(H_L / N_BP)), the remaining H_L - t_1 rows are split
 *              evenly over bands 2..N_BP. A band's end is the smallest input
 *              row count from which the frontier of the last node reaches
 *              t_r -- for a chain of layers exactly the input height that
 *              Eq. (11) (first band) and Eq. (13) (middle bands) give by
 *              inverting the layers from the last one; the last band takes
 *              the remaining input rows (Eq. (14)). The partition is made
 *              for the backward bands (N_BP = n_bands * bp_refine, as the
 *              paper sizes it for BP); the forward bands are every
 *              bp_refine-th of them. */
enum { LRCNN_EVEN = 0, LRCNN_BALANCED = 1, LRCNN_EXPLICIT = 2, LRCNN_PAPER_2PS = 3 };
enum { LRCNN_HYBRID_AUTO = -1 };

typedef struct {
  int32_t batch, in_c, in_h, in_w;
  int32_t dtype;             /* LRCNN_F32 | LRCNN_BF16                        */
  int32_t mode;              /* LRCNN_CARRY | LRCNN_RECOMPUTE                 */
  int32_t n_bands;           /* N >= 1: bands of the forward pass             */
  int32_t policy;            /* LRCNN_EVEN | BALANCED | EXPLICIT | PAPER_2PS  */
  const int32_t *bounds;     /* host array, used when policy == EXPLICIT      */
  int32_t bp_refine;         /* >= 1 (0 reads as 1): the backward pass splits */
                             /* every forward band evenly into bp_refine      */
                             /* bands, N_BP = N * bp_refine (the paper's finer */
                             /* BP granularity, Section III-C)                */
  int32_t hybrid_from;       /* 0: every node row-centric. k in [2, n-1]: the  */
                             /* hybrid variants (2PS-H / OverL-H, checkpoints  */
                             /* integrated with row partitioning, Sections     */
                             /* IV-A and IV-B): nodes 0..k-1 are row-centric,  */
                             /* node k-1 is a checkpoint kept at full size,   */
                             /* nodes k..n-1 run layer-wise over whole maps.  */
                             /* No node >= k may read a node below k-1.        */
                             /* LRCNN_HYBRID_AUTO (-1): the planner takes the  */
                             /* valid k with the smallest workspace (0 if no   */
                             /* checkpoint beats the all-row-centric plan).    */
  int32_t first_rows;        /* PAPER_2PS: H_1^L, rows of the last node that  */
                             /* the first band completes (0: ceil(H_L/N_BP)); */
                             /* ignored by the other policies                 */
} lrcnn_config;

/* Opaque plan handle (host memory only). */
typedef struct lrcnn_plan_s lrcnn_plan_t;

/* Analytic figures of a plan. Byte counts include the batch. */
typedef struct {
  int32_t n_nodes, n_bands, mode, dtype;  /* n_bands: forward bands          */
  int32_t out_h, out_w, out_c;
  size_t workspace_bytes;          /* forward_rows + backward_rows          */
  size_t layerwise_workspace_bytes;/* lrcnn_layerwise_reference_gpu         */
  size_t strip_bytes;              /* CARRY: shared rows kept FP -> BP      */
  size_t band_cache_bytes;         /* largest band's cached feature maps    */
  size_t delta_bytes;              /* float32 error windows (peak)          */
  size_t carry_bytes;              /* CARRY: float32 error carried to r-1   */
  size_t partial_bytes;            /* weight-gradient partial sums          */
  double omega_bytes;              /* Eq. (3): all node outputs, full size  */
  double omega_fp_bytes;           /* Eq. (7) analogue: peak of FP          */
  double omega_bp_bytes;           /* Eq. (8) analogue: peak of BP          */
  double flops_tau;                /* tau (Section IV-B): forward convs     */
  double flops_rows;               /* FLOPs of forward_rows+backward_rows   */
  double flops_layerwise;          /* 3 tau                                 */
  int64_t shared_rows;             /* CARRY: sum of kept rows over bands    */
  int64_t halo_rows;               /* RECOMPUTE: rows computed by more than */
                                   /* one band, summed over nodes and bands */
  int32_t bp_bands;                /* backward bands (n_bands * bp_refine)  */
  size_t fp_window_bytes;          /* forward windows (lifetime-packed when */
                                   /* bp_refine > 1, else the band cache)   */
  int32_t hybrid_from;             /* the checkpoint in use (0: none); the  */
                                   /* planner's choice for LRCNN_HYBRID_AUTO */
} lrcnn_plan_info;

/* Build a plan: shapes of every node, per-band row intervals, workspace
 * layout, analytic memory (Eqs. (3), (7), (8), (12)) and FLOPs (tau,
 * Section IV-B). Pure host code; needs no GPU. `nodes`, `cfg` and
 * `cfg->bounds` are read during the call only. On success *out owns a plan
 * that the caller releases with lrcnn_plan_destroy.
 * Errors: EINVAL (null pointer, bad enum, a hybrid checkpoint that an edge
 * crosses), ESHAPE (bad ids, channel or size mismatch, a layer with empty
 * output), EPARTITION (bad bounds). */
int lrcnn_plan(const lrcnn_node *nodes, int32_t n_nodes,
               const lrcnn_config *cfg, lrcnn_plan_t **out);

/* Fill *info. Errors: EINVAL on null. */
int lrcnn_plan_query(const lrcnn_plan_t *plan, lrcnn_plan_info *info);

/* Output shape of node `node`: shape = {H, W, C}. Errors: EINVAL. */
int lrcnn_plan_node_shape(const lrcnn_plan_t *plan, int32_t node,
                          int32_t shape[3]);

/* Rows of node `node` in band `band` (0-based) of the forward (phase 0) or
 * backward (phase 1) partition: rows[0..1] = the rows the band computes and
 * owns [a, b); rows[2..3] = the rows it holds [lo, hi) (CARRY: own rows plus
 * the rows shared from earlier bands; RECOMPUTE: the band's receptive cone).
 * Errors: EINVAL. */
int lrcnn_plan_band_rows(const lrcnn_plan_t *plan, int32_t phase, int32_t band,
                         int32_t node, int32_t rows[4]);

void lrcnn_plan_destroy(lrcnn_plan_t *plan);

/* Device bytes of one training step under `plan`: the workspace
 * (row-centric, or layer-wise when layerwise != 0) plus the xi of
 * Eqs. (9)-(10) -- every other buffer the step touches: x, y, dy (storage
 * dtype), the weights (storage dtype), their float32 gradients, the float32
 * affine scale and shift, and dx when want_dx != 0. Each buffer is counted
 * at the 256-byte granularity the library uses; a caller's allocator may
 * round further. Errors: EINVAL on null. */
int lrcnn_plan_step_bytes(const lrcnn_plan_t *plan, int32_t layerwise,
                          int32_t want_dx, size_t *bytes);

/* Memory budget of the budget-driven planner and the batch search. */
typedef struct {
  size_t budget_bytes;  /* M: device bytes the step may use               */
  int32_t max_bands;    /* largest N_BP tried; 0: min(256, partitioned   */
                        /* height: input rows in CARRY, output rows in    */
                        /* RECOMPUTE)                                     */
  int32_t max_refine;   /* largest N_BP / N_FP tried (0 reads as 1)       */
  int32_t want_dx;      /* count dx in xi                                 */
} lrcnn_budget;

/* Budget-driven row granularity (Section III-C, Eqs. (9)-(10); the memory
 * bound of 2PS, Eq. (12), and of OverL, Section IV-B): the plan with the
 * smallest backward band count N_BP = N whose step fits the budget
 * (lrcnn_plan_step_bytes(plan, 0, want_dx) <= budget_bytes), and for that
 * N_BP the smallest forward band count N_FP (a divisor of N_BP with
 * N_BP / N_FP <= max_refine). Small N is preferred because it gives the
 * kernels the most parallel work (the paper's second principle). The exact
 * workspace of each candidate plan stands in for the paper's analytic
 * Omega, so the strips, error windows and split-K buffers are counted too.
 * cfg->n_bands and cfg->bp_refine are ignored; cfg->policy must be EVEN,
 * BALANCED or PAPER_2PS. Candidates are tried in increasing (N_BP, N_FP)
 * order, each a full host-side plan (milliseconds). With PAPER_2PS each
 * (N_BP, N_FP) also tries H_1^L from H_L down to ceil(H_L / N_BP) and takes
 * the largest that fits (Eq. (12): the largest first band, the fewest
 * bands); cfg->first_rows is ignored.
 * Errors: EINVAL (null, EXPLICIT policy, bad budget), the errors of
 * lrcnn_plan, EINFEASIBLE (no candidate up to max_bands fits). */
int lrcnn_plan_for_budget(const lrcnn_node *nodes, int32_t n_nodes,
                          const lrcnn_config *cfg, const lrcnn_budget *budget,
                          lrcnn_plan_t **out);

/* Largest batch whose step fits the budget: the largest B with
 * lrcnn_plan_step_bytes(plan(B), layerwise, want_dx) <= budget_bytes, for
 * the row-centric step of cfg (layerwise == 0) or the layer-wise baseline
 * (layerwise != 0) -- the paper's largest-batch comparison (Section V).
 * cfg->batch is ignored; budget->max_bands and max_refine are unused. The
 * search doubles B until the step no longer fits (at most 2^24), then
 * bisects; step bytes grow with B. On success *batch >= 1.
 * Errors: EINVAL (null), the errors of lrcnn_plan, EINFEASIBLE (B = 1 does
 * not fit). */
int lrcnn_max_batch(const lrcnn_node *nodes, int32_t n_nodes,
                    const lrcnn_config *cfg, int32_t layerwise,
                    const lrcnn_budget *budget, int32_t *batch);

/* Row-centric FP (Algorithm 1, FP loop): writes y. In CARRY mode the rows
 * shared between bands are left in `workspace` for lrcnn_backward_rows.
 * mask_out (nullable host array; entries nullable): per node a device
 * uint8 [B][H][W][C] buffer that receives the ReLU mask (1 where the output
 * is > 0) of CONV/ADD nodes with ReLU and the argmax (row-major index inside
 * the window) of MAXPOOL nodes.
 * Errors: EINVAL, EWORKSPACE (ws_bytes < workspace_bytes), EHIP. */
int lrcnn_forward_rows(lrcnn_plan_t *plan, const void *x,
                       const void *const *w,
                       const float *const *aff_scale,
                       const float *const *aff_shift,
                       void *y, void *workspace, size_t ws_bytes,
                       void *const *mask_out, void *stream);

/* Allocation-free lrcnn_forward_rows, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc). The workspace is the library's own
 * static device array of LRCNN_STATIC_WORKSPACE_BYTES (64 MiB), one per
 * device, held from the library's load until the process ends; its device
 * address is looked up once per device on the first call there. The call
 * allocates no device memory; the caller still owns x, w, aff_*, y and
 * mask_out, with the meaning, layout and results of lrcnn_forward_rows.
 * Every call on a device shares that device's array, which keeps the last
 * call's contents (the forward initialises every row it reads): calls that
 * overlap on one device (several streams or threads) race. A later
 * lrcnn_backward_rows cannot use this forward's shared rows (ESTATE).
 * Errors: as lrcnn_forward_rows; EWORKSPACE when the plan's workspace_bytes
 * exceed LRCNN_STATIC_WORKSPACE_BYTES; EHIP when the array's device address
 * cannot be obtained. */
#define LRCNN_STATIC_WORKSPACE_BYTES (64u << 20)
int lrcnn_forward_rows_static(lrcnn_plan_t *plan, const void *x,
                              const void *const *w,
                              const float *const *aff_scale,
                              const float *const *aff_shift, void *y,
                              void *const *mask_out, void *stream);

/* Row-centric BP (Algorithm 1, BP loop), bands in reverse: recompute each
 * band, propagate the error dy = dL/dy, overwrite dw[node] (float32,
 * [C_out][kh][kw][C_in]) with the weight gradient of every conv node and,
 * when dx != NULL, write dL/dx. CARRY mode needs the workspace of the
 * preceding lrcnn_forward_rows on this plan, unchanged.
 * Errors: EINVAL, EWORKSPACE, ESTATE (CARRY without a preceding forward on
 * this plan and workspace), EHIP. */
int lrcnn_backward_rows(lrcnn_plan_t *plan, const void *x,
                        const void *const *w,
                        const float *const *aff_scale,
                        const float *const *aff_shift,
                        const void *dy, float *const *dw, void *dx,
                        void *workspace, size_t ws_bytes, void *stream);

/* Layer-by-layer ("column", Eqs. (1)-(3)) training step on the GPU with the
 * same kernels: full-height feature maps of every node are kept from FP to
 * BP and nothing is recomputed. Writes y, dw and (if non-NULL) dx and
 * mask_out as above. Needs layerwise_workspace_bytes of workspace.
 * Errors: EINVAL, EWORKSPACE, EHIP. */
int lrcnn_layerwise_reference_gpu(lrcnn_plan_t *plan, const void *x,
                                  const void *const *w,
                                  const float *const *aff_scale,
                                  const float *const *aff_shift,
                                  const void *dy, void *y, float *const *dw,
                                  void *dx, void *workspace, size_t ws_bytes,
                                  void *const *mask_out, void *stream);

/* ---- Full training step: classifier head, loss, update (Algorithm 1:
 * fully connected FP, Loss, fully connected BP after the last band's FP, and
 * the parameter update once every band's BP is done). Readings: one fully
 * connected layer over the trunk output flattened per image in NHWC order
 * (K = H_L * W_L * C_L features), softmax cross-entropy averaged over the
 * batch, plain SGD; the fixed affine parameters are not trained. */

/* Device scratch bytes lrcnn_head_loss needs for n_classes classes (1..64).
 * Errors: EINVAL. */
int lrcnn_head_workspace_bytes(const lrcnn_plan_t *plan, int32_t n_classes,
                               size_t *bytes);

/* y: the trunk output written by lrcnn_forward_rows (plan dtype,
 * [B][H_L][W_L][C_L]); fc_w: float32 [n_classes][K]; fc_b: float32
 * [n_classes]; labels: int32 [B] in [0, n_classes). Writes logits (float32
 * [B][n_classes]), loss (one float32: the batch mean), dy = dL/dy (plan
 * dtype, shape of y: the upstream gradient for lrcnn_backward_rows),
 * d_fc_w and d_fc_b (float32, overwritten). head_ws: device scratch of
 * lrcnn_head_workspace_bytes. A label outside [0, n_classes) makes the loss
 * NaN (nothing is read out of bounds). All device pointers 16-byte aligned.
 * Errors: EINVAL, EWORKSPACE, EHIP. */
int lrcnn_head_loss(const lrcnn_plan_t *plan, const void *y, const float *fc_w,
                    const float *fc_b, const int32_t *labels, int32_t n_classes,
                    float *logits, float *loss, void *dy, float *d_fc_w,
                    float *d_fc_b, void *head_ws, size_t head_ws_bytes,
                    void *stream);

/* theta <- theta - lr * g for every conv node's weights w[v] (plan dtype,
 * updated in float32 and rounded to the storage dtype) with dw[v] (float32,
 * from lrcnn_backward_rows), and, when fc_w is not NULL, for the head
 * (fc_w, fc_b with d_fc_w, d_fc_b; n_classes classes). Errors: EINVAL,
 * EHIP. */
int lrcnn_sgd_update(const lrcnn_plan_t *plan, float lr, void *const *w,
                     float *const *dw, float *fc_w, const float *d_fc_w,
                     float *fc_b, const float *d_fc_b, int32_t n_classes,
                     void *stream);

/* ---- Feed-forward blocks with 8-bit activation checkpoints. What a block keeps
 * from its forward to its backward pass (a norm's input, a linear layer's
 * input, an activation's input) is held in 8 bits a value, and the backward
 * pass reads that. The block's linear products and input gradients are 1x1
 * convolutions (plans above).
 *
 * Further conventions of these entry points:
 *  - A matrix is row-major, `rows` x `cols`, with a row stride ld* in elements
 *    (0: cols, else >= cols). Storage type: `dtype` (float32 or bfloat16).
 *    Matrices and float32 vectors need only their element's alignment;
 *    checkpoints and workspaces 16 bytes. Any width from 1 on, any number of
 *    rows from 0 on.
 *  - An output may be an input of the same call only where both are the same
 *    matrix (pointer, stride and type); other overlaps are not allowed.
 *  - Sums, statistics and activations are computed in float32 and rounded once.
 *    Every sum runs in a fixed order: results are reproducible run to run.
 *  - accumulate != 0: weight gradients are added to what is there (bands,
 *    micro-batches), else overwritten.
 *  - Errors: EINVAL (null or misaligned pointer, arguments that do not go
 *    together), ESHAPE, EDTYPE, EWORKSPACE, EHIP. Nothing is enqueued by a
 *    call that refuses its arguments.
 *
 * The checkpoint of a matrix is one buffer of lrcnn_act8_bytes bytes:
 * codes int8 [rows][pitch], pitch = cols rounded up to 32 (zeros behind the
 * last column); then, from the next multiple of 256 bytes, exponent bytes
 * [rows][pitch / 32], one for each group of 32 columns. With m the group's
 * largest magnitude and bits(m) its float32 bits,
 *   E = max((bits(m) + 2^16) >> 23, 7),  code = rint(x * 2^(133 - E)),
 * the code (ties to even) within [-127, 127], and the value stands for
 * code * 2^(E - 133): within 2^(E - 134) of x. E is at most 254 (codes are then
 * held to +-127); a group with an infinity or a NaN has E = 255, codes 0, and
 * stands for NaN. The values are exact in bfloat16 and float32. */

/* Bytes of the checkpoint of a rows x cols matrix. */
int lrcnn_act8_bytes(int64_t rows, int64_t cols, size_t *bytes);

/* Checkpoint of x. */
int lrcnn_act8_pack(int64_t rows, int64_t cols, int32_t dtype, const void *x,
                    int64_t ldx, void *ckpt, void *stream);

/* y = what the checkpoint stands for (in `dtype`, whatever it was packed
 * from). */
int lrcnn_act8_unpack(int64_t rows, int64_t cols, int32_t dtype,
                      const void *ckpt, void *y, int64_t ldy, void *stream);

/* Layer norm of each row: t = x, or x + residual rounded to the storage type
 * (written to `total` where not NULL);
 *   xh = (t - mean) * rstd, rstd = 1 / sqrt(var + eps), y = gamma * xh + beta.
 * gamma, beta: float32 [cols], NULL for 1 and 0. mean, rstd: float32 [rows],
 * nullable. ckpt (nullable): receives the checkpoint of xh, which serves both
 * lrcnn_layer_norm_backward and, with gamma and beta as scale and shift, the
 * lrcnn_linear_wgrad of a linear layer that reads y. cols <= 16384. */
int lrcnn_layer_norm_forward(int64_t rows, int64_t cols, int32_t dtype,
                             const void *x, int64_t ldx, const void *residual,
                             int64_t ldr, const float *gamma, const float *beta,
                             float eps, void *total, int64_t ldt, void *y,
                             int64_t ldy, float *mean, float *rstd, void *ckpt,
                             void *stream);

/* Device scratch bytes of lrcnn_layer_norm_backward. */
int lrcnn_layer_norm_workspace_bytes(int64_t rows, int64_t cols, size_t *bytes);

/* Gradients of the layer norm from dy = dL/dy and either its input x (the sum
 * with the residual, where there was one) with mean, or ckpt; and rstd:
 *   g = gamma * dy, dx = rstd * (g - mean(g) - xh * mean(g * xh)) [+ dres],
 *   dgamma = sum over rows of dy * xh, dbeta = sum over rows of dy.
 * dres (nullable): the gradient that reaches t past the norm. dgamma, dbeta:
 * float32 [cols], each nullable (workspace may be NULL if both are). */
int lrcnn_layer_norm_backward(int64_t rows, int64_t cols, int32_t dtype,
                              const void *dy, int64_t lddy, const void *x,
                              int64_t ldx, const float *mean, const void *ckpt,
                              const float *rstd, const float *gamma,
                              const void *dres, int64_t lddr, void *dx,
                              int64_t lddx, float *dgamma, float *dbeta,
                              int32_t accumulate, void *workspace,
                              size_t ws_bytes, void *stream);

/* Activations: relu; gelu, x * Phi(x); its tanh form; silu, x / (1 + e^-x);
 * none, x itself, where a call says that it takes it. */
enum {
  LRCNN_ACT_NONE = -1,
  LRCNN_ACT_RELU = 0,
  LRCNN_ACT_GELU = 1,
  LRCNN_ACT_GELU_TANH = 2,
  LRCNN_ACT_SILU = 3
};

/* a = f(u), or f(u) * v where v is not NULL (gated). Writes any of a and the
 * checkpoints of u, v and a (nullable, at least one given; the checkpoint of a
 * is formed from its float32 value). */
int lrcnn_activation_forward(int64_t rows, int64_t cols, int32_t dtype,
                             int32_t kind, const void *u, int64_t ldu,
                             const void *v, int64_t ldv, void *a, int64_t lda,
                             void *ckpt_u, void *ckpt_v, void *ckpt_a,
                             void *stream);

/* du = da * f'(u) [* v], dv = da * f(u), from u (and v), or from their
 * checkpoints in place of them. ckpt_a (nullable): receives the checkpoint of
 * f(u) [* v], the input of the linear layer behind the activation, for
 * its lrcnn_linear_wgrad. f'(0) of relu is 0. */
int lrcnn_activation_backward(int64_t rows, int64_t cols, int32_t dtype,
                              int32_t kind, const void *da, int64_t ldda,
                              const void *u, int64_t ldu, const void *v,
                              int64_t ldv, const void *ckpt_u,
                              const void *ckpt_v, void *du, int64_t lddu,
                              void *dv, int64_t lddv, void *ckpt_a,
                              void *stream);

/* Device scratch bytes of lrcnn_linear_wgrad for up to `rows` rows (0: none,
 * NULL will do). Never less than for fewer rows: the workspace of the largest
 * band or micro-batch serves all of them. */
int lrcnn_linear_wgrad_workspace_bytes(int64_t rows, int64_t n_in,
                                       int64_t n_out, int32_t dtype,
                                       size_t *bytes);

/* Weight and bias gradient of a linear layer y = x W^T + b, W [n_out][n_in],
 * from dy = dL/dy (rows x n_out) and a checkpoint (rows x n_in) of q with
 * x = scale * q + shift per column (float32 [n_in], NULL for 1 and 0):
 *   dw[n][k] = sum over rows of dy[.][n] * x[.][k]   (float32, dense)
 *   db[n]    = sum over rows of dy[.][n]             (float32, nullable)
 * Products are exact, sums float32, for either dtype of dy; but of a float32 dy
 * what bfloat16 numbers cannot hold, 2^-134 at most, is lost. A value of dy that
 * is not finite makes its row of dw, and its db, not finite (NaN where the
 * exact sum may be an infinity); a group of the checkpoint that stands for NaN
 * makes its 32 columns of dw NaN. ESHAPE beyond 2^24 features, 2^30 rows, a
 * row stride of dy of 2^24, or 2^24 tiles of 128 x 128 of dw. */
int lrcnn_linear_wgrad(int64_t rows, int64_t n_in, int64_t n_out,
                       int32_t dtype, const void *dy, int64_t lddy,
                       const void *ckpt, const float *scale,
                       const float *shift, float *dw, float *db,
                       int32_t accumulate, void *workspace, size_t ws_bytes,
                       void *stream);

/* ---- Group norm of a feature map, dropout and the gated feed-forward block. The
 * conventions of the entry points above hold. */

/* Device scratch bytes of lrcnn_group_norm_forward and _backward. Never less
 * than for fewer images or pixels: the workspace of the largest batch or band
 * serves all of them. */
int lrcnn_group_norm_workspace_bytes(int64_t batch, int64_t pixels,
                                     int64_t channels, int64_t groups,
                                     size_t *bytes);

/* Group norm with an activation, channels last: x is a map of `batch` images of
 * `pixels` pixels, a matrix of batch * pixels rows and `channels` columns.
 * Channels go by `groups` equal runs of neighbours; over the pixels and
 * channels of one group of one image
 *   xh = (x - mean) * rstd, rstd = 1 / sqrt(var + eps),
 *   y = f(gamma * xh + beta).
 * kind: f, an activation or LRCNN_ACT_NONE. gamma, beta: float32 [channels],
 * NULL for 1 and 0. mean, rstd: float32 [batch][groups], nullable. ckpt
 * (nullable): receives the checkpoint of xh, for lrcnn_group_norm_backward.
 * Without images or pixels nothing is written. ESHAPE where groups does not
 * divide channels, or beyond 2^20 images or channels, 2^21 images times groups
 * or 2^23 images times tiles of 512 channels. */
int lrcnn_group_norm_forward(int64_t batch, int64_t pixels, int64_t channels,
                             int64_t groups, int32_t dtype, int32_t kind,
                             const void *x, int64_t ldx, const float *gamma,
                             const float *beta, float eps, void *y, int64_t ldy,
                             float *mean, float *rstd, void *ckpt,
                             void *workspace, size_t ws_bytes, void *stream);

/* Gradients of the group norm with its activation from dy = dL/dy and either
 * its input x with mean, or ckpt; and rstd:
 *   e = dy * f'(gamma * xh + beta), q = gamma * e,
 *   dx = rstd * (q - mean(q) - xh * mean(q * xh)), means over the group,
 *   dgamma = sum over rows of e * xh, dbeta = sum over rows of e.
 * dgamma, dbeta: float32 [channels], each nullable; their sums over slabs and
 * images are in 64 bits. Without images or pixels they are zero, or where they are
 * added to as they were. */
int lrcnn_group_norm_backward(int64_t batch, int64_t pixels, int64_t channels,
                              int64_t groups, int32_t dtype, int32_t kind,
                              const void *dy, int64_t lddy, const void *x,
                              int64_t ldx, const float *mean, const void *ckpt,
                              const float *rstd, const float *gamma,
                              const float *beta, void *dx, int64_t lddx,
                              float *dgamma, float *dbeta, int32_t accumulate,
                              void *workspace, size_t ws_bytes, void *stream);

/* Dropout whose mask is never stored: y = x * keep / (1 - p) [+ residual],
 * rounded once; the backward pass is the same call on the gradient, without the
 * residual. A dropped element counts as 0, whatever x holds there.
 * rng: two 64-bit numbers in device memory, {seed, offset}, read by the kernel:
 * a program advances the offset from step to step, also between replays of a
 * captured graph. site, in [0, 65536): tells the dropouts of one step apart.
 * first_row: the matrix' first row within a larger one, so that bands and
 * micro-batches draw what the whole would.
 * Random bits: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011) with the
 * seed's halves as key and, for g = (first_row + row) * ceil(cols / 8) + col / 8,
 * the counter (g's low word, g >> 32 | site << 16, the offset's halves). Column c
 * takes 16 bits of word (c % 8) / 2, the low ones where c is even, and is
 * dropped where they are less than rint(65536 p); keep / (1 - p) is with that
 * share. p in [0, 1]. ESHAPE where g could reach 2^48. */
int lrcnn_dropout(int64_t rows, int64_t cols, int32_t dtype, const void *x,
                  int64_t ldx, const void *residual, int64_t ldr, double p,
                  const uint64_t *rng, int32_t site, int64_t first_row, void *y,
                  int64_t ldy, void *stream);

/* Gated feed-forward block:
 *   u = x Wu^T + bu, v = x Wv^T + bv, a = f(u) * v, z = a W2^T + b2.
 * Both projections, the activation and the product are one kernel; z is a second
 * one on `a` as stored. w1 [2 hidden][n_in] holds Wu, then Wv; w2
 * [n_out][hidden]; both dense, of the matrices' type. b1 float32 [2 hidden], b2
 * float32 [n_out], nullable. z may be NULL (w2 and b2 are not read then, n_out is
 * ignored). For the backward pass, each nullable: uv [rows][2 hidden] receives u
 * and v; ckpt_u, ckpt_v the checkpoints of their float32 values. In place: z may
 * be x; a and uv may not, nor z a: EINVAL.
 * ESHAPE beyond 2^24 features or 2^30 rows, and from 2^22 tiles of 128 x 128 of
 * x, [u v] or z on. */
int lrcnn_gated_ffn_forward(int64_t rows, int64_t n_in, int64_t hidden,
                            int64_t n_out, int32_t dtype, int32_t kind,
                            const void *x, int64_t ldx, const void *w1,
                            const float *b1, void *a, int64_t lda, void *uv,
                            int64_t lduv, void *ckpt_u, void *ckpt_v,
                            const void *w2, const float *b2, void *z,
                            int64_t ldz, void *stream);

/* Backward pass of the block from dz = dL/dz:
 *   da = dz W2, du = da * f'(u) * v, dv = da * f(u), dx = [du dv] W1,
 * the first three in one kernel, dx from du and dv as stored. u and v come from
 * uv or from their checkpoints (exactly one of the two). w2t [hidden][n_out] and
 * w1t [n_in][2 hidden] are the transposed weights, dense. duv [rows][2 hidden]
 * receives du and dv; ckpt_a (nullable) the checkpoint of f(u) * v; dx (NULL: not
 * wanted, w1t is not read then, n_in is ignored). The weights' gradients are
 * lrcnn_linear_wgrad's: of w2 from dz and ckpt_a, of w1 from duv and the
 * checkpoint of x. In place: duv may be uv (with uv's stride, else EINVAL), dx may be
 * dz or uv (not where that is duv), ckpt_a may be ckpt_u or ckpt_v; duv may not be
 * dz: EINVAL. ESHAPE as in the forward pass, by dz, [du dv] and dx. */
int lrcnn_gated_ffn_backward(int64_t rows, int64_t n_in, int64_t hidden,
                             int64_t n_out, int32_t dtype, int32_t kind,
                             const void *dz, int64_t lddz, const void *w2t,
                             const void *uv, int64_t lduv, const void *ckpt_u,
                             const void *ckpt_v, void *duv, int64_t ldduv,
                             void *ckpt_a, const void *w1t, void *dx,
                             int64_t lddx, void *stream);

/* Message of the last failed call on this thread ("" if none). */
const char *lrcnn_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* LRCNN_H */
