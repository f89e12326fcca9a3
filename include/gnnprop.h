/*
 * gnnprop -- GraphSAGE feature propagation on a sampled subgraph, forward
 * and backward, on AMD Instinct MI355X (gfx950).
 *
 * The operations follow "Accurate, Efficient and Scalable Training of Graph
 * Neural Networks" (Zeng, Zhou, Srivastava, Kannan, Prasanna):
 *   - one layer's forward, Section 2.1, Eq. "graphsage forward":
 *       Y = ReLU( X W_self || A_s X W_neigh )      (self half first)
 *     with A_s the subgraph's normalised adjacency (D^-1 A for GraphSAGE);
 *   - its backward, Section 5.1, Eq. "gcn backward";
 *   - the three kernels Section 5.1 names: sparse feature / gradient
 *     propagation (CSR SpMM), dense weight transformation (GEMM on the
 *     matrix cores), and the sparse adjacency transpose (Section 5.2,
 *     Algorithm 6);
 *   - the computation-order choice of Section 6.1.
 *
 * Conventions for every entry point
 *   - Pointers named as device pointers must point to memory of the current
 *     HIP device; the library never takes ownership and never frees them.
 *   - Dense matrices are row-major fp32 with an explicit leading dimension
 *     (row stride, in elements, >= the row width).  Any 4-byte-aligned
 *     pointer and any stride is accepted; 16-byte alignment of the base and a
 *     stride that is a multiple of 4 enable the vector paths.
 *   - Work is enqueued on `stream` (NULL = the null stream) and is complete
 *     once the stream is synchronised.  Only gnn_csr_validate synchronises.
 *   - Argument errors are reported synchronously, before anything is
 *     enqueued; a failed launch returns GNN_ERR_HIP.  Nothing is printed and
 *     no C++ exception crosses this interface.
 *   - Outputs are overwritten, never accumulated into.  Inputs and outputs
 *     must not overlap unless an entry point says otherwise.
 *   - gnn_prop_fwd / gnn_prop_bwd / gnn_spmm / gnn_gemm allocate no device
 *     memory: scratch comes from the caller's `workspace`.
 *   - `workspace`, `saved` and plan buffers (csr->plan included) must start
 *     16-byte aligned, as hipMalloc memory does; any other address is
 *     GNN_ERR_UNSUPPORTED.
 */
#ifndef GNNPROP_H
#define GNNPROP_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum gnn_status {
  GNN_OK = 0,
  GNN_ERR_NULL = -1,        /* a required pointer is NULL */
  GNN_ERR_SHAPE = -2,       /* a size or leading dimension is invalid */
  GNN_ERR_CSR = -3,         /* gnn_csr_validate found an invalid CSR */
  GNN_ERR_UNSUPPORTED = -4, /* option not supported */
  GNN_ERR_WORKSPACE = -5,   /* workspace or plan buffer too small */
  GNN_ERR_HIP = -6,         /* a HIP runtime call or launch failed */
  GNN_ERR_ALIAS = -7        /* outputs overlap inputs where forbidden */
} gnn_status;

/* Layer flags. */
/* GEMM products.  By default every fp32 operand of a weight transformation
 * is split exactly into three bf16 pieces (x = hi + mid + lo, each rounded
 * to nearest even) and the six piece products down to 2^-16 of hi x hi are
 * accumulated in fp32 on the bf16 matrix cores: fp32 operands, results and
 * accumulation, with a product error below 2^-24 relative (measured against
 * fp64: no larger than that of the fp32 matrix-core instruction).  Operands
 * must be finite and below bf16's largest finite value (about 3.39e38) in
 * magnitude: an infinite operand makes its outputs NaN where the fp32
 * instruction gives infinities (use GNN_FLAG_F32_MFMA for such data).  The
 * two flags below select other arithmetic; setting both is
 * GNN_ERR_UNSUPPORTED. */
#define GNN_FLAG_BF16 0x1u /* GEMM operands rounded to bf16 (round to nearest
                              even), fp32 accumulation; the aggregation sums
                              in fp32 (in the backward pass its output T and
                              the mask's G_s are kept in the workspace already
                              rounded, as only the GEMMs read them); all
                              outputs fp32 */
#define GNN_FLAG_F32_MFMA 0x8u /* GEMM products on the fp32 matrix-core
                                  instruction (v_mfma_f32_32x32x2_f32) */
/* GraphSAGE layers only (gnn_prop_fwd / gnn_prop_bwd).  Section 2.1 defines
 * the layer's A_s as D^-1 A, D the diagonal of A's row sums; with this flag
 * the aggregations take A_s from the pattern alone, A the 0/1 matrix of the
 * stored entries (self loops as stored) and deg(v) = indptr[v+1] - indptr[v]:
 * the forward sums each row's neighbour rows unweighted and scales the sum
 * by 1/deg(v), the transposed aggregation weighs entry (u, v) by 1/deg(v)
 * (the value (A_s)^T holds there when the pattern is symmetric, as the
 * backward pass requires anyway).  csr->values and csr->values_t are then
 * not read and may be NULL.  Results equal those of the same call with
 * values = 1/deg in float (values_t from gnn_csr_transpose_values) up to
 * rounding: the forward rounds the sum before the scaling. */
#define GNN_FLAG_ROW_NORMALIZED 0x10u
/* Backward pass only (Algorithm 1's layer loop, backward direction): the
 * layers of a stack share their ReLU masks.  Layer l's input X is layer
 * l-1's output, so 1[X > 0] is layer l-1's mask and can be applied where
 * layer l produces dX; layer l-1 then receives its G directly. */
#define GNN_FLAG_DY_MASKED 0x2u /* dY is already G = dY * 1[Y > 0]: no
                                   masking pass, dY is read in place */
#define GNN_FLAG_DX_MASKED 0x4u /* dX is written as dX * 1[X > 0] (selected,
                                   not multiplied), i.e. the next layer
                                   down's G when X is that layer's output */

/* The sampled subgraph's adjacency A_s in CSR (Section 5.2: Indptr,
 * Indices, Data).  All arrays are device memory.
 *   indptr  [n+1]  indptr[0] = 0, non-decreasing, indptr[n] = nnz
 *   indices [nnz]  column ids in [0,n), ascending within each row
 *   values  [nnz]  A_s entries (any values; D^-1 A for GraphSAGE)
 *   values_t[nnz]  entries of (A_s)^T on the same indptr/indices, from
 *                  gnn_csr_transpose_values; needed by the backward pass
 *                  and by gnn_spmm with transpose = 1.  The transpose reuses
 *                  indptr/indices, so the pattern must be symmetric
 *                  (undirected subgraph, Section 5.2).
 *   plan           device buffer written by gnn_csr_build_plan (or
 *                  gnn_csr_prepare): per window of 256 stored entries the
 *                  rows whose first entry lies in it and their entry range,
 *                  and the row of every entry. */
typedef struct gnn_csr {
  int32_t n;
  int64_t nnz;
  const int32_t* indptr;
  const int32_t* indices;
  const float* values;
  const float* values_t;
  const void* plan;
} gnn_csr;

/* One layer's shape.  X is n x f_in (stride ld_x); Y and dY are n x 2h
 * (stride ld_y), self half in columns [0,h), neighbour half in [h,2h);
 * dX is n x f_in (stride ld_dx); W_self and W_neigh are f_in x h, dense
 * row-major (stride h); biases are [h].
 *   order: 0 = choose by gnn_choose_order, 1 = (A_s X) W_neigh,
 *          2 = A_s (X W_neigh).  Both orders compute the same values. */
typedef struct gnn_layer {
  int32_t f_in;
  int32_t h;
  int64_t ld_x;
  int64_t ld_y;
  int64_t ld_dx;
  int32_t order;
  uint32_t flags;
} gnn_layer;

/* Human-readable name of a status code (static storage). */
const char* gnn_status_string(gnn_status s);

/* Section 6.1: for A (sparse n x n) . W1 (n x f1) . W2 (f1 x f2), order 1
 * (A W1) W2 costs delta n^2 f1 + n f1 f2 multiply-adds and order 2
 * A (W1 W2) costs delta n^2 f2 + n f1 f2.  Returns 1 when f1 <= f2 (ties go
 * to order 1), else 2.  For a layer, f1 = f_in and f2 = h. */
int32_t gnn_choose_order(int32_t f_in, int32_t h);

/* ---------------------------------------------------- per-subgraph prep */

/* Section 5.2, Algorithm 6: values of (A_s)^T on the pattern of A_s.  For
 * each stored (v,u), writes values[pos(v,u)] to values_t[pos(u,v)]; a pure
 * permutation, bit-exact.  Requires csr->indptr/indices/values; the pattern
 * must be symmetric with ascending indices per row (check with
 * gnn_csr_validate).  values_t is device memory of nnz floats.  If
 * csr->plan is non-NULL it must hold this graph's plan (gnn_csr_build_plan,
 * enqueued before), whose per-entry rows then give one thread to each
 * entry; with plan == NULL one wavefront handles each row. */
gnn_status gnn_csr_transpose_values(const gnn_csr* csr, float* values_t,
                                    hipStream_t stream);

/* Bytes of the aggregation work plan for a graph of n rows and nnz entries. */
size_t gnn_plan_bytes(int32_t n, int64_t nnz);

/* Builds the aggregation work plan into `plan` (device memory of at least
 * gnn_plan_bytes(n, nnz) bytes).  The stored entries are cut into windows of
 * 256; window k gets the rows whose first entry lies in it (so a row, hub
 * rows included, is never shared between windows) and their entry range,
 * and every entry its row.  The aggregation gives each window to one
 * workgroup and splits its entries evenly over lane groups; the parts of a
 * row cut between groups are added in a fixed order, so results are
 * deterministic.  Reads csr->n, nnz and indptr. */
gnn_status gnn_csr_build_plan(const gnn_csr* csr, void* plan,
                              size_t plan_bytes, hipStream_t stream);

/* Both per-subgraph preparations (Section 5.2) in one launch: the plan of
 * gnn_csr_build_plan into `plan` (plan_bytes >= gnn_plan_bytes) and the
 * transposed values of gnn_csr_transpose_values into values_t (nnz floats).
 * The results are bit for bit those of the two separate calls.  The
 * pattern must be symmetric with ascending indices per row; csr->values_t
 * and csr->plan are not read.  plan and values_t may not overlap each
 * other or the CSR arrays (GNN_ERR_ALIAS). */
gnn_status gnn_csr_prepare(const gnn_csr* csr, void* plan, size_t plan_bytes,
                           float* values_t, hipStream_t stream);

/* Checks the CSR on the device and synchronises `stream`: indptr
 * monotone with indptr[0] = 0 and indptr[n] = nnz, indices in range and
 * strictly ascending per row, and, if require_symmetric, that every stored
 * (v,u) has a stored (u,v).  Returns GNN_OK or GNN_ERR_CSR.  May allocate a
 * few bytes of device memory. */
gnn_status gnn_csr_validate(const gnn_csr* csr, int32_t require_symmetric,
                            hipStream_t stream);

/* gnn_csr_validate for callers that cannot allocate device memory (serving
 * loops, harnesses that forbid hipMalloc): the same checks and the same
 * result, with the status word the check writes kept in a 256-byte array
 * of static device memory that the library holds on each device it runs on
 * until the process ends, instead of a hipMalloc'd word.  That scratch does
 * not grow with the graph, so no size limit applies beyond those of
 * gnn_csr_validate.  Every call on one device shares the array (each call
 * clears it first): calls that overlap on one device race and must be
 * serialised by the caller.  Synchronises `stream`; calls no hipMalloc or
 * hipFree. */
gnn_status gnn_csr_validate_noalloc(const gnn_csr* csr,
                                    int32_t require_symmetric,
                                    hipStream_t stream);

/* ------------------------------------------------------------ one layer */

/* Device bytes the forward pass saves for the backward pass, and the
 * scratch bytes forward and backward need.  Order 1 saves A_s X (n x f_in
 * floats).  With split products (neither product flag) there is also room
 * for the bf16 pieces of W_self^T and W_neigh^T (3 x 2 x ceil(h / 16) x 16 x
 * f_in bytes each); where the input gradient's product takes pieces, the
 * forward's weight split writes them, so that the backward pass does not
 * split the weights again.  With
 * GNN_FLAG_BF16 or GNN_FLAG_F32_MFMA order 2 saves nothing.  Both sizes
 * depend only on csr->n, csr->nnz, the layer shape, its order and its
 * product flag. */
size_t gnn_prop_saved_bytes(const gnn_csr* csr, const gnn_layer* layer);
size_t gnn_prop_workspace_bytes(const gnn_csr* csr, const gnn_layer* layer);

/* Forward of one layer, Section 2.1 Eq. "graphsage forward":
 *   Y[:, 0:h]  = ReLU(X W_self + b_self)
 *   Y[:, h:2h] = ReLU(A_s X W_neigh + b_neigh)
 * b_self / b_neigh may be NULL (no bias: the paper's form).  Needs
 * csr->values and csr->plan.  `saved` (gnn_prop_saved_bytes, may be NULL
 * when that is 0 or csr->n is 0) receives what gnn_prop_bwd needs and must
 * be passed to it unchanged.  Y must not overlap X. */
gnn_status gnn_prop_fwd(const gnn_csr* csr, const gnn_layer* layer,
                        const float* X, const float* W_self,
                        const float* W_neigh, const float* b_self,
                        const float* b_neigh, float* Y, void* saved,
                        void* workspace, size_t workspace_bytes,
                        hipStream_t stream);

/* Backward of one layer, Section 5.1 Eq. "gcn backward", given the forward
 * output Y (its sign pattern is the ReLU mask: G = dY * 1[Y > 0], 0 at the
 * kink) and dY = dL/dY:
 *   dW_self  = X^T G[:, 0:h]
 *   dW_neigh = (A_s X)^T G[:, h:2h]
 *   dX       = G[:, 0:h] W_self^T + (A_s)^T G[:, h:2h] W_neigh^T
 *   db_self, db_neigh = column sums of the two halves of G
 * dX may be NULL (not computed; e.g. the first layer).  db_* may be NULL.
 * layer->flags may add GNN_FLAG_DY_MASKED (dY already masked) and
 * GNN_FLAG_DX_MASKED (dX returned masked by 1[X > 0]) to the product flags
 * (GNN_FLAG_BF16 or GNN_FLAG_F32_MFMA, or neither: split products).
 * Needs csr->values, csr->values_t and csr->plan, and the `saved` buffer of
 * the matching gnn_prop_fwd call with the same layer (same order and product
 * flag) and the same weights: with split products the input gradient takes
 * either the weights or their pieces saved by that call (as in training,
 * where the backward pass follows the forward pass that used the weights).
 * Outputs must not overlap inputs. */
gnn_status gnn_prop_bwd(const gnn_csr* csr, const gnn_layer* layer,
                        const float* X, const float* W_self,
                        const float* W_neigh, const float* Y, const float* dY,
                        const void* saved, float* dX, float* dW_self,
                        float* dW_neigh, float* db_self, float* db_neigh,
                        void* workspace, size_t workspace_bytes,
                        hipStream_t stream);

/* ------------------------------------------------- GCN and MixHop layers */

/* The GNN variants of Section 2.1 on the same three kernels; their
 * backward keeps the A_hat terms of the Section 5.1 gradients.
 * csr->values must hold A_hat = (I + D)^-1/2 (I + A) (I + D)^-1/2 (the
 * pattern storing the self loops); it is symmetric, so csr->values_t may
 * point to csr->values.  layer->h is one path's output width; layer->flags
 * may hold one product flag (GNN_FLAG_BF16 or GNN_FLAG_F32_MFMA) only.  Sizes
 * of `saved` and workspace come from the matching queries; ownership and
 * aliasing rules are those of gnn_prop_fwd / gnn_prop_bwd.
 *
 * GCN (Eq. "gcn forward"): Y = ReLU(A_hat X W + b), Y n x h (stride
 * ld_y >= h), W f_in x h row-major, b [h] or NULL; order as for GraphSAGE
 * (1: (A_hat X) W, A_hat X saved; 2: A_hat (X W)).  Backward: G = dY *
 * 1[Y > 0], dW = (A_hat X)^T G, dX = A_hat^T G W^T (dX may be NULL),
 * db = column sums of G (db may be NULL). */
size_t gnn_gcn_saved_bytes(const gnn_csr* csr, const gnn_layer* layer);
size_t gnn_gcn_workspace_bytes(const gnn_csr* csr, const gnn_layer* layer);
gnn_status gnn_gcn_fwd(const gnn_csr* csr, const gnn_layer* layer,
                       const float* X, const float* W, const float* b,
                       float* Y, void* saved, void* workspace,
                       size_t workspace_bytes, hipStream_t stream);
gnn_status gnn_gcn_bwd(const gnn_csr* csr, const gnn_layer* layer,
                       const float* X, const float* W, const float* Y,
                       const float* dY, const void* saved, float* dX,
                       float* dW, float* db, void* workspace,
                       size_t workspace_bytes, hipStream_t stream);

/* MixHop (Eq. "mixhop forward"), K >= 0 hops:
 *   Y = ReLU( X W_0 || A_hat X W_1 || ... || A_hat^K X W_K  + b )
 * Y is n x (K+1)h (stride ld_y >= (K+1)h), hop k in columns [kh, (k+1)h);
 * W is f_in x (K+1)h row-major with W_k in the same columns; b is [(K+1)h]
 * or NULL.  The features are propagated first (A_hat^k X for k = 1..K, kept
 * in `saved`); layer->order must be 0 or 1.  Backward: G = dY * 1[Y > 0],
 * G_k its hop-k columns; dW_k = (A_hat^k X)^T G_k (dW laid out like W);
 * dX = sum_k (A_hat^k)^T G_k W_k^T (may be NULL); db = column sums of G
 * (may be NULL). */
size_t gnn_mixhop_saved_bytes(const gnn_csr* csr, const gnn_layer* layer,
                              int32_t K);
size_t gnn_mixhop_workspace_bytes(const gnn_csr* csr, const gnn_layer* layer,
                                  int32_t K);
gnn_status gnn_mixhop_fwd(const gnn_csr* csr, const gnn_layer* layer,
                          int32_t K, const float* X, const float* W,
                          const float* b, float* Y, void* saved,
                          void* workspace, size_t workspace_bytes,
                          hipStream_t stream);
gnn_status gnn_mixhop_bwd(const gnn_csr* csr, const gnn_layer* layer,
                          int32_t K, const float* X, const float* W,
                          const float* Y, const float* dY, const void* saved,
                          float* dX, float* dW, float* db, void* workspace,
                          size_t workspace_bytes, hipStream_t stream);

/* ----------------------------------------------------------- GAT layer */

/* Section 2.1, Eqs. "gat forward" and "gat attention": on the stored
 * entries (u, v) of the subgraph (edges and self loops; the CSR's values
 * are not used, its pattern must be symmetric and its plan built),
 *   P = X W,  att_uv = LeakyReLU(a1 . P_u + a2 . P_v)  (slope alpha in
 *   [0, 1] below 0),  Y = ReLU(A_att P)
 * with a = [a1; a2] (2h floats, device).  layer: f_in, h, ld_x, ld_y
 * (Y is n x h), ld_dx; order is ignored; flags: GNN_FLAG_BF16 or
 * GNN_FLAG_F32_MFMA for the products.  att_out (nnz floats, may be NULL) receives the attention
 * values in CSR order.  `saved` (gnn_gat_saved_bytes) carries P, the
 * scores and the attention values from the forward to the backward call.
 * Backward: dW (f_in x h), da (2h) and optionally dX, by the chain rule
 * (the per-entry products G_u . P_v form an SDDMM).  No output may overlap
 * an input, another output or the workspace (gnn_gat_workspace_bytes). */
size_t gnn_gat_saved_bytes(const gnn_csr* csr, const gnn_layer* layer);
size_t gnn_gat_workspace_bytes(const gnn_csr* csr, const gnn_layer* layer);
gnn_status gnn_gat_fwd(const gnn_csr* csr, const gnn_layer* layer, const float* X,
                       const float* W, const float* a, float alpha, float* Y,
                       float* att_out, void* saved, void* workspace,
                       size_t workspace_bytes, hipStream_t stream);
gnn_status gnn_gat_bwd(const gnn_csr* csr, const gnn_layer* layer, const float* X,
                       const float* W, const float* a, float alpha, const float* Y,
                       const float* dY, const void* saved, float* dX, float* dW,
                       float* da, void* workspace, size_t workspace_bytes,
                       hipStream_t stream);

/* --------------------------------------- classifier, loss, weight update */

/* Section 3.1 (Eqs. "mlp forward", "loss forward") and Algorithm 1: the
 * classifier head and loss that follow the GNN layers, with the gradients
 * of Section 5.1:
 *   XM = ReLU(X W)      X n x f (stride ld_x), W f x C row-major
 *   Y  = row softmax of XM (GNN_LOSS_SOFTMAX) or sigmoid(XM) element-wise
 *        (GNN_LOSS_SIGMOID)
 *   loss = (1/n) sum over rows of the cross-entropy of Y against T
 *        (n x C, stride ld_t, entries 0 or 1; one 1 per row for softmax)
 *   G  = (Y - T) / n * 1[XM > 0];   dW = X^T G (f x C);   dX = G W^T
 * `loss` is one float of device memory.  Optional outputs (NULL to skip):
 * xm = X_MLP (n x C, stride ld_xm), probs = Y (stride ld_p), dX (stride
 * ld_dx).  flags: GNN_FLAG_BF16 or GNN_FLAG_F32_MFMA for the three products.  The loss is summed
 * in a fixed order (bit-reproducible).  No output may overlap an input,
 * another output or the workspace.  Workspace:
 * gnn_classifier_workspace_bytes(n, f, C).  n = 0 gives loss 0 and dW = 0. */
#define GNN_LOSS_SOFTMAX 0
#define GNN_LOSS_SIGMOID 1
size_t gnn_classifier_workspace_bytes(int32_t n, int32_t f, int32_t C);
gnn_status gnn_classifier(int32_t n, int32_t f, int32_t C, int32_t kind,
                          uint32_t flags, const float* X, int64_t ld_x,
                          const float* W, const float* T, int64_t ld_t,
                          float* xm, int64_t ld_xm, float* probs, int64_t ld_p,
                          float* loss, float* dW, float* dX, int64_t ld_dx,
                          void* workspace, size_t workspace_bytes,
                          hipStream_t stream);

/* Weight update of Algorithm 1 (which leaves the rule open: plain gradient
 * descent, or Adam) on `count` contiguous floats (device):
 *   SGD:   W -= lr G
 *   Adam:  m = b1 m + (1 - b1) G;  v = b2 v + (1 - b2) G^2;
 *          W -= lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),  t >= 1
 * m and v (zero before the first step) are updated in place; no two
 * arrays may overlap.  The hyperparameters are host doubles: 1 - b1,
 * 1 - b2 and the bias corrections are formed in double and rounded once to
 * fp32, the precision of the update itself. */
gnn_status gnn_sgd_step(int64_t count, float* W, const float* G, double lr,
                        hipStream_t stream);
gnn_status gnn_adam_step(int64_t count, float* W, const float* G, float* m,
                         float* v, double lr, double beta1, double beta2,
                         double eps, int32_t t, hipStream_t stream);

/* ------------------------------- policy loss, clipping, update of many tensors */

/* Networks trained as policies: row i (a node, or a whole graph) chooses one
 * of C actions from the logits Z (n x C, stride ld_z), e.g. gnn_gemm's
 * product of the stack's output with a head's weights.
 *   lp_i = Z[i, a_i] - log sum_j exp Z[i, j]
 * action: n int32.  A row whose action lies outside [0, C) is left out: its
 * logits are not used (they may hold anything), its lp is written as 0 and
 * its gradient as 0.  Logits of -inf take an action out of a row's choice; a
 * row with every logit -inf is left out too, with lp = -inf.  Exponentials
 * are fp32's, at most 16 of them added in fp32 and all beyond in double: lp is
 * off by less than (20 + ln C) 2^-24 before its own rounding.
 *
 * gnn_action_logp writes lp (n floats): the old_logp / ref_logp that
 * gnn_policy_loss takes, of actions that were drawn from the logits.
 *
 * gnn_policy_loss: the clipped surrogate loss with a KL term, and its
 * gradient, with
 *   rho_i = exp(lp_i - old_logp_i)          (old_logp NULL: old_logp = lp)
 *   d_i   = ref_logp_i - lp_i,  kl_i = exp(d_i) - d_i - 1 >= 0
 *           (an unbiased sample of KL(policy || reference); ref_logp NULL: 0)
 *   l_i   = -min(rho_i A_i, clip(rho_i, 1 - clip_lo, 1 + clip_hi) A_i)
 *           + beta kl_i
 *   out   = [ sum_i w_i l_i,  sum_i w_i kl_i,  sum_i w_i 1[i is clipped] ]
 *   dZ[i, j] = w_i (dl_i / dlp_i) (1[j = a_i] - exp(Z[i, j]) / sum exp)
 *   dl_i / dlp_i = -A_i rho_i 1[i is not clipped] + beta (1 - exp(d_i))
 * where i is clipped if rho_i A_i > clip(rho_i, ...) A_i: decided as sums of
 * double exponentials decide it.  The three sums are formed in double.
 * advantage A, old_logp, ref_logp and weight w are n floats; weight NULL:
 * 1/n.  A row of weight 0 adds nothing and has a gradient of 0, whatever its
 * logits.  A chosen action with a logit of -inf has lp = -inf: its kl is
 * infinite, and its gradient not finite where beta > 0.  1 <= C <= 2^24,
 * 0 <= clip_lo <= 1, clip_hi >= 0 (infinity: no upper clip), beta finite >= 0,
 * needing ref_logp where beta > 0 (else GNN_ERR_SHAPE / GNN_ERR_NULL).
 * out: three floats.  logp (n floats) and dZ (n x C, stride ld_dz) may be
 * NULL.  Columns of dZ's rows past C are not written.  Everything is summed
 * in a fixed order (bit-reproducible).  n = 0 gives out = 0.  No output may
 * overlap an input, another output or the workspace
 * (gnn_policy_workspace_bytes, for both calls). */
size_t gnn_policy_workspace_bytes(int32_t n, int32_t C);
gnn_status gnn_action_logp(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                           const int32_t* action, float* logp, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);
gnn_status gnn_policy_loss(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                           const int32_t* action, const float* advantage,
                           const float* old_logp, const float* ref_logp,
                           const float* weight, double clip_lo, double clip_hi,
                           double beta, float* out, float* logp, float* dZ,
                           int64_t ld_dz, void* workspace, size_t workspace_bytes,
                           hipStream_t stream);

/* Acting, and teaching one network by another.  Rows of logits Z (n x C,
 * stride ld_z) as above; the order of a row's entries is: larger logits first,
 * equal ones (0 and -0 are) by their columns.  Logits of -inf are not there.
 * The first two calls leave out a row whose largest logit is not a finite
 * number, and one with a NaN.  1 <= C <= 2^24; temperatures T are 0 (the first
 * call) or 1e-6 to 1e6 (else GNN_ERR_SHAPE).
 *
 * gnn_sample_actions: each row draws an action by its random number u.  With
 *   e_j = exp((Z[i, j] - top) / T),  top the row's largest logit,
 * it keeps the shortest of these beginnings of the row's order:
 *   the first top_k                                     (0 or >= C: all)
 *   the shortest whose sum of e reaches top_p times that of the first top_k
 *                                                       (0 < top_p <= 1)
 *   those with Z[i, j] - top >= T ln(min_p)             (0 <= min_p <= 1)
 * and the action is the first of the kept entries, by columns, with which the
 * sum of their e passes u times the sum of all kept.  T = 0: the first entry
 * of the order, whatever the rest (u may be NULL).  Weights e are whole
 * multiples of a unit: 2^-51, where C > 2048 2^(log C - 62) with log C rounded
 * up, and where C > 2^18 the larger of 2^-51 and 2^(log s - 62), s being the
 * row's sum of e times at most 33/32 and log s rounded up.  Each is off by less
 * than 1e-13 and half a unit; nothing else is rounded but top_p's product and
 * log min_p, in double, so that an action does not depend on how a sum is
 * formed, and equal logits are equally likely.
 * u: n floats in [0, 1) (those below or NaN count as 0, those above as the
 * last number below 1).  action: n int32, -1 for rows left out.  logp (n
 * floats, may be NULL): the actions' log-probabilities under Z itself (T = 1,
 * nothing cut off), as gnn_action_logp gives them, 0 for rows left out: the
 * old_logp of gnn_policy_loss (where T is not 1 or something is cut off, not the
 * probability with which the action was drawn).  Workspace:
 * gnn_sample_workspace_bytes (0 up to 32,768 columns, some 50 KB a row beyond).
 *
 * gnn_top_logits: the first k entries of each row's order (1 <= k <=
 * GNN_TOP_MOST), with T > 0:
 *   index[i, r]  their columns (n x k int32, contiguous)
 *   logq[i, r] = Z[i, index] / T - log sum_j exp(Z[i, j] / T)     (n x k)
 *   rest[i]    = the share of all other entries                   (n, may be NULL)
 * Places past a row's entries, and rows left out, hold -1, -inf and a rest of
 * 0.  Workspace: gnn_top_workspace_bytes.
 *
 * gnn_distill_loss: a student's loss against such a list, and its gradient.
 *   q_r = exp(logq[i, r]) / N,  q_0 = rest[i] / N,  N = their sum
 *         (rest NULL: 0, so that logq may be any logits of the teacher / T)
 *   p   = softmax of Z[i] / T,  p_0 = the share of the entries not listed
 *   kl_i = T^2 [ sum_r q_r log(q_r / p_index(r)) + q_0 log(q_0 / p_0) ]
 *   out  = sum_i w_i kl_i                                    (one float)
 *   dZ[i, j] = w_i T (p_j - q_r)           for entries j = index[i, r]
 *              w_i T p_j (1 - q_0 / p_0)   for all others
 * An index outside [0, C) marks a place that is not used, and one that a row
 * repeats counts at its first place.  Rows are left out, with kl and gradient
 * 0, whose list has no index in range, or nothing but q of 0, or whose logits
 * are all -inf: of the first kind the logits may hold anything.  A row of
 * weight 0 adds nothing and has a gradient of 0.  weight: n floats (NULL: 1/n).
 * A q above 0 where the student has p = 0 makes kl infinite, a NaN or +inf among
 * a row's logits shows in its kl and gradient.  Columns of dZ's rows past C are
 * not written; kl (n floats) and dZ (stride ld_dz) may be NULL.  n = 0 gives
 * out = 0.  Exponentials of the row are fp32's, everything of the list is in
 * double, and so are all sums: kl is good to T^2 (6 ln C + 24) 2^-24 and its
 * rounding.  Workspace: gnn_distill_workspace_bytes.
 *
 * For all three: results are bit-reproducible, and no output may overlap an
 * input, another output or the workspace. */
#define GNN_TOP_MOST 256
size_t gnn_sample_workspace_bytes(int32_t n, int32_t C);
gnn_status gnn_sample_actions(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                              const float* u, double temperature, int32_t top_k,
                              double top_p, double min_p, int32_t* action,
                              float* logp, void* workspace, size_t workspace_bytes,
                              hipStream_t stream);
size_t gnn_top_workspace_bytes(int32_t n, int32_t C, int32_t k);
gnn_status gnn_top_logits(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                          int32_t k, double temperature, int32_t* index,
                          float* logq, float* rest, void* workspace,
                          size_t workspace_bytes, hipStream_t stream);
size_t gnn_distill_workspace_bytes(int32_t n, int32_t C, int32_t k);
gnn_status gnn_distill_loss(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                            int32_t k, const int32_t* index, const float* logq,
                            const float* rest, const float* weight,
                            double temperature, float* out, float* kl, float* dZ,
                            int64_t ld_dz, void* workspace, size_t workspace_bytes,
                            hipStream_t stream);

/* A set of tensors that are updated together (all weights of a model), each
 * of `count` contiguous elements (count 0: nothing).
 *   W, G     weights and gradients (device, 4-byte aligned; gradients may be
 *            shared by several tensors)
 *   m, v     Adam's moments: state_bits 32: floats; state_bits 8: one byte
 *            each, m in OCP e4m3 and v in OCP e5m2, times the scale of its
 *            block of 256 consecutive elements
 *   m_scale, v_scale  state_bits 8: ceil(count / 256) floats each; state_bits
 *            32: not used
 *   weight_decay      of this tensor (0 for biases, say)
 * Moments start as zeros (scales too).  Any such alignment takes the vector
 * path.  gnn_grad_norm alone needs only count and G: W, m, v and the scales
 * may then be NULL. */
typedef struct gnn_param {
  int64_t count;
  float* W;
  const float* G;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  double weight_decay;
} gnn_param;
#define GNN_STATE_BLOCK 256 /* elements that share a scale of 8-bit moments */

/* n tensors (host array p) with state_bits 32 or 8 and, for the calls below,
 * `plan`: the device buffer that gnn_params_build_plan filled for exactly
 * these tensors (pointers, counts, decay). */
typedef struct gnn_params {
  int32_t n;
  int32_t state_bits;
  const gnn_param* p;
  const void* plan;
} gnn_params;

/* Bytes of the plan, and its filling (a device buffer of at least that size,
 * 16-byte aligned): a table of the tensors and of the pieces of 1,024
 * elements that one workgroup takes, so that one launch covers every tensor.
 * Nothing is read from the host after the call returns; the plan itself, a
 * table of addresses, is written on `stream`, and a call on another stream has
 * to wait for that.  No W, m, v or scale may overlap anything else in the set
 * or the plan (GNN_ERR_ALIAS).  params->plan is not read. */
size_t gnn_params_plan_bytes(const gnn_params* params);
gnn_status gnn_params_build_plan(const gnn_params* params, void* plan,
                                 size_t plan_bytes, hipStream_t stream);

/* norm (one device float) = square root of the sum of squares of every
 * gradient of the set, squares and sums in double, in a fixed order. */
size_t gnn_grad_norm_workspace_bytes(const gnn_params* params);
gnn_status gnn_grad_norm(const gnn_params* params, float* norm, void* workspace,
                         size_t workspace_bytes, hipStream_t stream);

/* AdamW step t >= 1 on every tensor of the set, one launch:
 *   g = k G;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
 *   W = (1 - lr weight_decay) W
 *       - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
 * norm: device float (gnn_grad_norm's) or NULL.  NULL: k = 1, whatever
 * max_norm.  Else k = max_norm / norm where norm > max_norm (max_norm > 0) and
 * 1 elsewhere, and a norm that is not finite skips the step: nothing is
 * changed.  t is the caller's count: one that goes on over a skipped step has
 * bias corrections for a step more than the moments hold, so that the updates
 * after it are smaller than they might be (by (1 - b1) / (1 - b1^2) over the
 * root of the same of b2, 0.74 for 0.9 and 0.999, where the first step of all
 * is skipped; less and less later).
 * Without norm a NaN or infinite gradient makes its own weight and moments
 * non-finite, with 8-bit moments those of its whole block of 256 (so does one
 * whose square passes 1e43).
 * Hyperparameters are host values, taken at the call (a captured launch
 * replays with them): 0 <= beta1, beta2 < 1, eps >= 0 (with 0 a weight whose
 * v is 0 becomes NaN, as the formula says), lr finite.
 *
 * 8-bit moments: m, v and the update are formed from unrounded new moments
 * (in double), which are then stored with scale = max over the block / 448
 * (m) or / 57344 (v), at least 2^-126, and rounded stochastically: up with
 * the probability of their distance from the lower neighbour.  An average
 * with b2 = 0.999 moves by 0.1 % a step where e5m2's neighbours are 14 to
 * 25 % apart: rounding to nearest would hold it where it is, stochastic
 * rounding keeps its expectation.  A positive v is never stored as 0 (its
 * weight's next step would be divided by a root that is too small).  Element
 * e of a tensor whose predecessors in the set hold B blocks of 256 takes bits
 * of output (256 B + e) / 2 of the SplitMix64 generator started at output t
 * of the one started at `seed` (the lower 32 bits for even e: the lower 16 of
 * them for m, the upper 16 for v; r stands for (r + 1/2) / 2^16), so results
 * are a function of the arguments only.  seed is not used with 32 bits. */
gnn_status gnn_adamw_step(const gnn_params* params, double lr, double beta1,
                          double beta2, double eps, int32_t t, const float* norm,
                          double max_norm, uint64_t seed, hipStream_t stream);

/* ------------------------------------------- subgraph preparation (prep) */

/* The subgraph of the full training graph induced by a sampled node set
 * (the last step of the samplers, Section 4, Algorithms 2 and 3; Algorithm
 * 1's adjacency matrix of G_s), on the GPU against a full graph resident in
 * device memory:
 *   full graph: n_full nodes, CSR with int64 row pointers indptr (n_full + 1)
 *     and int32 indices (nnz_full), rows sorted, symmetric, unweighted;
 *   nodes: n_s full-graph ids (device), strictly ascending; node nodes[i]
 *     becomes node i of the subgraph;
 *   result: CSR sub_indptr (n_s + 1), sub_indices / sub_values (room for
 *     `capacity` entries; the sum over V_s of (full degree + 1) always
 *     suffices), every node with its self loop, rows sorted; values
 *     1/len_u (GNN_NORM_ROW: D^-1 A of Eq. "graphsage forward", D counting
 *     the stored entries) or 1/sqrt(len_u len_v) (GNN_NORM_SYM, the GCN
 *     layer's normalisation of Section 2.1);
 *   nnz_out (device int64) receives the number of stored entries;
 *   status_out (device int32) receives 0, or bits 1 (an id out of range:
 *     that row keeps its self loop only), 2 (ids not strictly ascending:
 *     the result is not meaningful), 4 (more entries than capacity: the
 *     excess is not written);
 *   map: n_full int32 of device scratch, all -1 on entry, all -1 again
 *     when the call's work completes (it maps full ids to V_s positions).
 * Nothing is read back to the host: the caller copies nnz_out / status_out
 * when it needs them.  Workspace: gnn_induce_workspace_bytes(n_s). */
#define GNN_NORM_ROW 0
#define GNN_NORM_SYM 1
size_t gnn_induce_workspace_bytes(int32_t n_s);
gnn_status gnn_induce_subgraph(int64_t n_full, int64_t nnz_full,
                               const int64_t* indptr, const int32_t* indices,
                               int32_t n_s, const int32_t* nodes, int32_t norm,
                               int32_t* map, int64_t capacity,
                               int32_t* sub_indptr, int32_t* sub_indices,
                               float* sub_values, int64_t* nnz_out,
                               int32_t* status_out, void* workspace,
                               size_t workspace_bytes, hipStream_t stream);

/* Algorithm 1's lookup of the minibatch features / labels by V_s:
 * dst row r = src row index[r] (width floats; src has src_rows rows of
 * stride ld_src, dst stride ld_dst); an index outside [0, src_rows) gives a
 * row of zeros.  dst may not overlap src or index. */
gnn_status gnn_gather_rows(int32_t rows, const int32_t* index, int32_t width,
                           const float* src, int64_t ld_src, int64_t src_rows,
                           float* dst, int64_t ld_dst, hipStream_t stream);

/* ------------------------------------------ sampling and the pool (host) */

/* Frontier sampling (Section 4.1, Algorithm 2) through the Dashboard of
 * Section 4.2 (Algorithms 3 and 4), host code.  Full graph in HOST memory
 * (int64 indptr of n_full + 1, int32 indices, symmetric, rows sorted).
 * m: frontier size; budget: n of Algorithm 2 (budget - m frontier updates;
 * budget >= m); eta >= 1: Dashboard enlargement (eta * m * d slots, d the
 * mean degree); clip > 1 drops |V_s| mod clip nodes chosen uniformly (the
 * node clipping of Section 6.2; 0 or 1: none).  V_s is the initial frontier
 * plus every node that enters the frontier, returned sorted and distinct in
 * `nodes` (room for `budget` ints), its size in *n_nodes.  The result is a
 * function of (graph, parameters, seed, id) only; random numbers are
 * SplitMix64 outputs used as a counter-based generator (stream start
 * states: outputs 4 id + k of the generator started at seed; k = 0 initial
 * frontier, 1 probes, 2 neighbour choice, 3 clipping; an integer below K is
 * floor(r K / 2^64)). */
gnn_status gnn_frontier_sample(int64_t n_full, const int64_t* indptr,
                               const int32_t* indices, int32_t m, int32_t budget,
                               double eta, int32_t clip, uint64_t seed, int64_t id,
                               int32_t* nodes, int32_t* n_nodes);

/* The subgraph pool of Algorithm 8: `threads` worker threads sample
 * subgraphs id = 0, 1, 2, ... (each exactly as gnn_frontier_sample with
 * that id) and keep at most `depth` of them ready; gnn_sampler_next hands
 * them out in id order, blocking until the next one is ready.  The graph
 * arrays must stay valid and unchanged until gnn_sampler_destroy, which
 * stops and joins the workers.  One consumer thread per pool. */
typedef struct gnn_sampler gnn_sampler;
gnn_status gnn_sampler_create(int64_t n_full, const int64_t* indptr,
                              const int32_t* indices, int32_t m, int32_t budget,
                              double eta, int32_t clip, uint64_t seed,
                              int32_t threads, int32_t depth, gnn_sampler** out);
gnn_status gnn_sampler_next(gnn_sampler* s, int32_t* nodes, int32_t* n_nodes,
                            int64_t* id);
void gnn_sampler_destroy(gnn_sampler* s);

/* ------------------------------------------------------------- kernels */

/* Feature / gradient propagation alone (Section 5.1's first kernel, the
 * per-slice product of Section 5.3, Algorithm 7):
 *   out = A_s . in        (transpose = 0, uses csr->values)
 *   out = (A_s)^T . in    (transpose = 1, uses csr->values_t)
 * in and out are n x w with strides ld_in, ld_out; needs csr->plan;
 * `workspace` of gnn_spmm_workspace_bytes(csr, w) bytes (may be NULL if 0;
 * the current kernel needs none and returns 0).  out must not overlap in. */
size_t gnn_spmm_workspace_bytes(const gnn_csr* csr, int32_t w);
gnn_status gnn_spmm(const gnn_csr* csr, int32_t transpose, int32_t w,
                    const float* in, int64_t ld_in, float* out,
                    int64_t ld_out, void* workspace, size_t workspace_bytes,
                    hipStream_t stream);

/* Measurement aid, not part of the method: the gathers of gnn_spmm alone.
 * It runs gnn_spmm's grid, column slices, lane groups, entry order and
 * loads (index, value, neighbour row slice) but keeps one sum per lane for
 * all of its entries instead of one per row: no per-entry row reads, no row
 * closing, no finishing of rows shared between lane groups.  Each plan
 * window's column totals (in a fixed order) go to the window's first row,
 * zeros to its other rows, so every row of `out` is written once and the
 * column sums of `out` equal those of A_s . in (resp. (A_s)^T . in).  Its
 * time bounds from below what the aggregation's gather order costs on the
 * device.  Same arguments and checks as gnn_spmm (no workspace); rows of
 * `in` and `out` must start 16-byte aligned (else GNN_ERR_UNSUPPORTED). */
gnn_status gnn_spmm_gather_floor(const gnn_csr* csr, int32_t transpose,
                                 int32_t w, const float* in, int64_t ld_in,
                                 float* out, int64_t ld_out, hipStream_t stream);

/* Dense weight transformation alone (Section 5.1's second kernel):
 *   C = op(A) op(B),  C is M x N (stride ldc),
 *   op(A) = A (M x K, stride lda)  or A^T with A stored K x M (trans_a = 1),
 *   op(B) = B (K x N, stride ldb)  or B^T with B stored N x K (trans_b = 1).
 * flags: GNN_FLAG_BF16 or GNN_FLAG_F32_MFMA (neither: split products).
 * `workspace` of gnn_gemm_workspace_bytes bytes. */
size_t gnn_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K);
gnn_status gnn_gemm(int32_t trans_a, int32_t trans_b, int32_t M, int32_t N,
                    int32_t K, const float* A, int64_t lda, const float* B,
                    int64_t ldb, float* C, int64_t ldc, uint32_t flags,
                    void* workspace, size_t workspace_bytes,
                    hipStream_t stream);

/* Measurement aid, not part of the method: the sustained rate of the
 * device's matrix cores, against which the products' rates are read.
 * Launches `blocks` workgroups of 512 threads (eight wavefronts, two
 * workgroups per CU as in the split-product GEMM); every wavefront issues
 * 4 x `iters` MFMAs on register operands into four independent accumulators,
 * with no memory traffic in the loop:
 *   GNN_PROBE_MFMA_BF16  v_mfma_f32_32x32x16_bf16, 32768 flop each
 *   GNN_PROBE_MFMA_F32   v_mfma_f32_32x32x2_f32,    4096 flop each
 * so one launch does blocks x 8 x 4 x iters x (flop each).  The caller times
 * the launch (events on `stream`) for the rate.  `sink` (device, blocks x
 * 512 floats, 4-byte aligned) receives each thread's accumulator sum.
 * `clocks` (device, two 8-byte-aligned uint64) receives the shader-clock
 * cycles (s_memtime) and the 100 MHz real-time ticks (s_memrealtime) that
 * the first wavefront of workgroup 0 counted over its loop: cycles / ticks
 * x 0.1 is the shader clock in GHz under this load.  Errors: an unknown
 * kind GNN_ERR_UNSUPPORTED, blocks or iters outside [1, max]
 * GNN_ERR_SHAPE, a NULL pointer GNN_ERR_NULL, misaligned pointers
 * GNN_ERR_UNSUPPORTED, `sink` overlapping `clocks` GNN_ERR_ALIAS. */
#define GNN_PROBE_MFMA_BF16 0
#define GNN_PROBE_MFMA_F32 1
#define GNN_PROBE_MAX_BLOCKS 65536
#define GNN_PROBE_MAX_ITERS 100000
gnn_status gnn_mfma_rate_probe(int32_t kind, int32_t blocks, int32_t iters,
                               float* sink, uint64_t* clocks, hipStream_t stream);

/* ----------------------------------------------------- kernel timing */

/* Kernels timed by the optional event timer. */
#define GNN_K_SPMM 0          /* aggregation (one kernel per product) */
#define GNN_K_SPMM_REDUCE 1   /* reserved: no separate reduction is launched */
#define GNN_K_GEMM_NN 2       /* C = A B            (forward transforms) */
#define GNN_K_GEMM_TN 3       /* C = A^T B          (weight gradients) */
#define GNN_K_GEMM_NT 4       /* C = A B^T          (input gradients) */
#define GNN_K_GEMM_TT 5       /* C = A^T B^T */
#define GNN_K_GEMM_REDUCE 6   /* split-K partial reduction */
#define GNN_K_MASK 7          /* ReLU mask of the output gradient */
#define GNN_K_COLSUM 8        /* bias-gradient column sums */
#define GNN_K_PLAN 9          /* aggregation plan build */
#define GNN_K_TRANSPOSE 10    /* transposed values (Algorithm 6) */
#define GNN_K_LOSS 11         /* classifier, policy or student's loss, its gradient */
#define GNN_K_UPDATE 12       /* weight update (SGD, Adam or AdamW) */
#define GNN_K_INDUCE 13       /* induced subgraph on the GPU */
#define GNN_K_GATHER 14       /* feature / label row gather */
#define GNN_K_SDDMM 15        /* GAT per-entry dot products */
#define GNN_K_WSPLIT 16       /* weights split into bf16 pieces (split products) */
#define GNN_K_NORM 17         /* norm of all gradients */
#define GNN_K_SAMPLE 18       /* actions drawn, top logits */
#define GNN_K_COUNT 19

/* When enabled, every kernel launch is bracketed by a pair of HIP events on
 * its stream.  gnn_timer_read synchronises on the recorded events and
 * returns, for one kernel id since the last reset, the summed milliseconds,
 * the launch count and the summed algorithmic work of those launches:
 * bytes for memory-bound kernels (aggregation: 4(n+1) + 8 nnz + 8 n w per
 * call, counted on GNN_K_SPMM), flops for the GEMMs (2 M N K).  Host-side
 * bookkeeping only; not thread safe. */
gnn_status gnn_timer_enable(int32_t enable);
gnn_status gnn_timer_reset(void);
gnn_status gnn_timer_read(int32_t kernel, double* ms, int64_t* launches,
                          double* work);

#ifdef __cplusplus
}
#endif
#endif /* GNNPROP_H */
