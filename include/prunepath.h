/*
 * prunepath.h -- C ABI of the GB300 (sm_103a) PrunePath sparse-FFN library.
 *
 * PrunePath (Sec. 3.1) routes each token x in R^d with a linear router
 *   g = W_r^T x                                   (Eq. routing_logits)
 *   p_j = exp(g_j) / sum_i exp(g_i)               (Eq. softmax_prob)
 * orders the experts by descending probability (pi), activates a prefix of
 * that order by cumulative probability mass     (Eq. tau_thresh_activate)
 * and evaluates only the activated expert slices of a MoEfied FFN
 *   y = sum_{e in A} sigmoid(g_e) * FFN_e(x)      (Eq. moe_output)
 * where FFN_e is the restriction of the gated FFN (Eq. ffn) to the e-th block
 * of d_e contiguous intermediate neurons        (Eq. moefication_decomp).
 *
 * ------------------------------------------------------------------------
 * Conventions shared by every entry point
 *  - Every tensor pointer is a DEVICE pointer owned by the caller, row-major,
 *    contiguous and 16-byte aligned.  The library never allocates, frees or
 *    keeps a tensor pointer beyond the call.  The one exception is the
 *    offline host routine pp_moefy_cluster, whose pointers are host pointers.
 *  - Weight layout ("expert neurons stored contiguously"):
 *      W_r    [E][d]      row j is the routing vector of expert j
 *                         (the paper's W_r in R^{d x E}, stored transposed)
 *      W_gate [d_ff][d]   row n holds neuron n's input weights; expert e is
 *      W_up   [d_ff][d]   the dense row block [e*d_e, (e+1)*d_e)
 *      W_down [d][d_ff]   expert e is the dense column block [e*d_e, (e+1)*d_e)
 *    x and y are [T][d].  Element type: pp_desc.dtype for x, y and all weights.
 *  - The selection (pp_selection) is [T][E] int32 ids in rank order (first
 *    counts[t] entries valid, the rest -1), counts [T] int32, gates [T][E]
 *    fp32 aligned with ids (sigmoid(g_e) for PP_GATE_SIGMOID, 1 for
 *    PP_GATE_NONE, 0 past counts[t]) and, optionally, logits [T][E] fp32 in
 *    expert order.
 *  - Every call is asynchronous on `stream` (a cudaStream_t passed as void*;
 *    NULL means the legacy default stream).  Argument errors are returned
 *    synchronously before anything is enqueued.  Errors found on the device
 *    (a bounded wait that timed out, a non-finite logit) are recorded in the
 *    workspace status word and read back by pp_get_device_status.
 *  - Workspace: caller-owned device memory of at least pp_workspace_size()
 *    bytes, 256-byte aligned, zeroed once by pp_workspace_init before its
 *    first use.  Calls that share a workspace must be ordered on one stream;
 *    calls on different workspaces are independent.  A workspace serves one
 *    device (it keeps per-SM launch counts of the fused decode kernel).
 *  - No C++ exception crosses this interface.
 *  - Supported shapes: d_expert == 64, d_ff == E * 64, 1 <= E <= 256,
 *    d a multiple of 8 (bf16) or 4 (fp32), 64 <= d <= 8192, T >= 0.
 *    Other shapes return PP_ERR_SHAPE.
 *  - p is the parameter of the cut rule (pp_desc.rule); NaN returns
 *    PP_ERR_INVALID_ARG under every rule.
 *      MIN_PREFIX, PAPER: the mass budget tau.  p >= 1 activates all E
 *        experts (the warm-up setting tau_warm = 1.05 of Sec. 3.2); p <= 0
 *        activates the top-1 expert only.
 *      TOPK: the expert count k = floor(p), at least 1 and at most E.
 *      LTE: the score threshold delta; p <= 0 activates all E experts and
 *        p >= 1 none (counts[t] = 0, y[t] = 0).
 */
#ifndef PRUNEPATH_H
#define PRUNEPATH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum pp_status {
    PP_OK = 0,
    PP_ERR_INVALID_ARG = 1, /* NULL pointer, NaN p, unknown enum value            */
    PP_ERR_SHAPE = 2,       /* shape outside the supported set (see above)        */
    PP_ERR_DTYPE = 3,       /* unsupported dtype / activation combination         */
    PP_ERR_ALIGN = 4,       /* a pointer is not 16-byte aligned                   */
    PP_ERR_WORKSPACE = 5,   /* workspace NULL, misaligned or too small            */
    PP_ERR_CUDA = 6,        /* a CUDA runtime call failed (launch, attribute)     */
    PP_ERR_TIMEOUT = 7,     /* device: a bounded wait gave up (sticky)            */
    PP_ERR_CAPACITY = 8,    /* device: an internal buffer would overflow (sticky) */
    PP_ERR_NONFINITE = 9,   /* device: a router logit was NaN/Inf (sticky); the
                               token gets counts[t] = 0 and y[t] = 0              */
    PP_ERR_UNSUPPORTED = 10,/* no device of compute capability 10.3 is current    */
    PP_ERR_HOST = 11        /* host memory or threads could not be obtained (the
                               offline host routine pp_moefy_cluster)             */
} pp_status;

typedef enum pp_dtype { PP_F32 = 0, PP_BF16 = 1 } pp_dtype;

/* FFN variant.  SWIGLU is Eq. (ffn) with phi = SiLU and needs W_gate; RELU
   and GELU_TANH are the non-gated forms h = phi(x W_up) (Sec. 2.1 notes the
   analysis covers any FFN separable along d_ff) and take W_gate = NULL. */
typedef enum pp_act { PP_ACT_RELU = 0, PP_ACT_GELU_TANH = 1, PP_ACT_SWIGLU = 2 } pp_act;

/* Output weighting.  SIGMOID is Eq. (moe_output); NONE weights every
   selected expert by 1, the plain decomposition of Eq. (moefication_decomp). */
typedef enum pp_gate { PP_GATE_SIGMOID = 0, PP_GATE_NONE = 1 } pp_gate;

/* Activation rule on the router logits g.  Every rule lists the activated
   experts in the descending order pi (ties by lower expert index).
   MIN_PREFIX: the shortest prefix of pi whose mass reaches p (keeps the rank
   that crosses p).  PAPER: Eq. (tau_thresh_activate) literally, rank 1 plus
   every rank with S_i < p.  Whenever S_E >= p, |PAPER| =
   max(1, |MIN_PREFIX| - 1).
   TOPK: the first k = floor(p) experts of pi, the fixed expert budget of the
   top-k reconstruction analysis (Sec. 4.3).
   LTE: every expert with sigmoid(g_e) > p, each expert thresholded on its
   own (Eq. lte_hard_set, the rule PrunePath is compared with in Sec. 2.3);
   LTE's own aggregation (Eq. lte_hard_output) is PP_GATE_NONE.  The device
   takes the same decision on the fp32 logit: g_e >= the smallest fp32 value
   above ln(p / (1 - p)), a bound the host computes in double precision. */
typedef enum pp_rule { PP_SEL_MIN_PREFIX = 0, PP_SEL_PAPER = 1, PP_SEL_TOPK = 2, PP_SEL_LTE = 3 } pp_rule;

typedef struct pp_desc {
    int d_model;   /* d                                   */
    int d_ff;      /* intermediate width, == n_experts*64 */
    int n_experts; /* E                                   */
    int d_expert;  /* d_e, must be 64                     */
    int dtype;     /* pp_dtype                            */
    int act;       /* pp_act                              */
    int gate;      /* pp_gate                             */
    int rule;      /* pp_rule                             */
} pp_desc;

typedef struct pp_selection {
    int32_t *ids;    /* [T][E] device, rank order, -1 padded          */
    int32_t *counts; /* [T]    device                                 */
    float *gates;    /* [T][E] device, aligned with ids               */
    float *logits;   /* [T][E] device, expert order; may be NULL      */
} pp_selection;

/* Bytes of workspace needed for calls with up to T tokens. */
size_t pp_workspace_size(const pp_desc *desc, int T);

/* Zero the whole workspace (status word, launch counts, accumulators) on
   `stream`.  Call once after allocating a workspace, and again to clear a
   sticky device error. */
pp_status pp_workspace_init(void *ws, size_t ws_bytes, void *stream);

/* Router and selection (Eq. routing_logits, softmax_prob,
   tau_thresh_activate).  x [T][d], W_r [E][d]; writes *out (out->logits may
   be NULL).  The softmax is max-shifted in fp32 with fp32 exponentials; the
   normaliser and the prefix masses are summed exactly (2^-31 fixed-point
   integers for up to 64 tokens per call, fp64 beyond), so the cut is decided
   by an exact comparison with p times the normaliser; the order is
   descending logit with ties broken by the lower expert index. */
pp_status pp_route(const pp_desc *desc, const void *x, int T, const void *W_r, float p,
                   const pp_selection *out, void *ws, size_t ws_bytes, void *stream);

/* Selection only, from given fp32 logits [T][E] (out->logits is ignored). */
pp_status pp_select(const pp_desc *desc, const float *logits, int T, float p,
                    const pp_selection *out, void *ws, size_t ws_bytes, void *stream);

/* Sparse FFN over a given selection (Eq. moe_output): for each token t,
   y[t] = sum_{r < counts[t]} gates[t][r] * FFN_{ids[t][r]}(x[t]).
   Reads sel->ids, sel->counts, sel->gates.  W_gate is NULL unless act is
   PP_ACT_SWIGLU.  Accumulation is fp32; y has the dtype of x. */
pp_status pp_sparse_ffn(const pp_desc *desc, const void *x, int T, const void *W_gate,
                        const void *W_up, const void *W_down, const pp_selection *sel, void *y,
                        void *ws, size_t ws_bytes, void *stream);

/* pp_route followed by pp_sparse_ffn, fused where the token count allows.
   sel_out may be NULL (the selection then stays in the workspace). */
pp_status pp_layer(const pp_desc *desc, const void *x, int T, const void *W_r, const void *W_gate,
                   const void *W_up, const void *W_down, float p, const pp_selection *sel_out,
                   void *y, void *ws, size_t ws_bytes, void *stream);

/* One layer of a chained decode step: the layer input is formed from the
   previous layer's input and output,
     x = RMSNorm(x_prev + y_prev) * gamma,   RMSNorm(v) = v / sqrt(mean(v^2) + eps)
   per token (the post-norm residual connection x_{l+1} = RMSNorm(x_l + y_l)
   that stacks the layers of the decode setting of Sec. 4.5), written to x,
   and then y = pp_layer(x).  x_prev, y_prev, x, y are [T][d]; gamma is [d];
   y_prev may be NULL (no residual term: the first layer) and gamma NULL
   (unit weights).  The sum and the mean square are fp32; x is stored in the
   desc dtype and the layer reads exactly that x.  For up to 4 bf16 / 8 fp32
   tokens the fused decode kernel forms x in its prologue (one launch);
   otherwise one more kernel runs first.  x and y must not overlap x_prev,
   y_prev or each other (PP_ERR_INVALID_ARG); eps >= 0. */
pp_status pp_layer_chained(const pp_desc *desc, const void *x_prev, const void *y_prev, const void *gamma,
                           float eps, int T, const void *W_r, const void *W_gate, const void *W_up,
                           const void *W_down, float p, const pp_selection *sel_out, void *x, void *y, void *ws,
                           size_t ws_bytes, void *stream);

/* pp_layer for callers that cannot allocate device memory where they run a
   layer -- a runtime that has given every byte to its own pool, a loop that
   must not block on an allocation's implicit synchronisation, a plug-in host
   that exposes no allocator.  The paper has no counterpart: this entry point
   exists only for those callers.
   Same computation and arguments as pp_layer, for T <= 4 tokens and without a
   workspace.  Like pp_layer, it runs the tokens in slices when one fused
   launch cannot hold them all (fp32 rows of a wide model).  Its scratch (status word, per-CTA launch counts, router
   logits and gate/up activations: 533,760 bytes) is one static
   device array that every GPU loading this library keeps until the process
   exits; no call allocates or frees.
   - T > 4 (like any shape pp_layer rejects) returns PP_ERR_SHAPE.
   - The first call on a device, made with that device current, looks up the
     array's address there; make that first call before any stream capture.
   - Every call reuses the same array and first clears its status word;
     calls that overlap on the GPU (other streams, other host threads) race
     on it, so the caller must serialise them.
   - status_out (optional, device uint32) receives the call's device-side
     status (a pp_status code) when the call has run on `stream`. */
pp_status pp_layer_noalloc(const pp_desc *desc, const void *x, int T, const void *W_r,
                           const void *W_gate, const void *W_up, const void *W_down, float p,
                           const pp_selection *sel_out, void *y, uint32_t *status_out, void *stream);

/* FFN-sparsity statistics (Sec. 4.1, s_FFN): adds sum_t counts[t] to
   acc[0] and a histogram of counts (0..E) to acc[1..E+1].  acc is
   [E+2] uint64 on the device, accumulated across calls (one per layer), so
   s_FFN = 1 - acc[0] / (N * L * E). */
pp_status pp_sparsity_stats(const int32_t *counts, int T, int n_experts, uint64_t *acc,
                            void *stream);

/* Router statistics of a batch of B = T tokens (forward values of the router
   terms of the training objective, reported as routing diagnostics):
     out[0] = L_ent  = -(1/B) sum_t sum_j p_tj log(p_tj + eps)  (Sec. 3.2, Eq. entropy_loss)
     out[1] = L_bal  = E sum_j ((1/B) sum_t p_tj)^2             (Sec. 3.2, Eq. load_balance_loss)
     out[2] = L_gate = (1/(B E)) sum_t sum_j sigmoid(g_tj)       (Sec. 4.2.3, gate-magnitude term)
   with p_tj the softmax of Eq. (softmax_prob).  logits [T][E] fp32 device
   (e.g. the logits pp_route writes); out: 3 doubles, device, 8-byte aligned.
   The softmax is max-shifted in fp32; the sums are fp32 in a fixed order,
   pairwise across blocks of 64 tokens, combined in fp64 (deterministic).  T >= 1 (else PP_ERR_SHAPE); eps NaN is
   PP_ERR_INVALID_ARG.  Uses the workspace of pp_workspace_size(desc, T).  A
   non-finite logit records PP_ERR_NONFINITE and makes out[0] NaN. */
pp_status pp_router_stats(const pp_desc *desc, const float *logits, int T, float eps, double *out, void *ws,
                          size_t ws_bytes, void *stream);

/* MoEfication preprocessing, clustering (Sec. 2.2): group the d_ff
   intermediate neurons of a dense FFN into E experts of d_e = 64 neurons by
   balanced k-means over their input weights, and return the permutation Pi
   that makes every expert a contiguous block (pp_moefy_permute applies it).
   An OFFLINE HOST routine, run once per model before serving: W_gate, W_up,
   init, perm, labels, iters and objective are HOST pointers; it runs on the
   calling thread and a pool of host threads and touches no GPU.
   - Features: neuron n's input weights -- row n of W_gate followed by row n
     of W_up for PP_ACT_SWIGLU (W_gate required), row n of W_up otherwise
     (W_gate ignored); W_gate, W_up are [d_ff][d] in desc->dtype, widened
     exactly.
   - Balanced k-means (the constrained k-means of Bradley, Bennett and
     Demiriz, 2000, with every cluster holding exactly 64 neurons): the
     centroids start at the features of neurons init[0..E) (distinct, in
     [0, d_ff); the random choice is the caller's); each iteration assigns
     the neurons to clusters with the least total squared Euclidean distance
     under the equal-size constraint (solved exactly, fp64), then moves every
     centroid to the mean of its members; it stops when an assignment repeats
     the previous one, or after max_iter (>= 1) assignments.
   - Outputs: perm [d_ff] int32 (new position j holds old neuron perm[j];
     cluster e fills positions [64e, 64e + 64) in ascending old index);
     labels [d_ff] int32, the cluster of each old neuron (may be NULL);
     *iters = assignments made and *objective = the last assignment's sum of
     squared distances (either may be NULL).
   - Host memory: about d_ff * (f * 4 + E * 8) bytes, f = d or 2d.
   Errors: PP_ERR_INVALID_ARG (NULL input or perm, bad init, max_iter < 1),
   PP_ERR_SHAPE / PP_ERR_DTYPE as for every call, PP_ERR_HOST. */
pp_status pp_moefy_cluster(const pp_desc *desc, const void *W_gate, const void *W_up, const int32_t *init,
                           int max_iter, int32_t *perm, int32_t *labels, int *iters, double *objective);

/* MoEfication preprocessing, repacking (Eq. permuted_weights:
   W~_gate = W_gate Pi, W~_up = W_up Pi, W~_down = Pi^T W_down).  With the
   neurons stored as rows of W_gate / W_up and columns of W_down:
     W_gate_out[j][:] = W_gate[perm[j]][:],  W_up_out[j][:] = W_up[perm[j]][:],
     W_down_out[:][j] = W_down[:][perm[j]]
   so that expert e of the MoEfied FFN is the block of new neurons
   [64e, 64e + 64) that every other call of this library reads.  Device
   pointers: perm [d_ff] int32; weights in desc->dtype; W_gate / W_gate_out
   are used only for PP_ACT_SWIGLU (required then).  No output may overlap an
   input or another output (PP_ERR_INVALID_ARG).  Device-side check: an
   entry of perm outside [0, d_ff), or repeated, records PP_ERR_INVALID_ARG
   in the workspace status (pp_get_device_status); rows and columns for
   out-of-range entries are written as zeros.  Workspace:
   pp_workspace_size(desc, 0) bytes, initialised. */
pp_status pp_moefy_permute(const pp_desc *desc, const int32_t *perm, const void *W_gate, const void *W_up,
                           const void *W_down, void *W_gate_out, void *W_up_out, void *W_down_out, void *ws,
                           size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------------
 * The attention side of a decode step: rotary positions, a paged key/value
 * cache, and attention of new tokens over it.  A step appends its new tokens
 * (pp_kv_append), attends (pp_tree_attention) and, when the new tokens were a
 * tree of drafts, keeps the accepted path (pp_kv_commit).  The paper leaves
 * attention unchanged; these calls supply the rest of the layer around the
 * sparse FFN.
 *
 * Shapes: heads of head_dim = D elements, n_heads query heads in groups of
 * n_heads / n_kv_heads that share one key head (query head h reads key head
 * h / (n_heads / n_kv_heads)).  D is a multiple of 8 (bf16) or 4 (fp32), at
 * most 256.  Token tensors q, k, v, out are [n_tokens][heads][D] with the
 * heads of a token contiguous and a caller-given stride between tokens (in
 * elements, a multiple of 16 bytes), so that the parts of one fused
 * projection [n_tokens][(n_heads + 2 n_kv_heads) D] can be passed as they are.
 * ------------------------------------------------------------------------ */

/* A layer's key and value pages: entry j of a sequence lies in page
   pages[b][j / page_size] at offset j % page_size, head h at
     base + page * page_stride + offset * token_stride + h * head_stride
   (strides in elements, multiples of 16 bytes; the same for k and v).  The
   strides give both usual orders of a page, [page_size][n_kv_heads][D] and
   [n_kv_heads][page_size][D].  What pages hold past a sequence's length may
   be anything, NaN included.  The calls that write (pp_kv_append,
   pp_kv_commit) want entries apart: from the smallest stride up, pages,
   tokens, heads and layers each step past all that the ones before span
   (PP_ERR_INVALID_ARG; a dimension of one may carry any stride). */
typedef struct pp_cache {
    int dtype;        /* pp_dtype of the pages and of q, k, v, out */
    int n_heads;      /* query heads, a multiple of n_kv_heads     */
    int n_kv_heads;
    int head_dim;     /* D                                         */
    int page_size;    /* tokens per page, >= 1                     */
    int n_pages;      /* pages behind k and v                      */
    int64_t page_stride, token_stride, head_stride;
    void *k, *v;      /* device                                    */
} pp_cache;

/* The step's sequences.  Sequence b brings the new tokens
   [q_start[b], q_start[b + 1]) of the token tensors, which follow ctx_len[b]
   cached ones; new token i is cache entry ctx_len[b] + i.  Tokens from
   q_start[n_seqs] on are padding: no call reads or writes anything for them.
   A sequence may bring no token and may have no cached one.  Found on the
   device: q_start not ascending or past n_tokens, a negative ctx_len, more
   entries than max_pages pages hold (the sequence is skipped) and a page
   number outside [0, n_pages) (its entries are not written and read as
   zeros) record PP_ERR_INVALID_ARG in the workspace status. */
typedef struct pp_batch {
    int n_seqs;
    int n_tokens;           /* rows of the token tensors           */
    int max_pages;          /* row length of pages                 */
    const int32_t *q_start; /* [n_seqs + 1] device                 */
    const int32_t *ctx_len; /* [n_seqs] device                     */
    const int32_t *pages;   /* [n_seqs][max_pages] device          */
} pp_batch;

/* Which elements of a head form pair i of the rot_dim / 2 rotated pairs:
   HALF (i, i + rot_dim / 2), INTERLEAVED (2 i, 2 i + 1). */
typedef enum pp_rope_layout { PP_ROPE_HALF = 0, PP_ROPE_INTERLEAVED = 1 } pp_rope_layout;

/* Rotation of the first rot_dim elements of a head (the others are copied):
   pair (a, b) at position s becomes
     scale * (a cos(s f_i) - b sin(s f_i),  b cos(s f_i) + a sin(s f_i)).
   The angle is reduced to one turn before it is rounded, so its error does
   not grow with the position. */
typedef struct pp_rotation {
    int rot_dim;           /* a multiple of 4, 4 <= rot_dim <= head_dim      */
    int layout;            /* pp_rope_layout                                 */
    float scale;           /* 1, or the attention factor of YaRN             */
    const float *inv_freq; /* f [rot_dim / 2], radians per position, device  */
} pp_rotation;

/* How the frequencies f_i = base^(-2 i / rot_dim) are stretched for contexts
   longer than the trained one.
   NONE; LINEAR: f_i / factor; NTK: base * factor^(rot_dim / (rot_dim - 2)) in
   place of base; BANDED: f_i where the wavelength 2 pi / f_i is below
   trained_len / high, f_i / factor where it is above trained_len / low, and
   the mean of both weighted by (trained_len f_i / 2 pi - low) / (high - low)
   between; YARN: f_i (1 - r_i) + f_i / factor r_i with r_i rising linearly
   from 0 to 1 between the pairs that turn `high` and `low` times over
   trained_len positions (rounded outwards to whole pairs), and the rotation
   scaled by 0.1 ln(factor) + 1. */
typedef enum pp_rope_scaling {
    PP_ROPE_NONE = 0, PP_ROPE_LINEAR = 1, PP_ROPE_NTK = 2, PP_ROPE_BANDED = 3, PP_ROPE_YARN = 4
} pp_rope_scaling;

/* HOST routine, run once per model: writes f (inv_freq [rot_dim / 2], host
   memory, computed in fp64 and rounded once) and *scale for a pp_rotation.
   low, high and trained_len are read for BANDED and YARN only.  Errors:
   PP_ERR_INVALID_ARG (NULL output, unknown kind, base or factor not positive
   and finite, high <= low, low <= 0, trained_len < 1), PP_ERR_SHAPE (rot_dim). */
pp_status pp_rope_frequencies(int scaling, int rot_dim, double base, double factor, double low, double high,
                              int trained_len, float *inv_freq, float *scale);

/* y = x rotated by its tokens' positions: x, y [n_tokens][n_heads][head_dim]
   in dtype, rows x_stride and y_stride elements apart, positions [n_tokens]
   int32 (any value).  inverse != 0 rotates back (sin replaced by -sin), which
   is also the backward pass: the gradient of x is the gradient of y rotated
   back.  y may be x itself with the same stride; other overlaps are
   PP_ERR_INVALID_ARG.  Arithmetic in fp32, rounded once. */
pp_status pp_rope(int dtype, const pp_rotation *rot, const int32_t *positions, int n_tokens, int n_heads,
                  int head_dim, const void *x, int64_t x_stride, void *y, int64_t y_stride, int inverse,
                  void *stream);

/* Norm of each query and key head ahead of its rotation: a head's row x
   becomes x / sqrt(mean(x^2) + eps) * gamma, with one weight vector for all
   query heads and one for all key heads.  Squares are summed in fp32. */
typedef struct pp_head_norm {
    float eps;            /* >= 0                                              */
    const void *q_gamma;  /* [head_dim] device, in the tensors' dtype; NULL: ones */
    const void *k_gamma;
} pp_head_norm;

/* q_out, k_out = q, k normed and then rotated by their tokens' positions, in
   one pass: q [n_tokens][n_heads][head_dim], k [n_tokens][n_kv_heads][head_dim]
   (n_kv_heads 0: no keys, any n_heads; k, k_out are not looked at).  rot NULL:
   no rotation, and positions are not looked at.  An output may be its own
   input with the same stride; other overlaps, with weights, positions and
   frequencies too, are PP_ERR_INVALID_ARG.  Arithmetic in fp32, rounded once
   at the end. */
pp_status pp_head_norm_rope(int dtype, const pp_head_norm *norm, const pp_rotation *rot, const int32_t *positions,
                            int n_tokens, int n_heads, int n_kv_heads, int head_dim, const void *q, int64_t q_stride,
                            const void *k, int64_t k_stride, void *q_out, int64_t q_out_stride, void *k_out,
                            int64_t k_out_stride, void *stream);

/* Backward pass of pp_head_norm_rope: from q, k as they went in and the
   gradients q_grad, k_grad of its outputs, the gradients dq, dk of q, k and
   (each unless NULL; written, not added to) dq_gamma, dk_gamma [head_dim] fp32
   of the weights, summed in fp32 over all tokens and heads in a fixed order.
   dq may be q_grad (or q) itself with the same stride, dk likewise; other
   overlaps of what is written, the workspace included, are PP_ERR_INVALID_ARG.
   Workspace: pp_head_norm_workspace_size bytes, 256-byte aligned; it need not
   be initialised, and is not looked at where no weight gradient is asked for. */
pp_status pp_head_norm_rope_grad(int dtype, const pp_head_norm *norm, const pp_rotation *rot, const int32_t *positions,
                                 int n_tokens, int n_heads, int n_kv_heads, int head_dim, const void *q,
                                 int64_t q_stride, const void *k, int64_t k_stride, const void *q_grad,
                                 int64_t q_grad_stride, const void *k_grad, int64_t k_grad_stride, void *dq,
                                 int64_t dq_stride, void *dk, int64_t dk_stride, float *dq_gamma, float *dk_gamma,
                                 void *ws, size_t ws_bytes, void *stream);

/* Workspace bytes of pp_head_norm_rope_grad (0 for an unsupported head_dim). */
size_t pp_head_norm_workspace_size(int head_dim);

/* Workspace bytes of pp_kv_append, pp_tree_attention and pp_kv_commit for
   this cache, whatever the batch (0 for an unsupported one).  Initialise it
   with pp_workspace_init; errors found on the device are read with
   pp_get_device_status.  A recorded bad argument does not keep this call or
   later ones from computing what is right; after PP_ERR_TIMEOUT (which
   replaces an earlier code) initialise the workspace again. */
size_t pp_attn_workspace_size(const pp_cache *cache);

/* Append the new tokens' keys and values to the cache and rotate on the way:
   k is rotated and written to its page, v copied to its page, q rotated into
   q_out (q and q_out may both be NULL; q_out may be q itself).  rot NULL: no
   rotation.  positions [n_tokens] int32, or NULL for ctx_len[b] + i (the
   nodes of a drafted tree sit at ctx_len[b] + depth instead).  One launch. */
pp_status pp_kv_append(const pp_cache *cache, const pp_batch *batch, const pp_rotation *rot,
                       const int32_t *positions, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                       const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride, void *ws,
                       size_t ws_bytes, void *stream);

/* Attention of the new tokens over the cache, their own entries (appended
   before) included:
     out_t = sum_j p_tj v_j,  p_t = softmax over the visible j of scale q_t . k_j
   for every query head.  Every new token sees all ctx_len[b] cached tokens of
   its sequence; of the sequence's new tokens it sees
     mask NULL:  those up to and including itself (a prompt, a single token);
     otherwise:  token j if bit j % 32 of word j / 32 of its mask row is set;
                 mask [n_tokens][mask_words] uint32, tokens past 32 mask_words
                 are not seen, bits past the sequence's tokens are not read
                 as tokens (a drafted tree: the node's ancestors and itself).
   A token that sees nothing gets zeros.  Entries that a token does not see
   do not reach its output, whatever they hold.  Scores, maxima, sums and
   outputs are fp32 (weights below 2^-126 of their maximum count as zero); the
   bf16 path rounds the softmax weights to bf16 for the product with v, and out
   is rounded once.  The same call gives the same bits every time.  out must
   not overlap q.  scale: positive and finite.  bf16 runs on the tensor cores,
   fp32 on the CUDA cores; one launch, or two where sequences bring many query
   rows a key head. */
pp_status pp_tree_attention(const pp_cache *cache, const pp_batch *batch, const void *q, int64_t q_stride,
                            const uint32_t *mask, int mask_words, float scale, void *out, int64_t out_stride,
                            void *ws, size_t ws_bytes, void *stream);

/* Keep the accepted path of a drafted tree: for sequence b the entries of its
   new tokens path[b][0] < path[b][1] < ... (n_accept[b] of them, numbered
   within the sequence's new tokens) move to the entries ctx_len[b],
   ctx_len[b] + 1, ..., and new_len[b] = ctx_len[b] + n_accept[b] (new_len may
   be NULL; it must not overlap the inputs).  cache gives the first layer's
   pages; layer l's lie l * layer_stride elements further (not read for one
   layer; 0 is refused for more); n_layers >= 1.  A
   path that is not ascending or leaves the sequence's new tokens, or
   n_accept outside [0, max_path], records PP_ERR_INVALID_ARG and leaves the
   sequence as it was (new_len[b] = ctx_len[b]).  One launch for all layers. */
pp_status pp_kv_commit(const pp_cache *cache, const pp_batch *batch, int n_layers, int64_t layer_stride,
                       const int32_t *path, int max_path, const int32_t *n_accept, int32_t *new_len, void *ws,
                       size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------------
 * The cache in 8 bits.  Keys and values are held as e4m3 codes with an fp32
 * scale for each block of tokens and key head: an entry's value is
 * code * scale.  A cache of half the bytes, for the attention of steps that
 * are bound by reading it.  The same steps as above: append, attend, commit;
 * and entries read back.
 * ------------------------------------------------------------------------ */

/* A layer's pages in 8 bits.  Codes lie as pp_cache's elements do, one byte
   each (strides in bytes, multiples of 16; head_dim a multiple of 16, at most
   256).  `block` consecutive entries (16, 32, 64 or 128; page_size is a
   multiple of it) share a scale: that of page p, head h and the block that
   starts at offset i block is scale[(p n_kv_heads + h) (page_size / block) + i].
   The scales that pp_kvq_append and pp_kvq_commit write are powers of two, at
   least 2^-60; others (a cache filled elsewhere) may be any positive normal
   number up to 2^119.  What is not finite is held as the NaN code; what is
   finite stays so (at the scale 2^120 magnitudes from 248 * 2^120 on become
   240 * 2^120, since the code 256 would be 2^128). */
typedef struct pp_cache8 {
    int dtype;        /* pp_dtype of q, k, v, out (the tensors, not the pages) */
    int n_heads, n_kv_heads, head_dim, page_size, n_pages;
    int block;        /* tokens that share a scale */
    int64_t page_stride, token_stride, head_stride;
    void *k, *v;      /* device, codes  */
    float *k_scale, *v_scale; /* device, [n_pages][n_kv_heads][page_size / block] */
} pp_cache8;

/* Workspace bytes of the calls on this cache (0 for an unsupported one), used
   as that of pp_attn_workspace_size. */
size_t pp_kvq_workspace_size(const pp_cache8 *cache);

/* pp_kv_append to an 8-bit cache.  norm (may be NULL) is applied to the heads
   of q and k ahead of the rotation; what is written is rounded once, from the
   fp32 values.  The scale of a block that holds no cached entry (none before
   ctx_len[b]) is the smallest power of two with 448 scale >= the largest
   finite magnitude of its new entries; a block that holds cached ones keeps
   its scale unless 448 times it is less than that, and then gets the new
   entries' scale, its cached codes rounded again at it.  So the block that the
   first new token falls into is rewritten: it belongs to one sequence.  Scales
   do not shrink while entries stay: a drafted token that made its block's
   scale grow leaves it so when it is rejected, and cached values below 2^-6 of
   that scale are held in steps of 2^-9 of it. */
pp_status pp_kvq_append(const pp_cache8 *cache, const pp_batch *batch, const pp_head_norm *norm, const pp_rotation *rot,
                        const int32_t *positions, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                        const void *v, int64_t v_stride, void *q_out, int64_t q_out_stride, void *ws, size_t ws_bytes,
                        void *stream);

/* Entries back as numbers: row t of k_out, v_out [n_tokens][n_kv_heads]
   [head_dim] (cache->dtype) becomes the entry of the batch's token t, entry
   ctx_len[b] + i of its sequence: with ctx_len 0 and q_start at the sequences'
   lengths, whole sequences; with a step's own batch, what it appended.  Values
   are rounded once (powers of two as scales: not at all).  Rows of padding and
   of skipped sequences are left as they are; entries of a bad page give zeros. */
pp_status pp_kvq_read(const pp_cache8 *cache, const pp_batch *batch, void *k_out, int64_t k_out_stride, void *v_out,
                      int64_t v_out_stride, void *ws, size_t ws_bytes, void *stream);

/* pp_tree_attention over an 8-bit cache: the same masks, shapes and results,
   with code * scale for the keys and values.  bf16, where sequences bring up
   to 16 query rows a key head on average (where one may bring many, for those
   with up to 16 alone): the codes are multiplied as they are, and queries and
   weights as sums of e4m3 numbers; up to three launches.  That holds a query
   element exactly down to 2^-14 of its head's largest, and below to 2^-21 of
   the largest; and a weight, times its block's value scale, to 2^-8 of itself
   (as in bf16) or 2^-41 of the largest such product of its row.  With more
   rows, the codes are made bf16 (exact for powers of two as scales), which
   costs more than reading half the bytes saves: for drafted trees and prompts
   pp_tree_attention over a bf16 cache is the faster call. */
pp_status pp_kvq_tree_attention(const pp_cache8 *cache, const pp_batch *batch, const void *q, int64_t q_stride,
                             const uint32_t *mask, int mask_words, float scale, void *out, int64_t out_stride, void *ws,
                             size_t ws_bytes, void *stream);

/* pp_kv_commit on an 8-bit cache: layer l's codes lie l * layer_stride bytes
   and its scales l * scale_layer_stride floats further.  The entries' values
   move.  Of the blocks that they move into, one in which entries stay (cached
   ones, or accepted ones in their place already) keeps its scale as in
   pp_kvq_append, any other gets the scale that its entries need.  Entries past
   the accepted ones are lost. */
pp_status pp_kvq_commit(const pp_cache8 *cache, const pp_batch *batch, int n_layers, int64_t layer_stride,
                        int64_t scale_layer_stride, const int32_t *path, int max_path, const int32_t *n_accept,
                        int32_t *new_len, void *ws, size_t ws_bytes, void *stream);

/* Synchronise `stream` and return the sticky device status of `ws`. */
pp_status pp_get_device_status(void *ws, void *stream);

/* Diagnostic: pp_layer for one bf16 token (T = 1) through the timeline
   instantiation of the fused decode kernel, which computes the same y and
   also records the GPU global timer (ns) at the phase boundaries of every
   CTA: stamps[CTA * 16 + i] for i = first instruction, preceding grid
   complete, x loaded, router logits published, selection made, union formed,
   gate/up loads issued, gate/up activations published, first activations of
   the down projection received, down products done, y written (0 where a CTA
   skips a phase: the caller zeroes stamps first, so that consecutive layers
   need nothing between their launches).  stamps: device uint64, at least
   256 * 16 entries (stamps_bytes).  Errors as pp_layer; a dtype
   other than bf16 is PP_ERR_DTYPE. */
pp_status pp_debug_decode_timeline(const pp_desc *desc, const void *x, const void *W_r, const void *W_gate,
                                   const void *W_up, const void *W_down, float p, void *y, void *ws,
                                   size_t ws_bytes, uint64_t *stamps, size_t stamps_bytes, void *stream);

/* Test hook for failure detection: enqueue one kernel that waits on a
   workspace flag nothing sets, with a limit of timeout_ns nanoseconds; it
   then records PP_ERR_TIMEOUT in the workspace status and returns.  No GPU
   fault, trap or hang is involved. */
pp_status pp_debug_wait_timeout(void *ws, size_t ws_bytes, long long timeout_ns, void *stream);

/* Human-readable name of a status code (static string). */
const char *pp_status_string(pp_status s);

/* Library version, "major.minor.patch". */
const char *pp_version(void);

#ifdef __cplusplus
}
#endif

#endif /* PRUNEPATH_H */
