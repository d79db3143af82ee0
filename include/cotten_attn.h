/*
 * cotten_attn.h -- C ABI of the MI355X (gfx950) cosine-similarity attention library.
 *
 * The operation (Cotten4Rec, section "Model Description"): for every head-slice
 * (b,h) with per-head matrices Q, K, V of N rows and d_h columns,
 *
 *     xhat   = x / sqrt(sum_c x_c^2 + eps)        row-wise, for rows of Q and of K
 *                                                 (section "Cosine Similarity and
 *                                                  CUDA Kernel": eps inside the root)
 *     S      = sum_j m_j khat_j^T v_j             d_h x d_h state of the reordered
 *                                                 CosineAttention  Qhat (Khat^T V)
 *     O_i    = scale * qhat_i S                   scale = the scalar normaliser
 *                                                 1/n^m of the scaled CosineAttention
 *
 * m_j in {0,1} is a key-padding mask (1 = valid key).  The mask acts on keys
 * only: O and dQ are produced for all N query rows, and dO of every row flows
 * into the gradients.  The backward entry point returns the exact gradients of
 * the expression above,
 *
 *     dS   = scale * sum_i qhat_i^T dO_i
 *     dQ_i = (g_i - qhat_i (qhat_i . g_i)) / r(q_i),   g_i = scale * dO_i S^T
 *     dV_j = m_j * khat_j dS
 *     dK_j = m_j * (h_j - khat_j (khat_j . h_j)) / r(k_j),   h_j = v_j dS^T
 *
 * with r(x) = sqrt(sum_c x_c^2 + eps); dK and dV rows of masked keys are written
 * as exact zeros.  If a batch row has no valid key, O = 0 for it.
 *
 * Learnable normaliser (the scaled CosineAttention, scale = 1/n^m with a learnable
 * exponent).  Instead of one scalar the caller may pass one scale per slice,
 * params->slice_scale[b*H+h], and ask the backward for
 *
 *     dlog_scale[b*H+h] = d loss / d log(scale_bh) = sum_i dO_i . O_i  (= <S, dS>)
 *
 * which costs the kernels nothing extra in memory traffic.  cotten_normaliser_fwd
 * fills slice_scale from one exponent per head and one n per sequence,
 * scale_bh = n_b^(-m_h), and cotten_normaliser_bwd reduces dlog_scale to the
 * gradient of the exponents, dm_h = -sum_b ln(n_b) * dlog_scale[b*H+h].
 *
 * Memory.  Every pointer is a DEVICE pointer owned by the caller.  Q, K, V, O,
 * dO, dQ, dK, dV are [B, H, N, d_h] row-major and contiguous (each slice (b,h) is
 * one contiguous N x d_h block) or, with params->layout = COTTEN_BNHD, [B, N, H, d_h]
 * (the layout of the per-head split of a d_model-wide projection: no transposes
 * around the call); element type given by `dtype`; mask is [B, N]
 * bytes shared by the H heads, or NULL for "every key valid".  Tensor base
 * pointers must be 16-byte aligned.  Outputs must not overlap inputs or each
 * other.  Masked K/V rows are never dereferenced into arithmetic: they may hold
 * anything, NaN and Inf included.
 *
 * Arithmetic.  Row norms, the state and every accumulation are fp32 whatever
 * the I/O type (the paper keeps norms and partial sums in float32 under 16-bit
 * I/O).  Results are deterministic: reductions use a fixed order, no float
 * atomics, so two calls on the same inputs give identical bits.
 *
 * Execution.  Calls only enqueue kernels on `stream` (a hipStream_t passed as
 * void*; NULL = the default stream) and return; they never synchronise.  The
 * library runs on the device that is current in the calling thread.
 *
 * Workspace.  Long sequences are split over several workgroups per slice; the
 * partial d_h x d_h states travel through a workspace of
 * cotten_attn_workspace_bytes(...) bytes (0 when a shape needs none: every
 * sequence of at most 256 rows, except in the backward over fewer than 86 slices of
 * 16-bit d_h = 128, and longer ones when B*H fills the device).  The size of a shape may
 * change from one version of the library to the next: ask for it.  The
 * library never allocates, frees or synchronises: the caller brings the
 * workspace through cotten_params (its contents need no initialisation and mean
 * nothing afterwards; calls that share one must be ordered on one stream).  A
 * call whose shape needs a workspace and has none - params->workspace NULL, or
 * one of the plain entry points, which carry no params - returns
 * COTTEN_ERR_WORKSPACE_TOO_SMALL and enqueues nothing.  fp32 calls also run, slower, in less
 * than they ask for: cut into as many parts as the workspace holds the states of, two
 * or more (results agree to fp32 rounding of the states), and, where about a third of the
 * compute units or more work on uncut sequences, whole without one.
 *
 * Errors.  Every entry point returns a cotten_status; 0 is success, negative
 * values are listed below.  Argument validation happens on the host before any
 * device work and never touches the GPU, so a failed call has enqueued nothing.
 */
#ifndef COTTEN_ATTN_H_
#define COTTEN_ATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum cotten_dtype {
  COTTEN_F32 = 0,  /* float I/O                                   */
  COTTEN_BF16 = 1, /* bfloat16 I/O, fp32 norms and accumulation   */
  COTTEN_F16 = 2   /* IEEE half I/O, fp32 norms and accumulation (the mixed-precision mode
                      the paper trains in).  Results beyond +-65504 become Inf; the state
                      scale*S handed to the matrix cores is held in half as well, so
                      |scale * S| must stay in range (it does for scale ~ 1/N; the causal
                      variant takes states of any size)                                  */
} cotten_dtype;

typedef enum cotten_layout {
  COTTEN_BHND = 0, /* [B, H, N, d_h]: every slice (b,h) is one contiguous block (default)   */
  COTTEN_BNHD = 1  /* [B, N, H, d_h]: what the Q/K/V projections of a transformer layer
                      write and what its output projection reads; the d_h elements of a
                      row stay contiguous, the rows of a slice are H*d_h elements apart   */
} cotten_layout;

typedef enum cotten_feature_map {
  COTTEN_MAP_COSINE = 0, /* rows of Q and K divided by sqrt(sum_c x_c^2 + eps): the cosine
                            attention of the paper (default)                                */
  COTTEN_MAP_ELU1 = 1    /* ELU(x) + 1 element-wise on Q and K (x + 1 above zero, exp(x) below):
                            the linear-attention comparison model of the paper's section
                            "Linear Attention Models", on the same two products
                            O = scale * phi(Q) (phi(K)^T V) and their exact gradients.  No
                            normalising denominator (the section names none), eps unused.
                            Every supported element type and d_h; not with causal
                            (COTTEN_ERR_BAD_PARAM)                                          */
} cotten_feature_map;

typedef enum cotten_status {
  COTTEN_OK = 0,
  COTTEN_ERR_NULL_POINTER = -1,         /* a required tensor pointer is NULL            */
  COTTEN_ERR_BAD_SHAPE = -2,            /* B, H or N < 1, sizes overflow the launch, or
                                           params->layout is not a cotten_layout         */
  COTTEN_ERR_UNSUPPORTED_HEAD_DIM = -3, /* d_h not in {16, 32, 64, 128}                 */
  COTTEN_ERR_BAD_DTYPE = -4,            /* dtype is not a cotten_dtype                  */
  COTTEN_ERR_MISALIGNED = -5,           /* a tensor or workspace pointer not 16-B aligned */
  COTTEN_ERR_WORKSPACE_TOO_SMALL = -6,  /* the shape needs a workspace and params->workspace is
                                           NULL or params->workspace_bytes is too small
                                           (see Workspace, above)                        */
  COTTEN_ERR_BAD_PARAM = -7,            /* params->scale or params->eps is NaN or Inf, or
                                           an option combination that is not available   */
  COTTEN_ERR_LAUNCH = -8,               /* the HIP runtime refused a launch             */
  COTTEN_ERR_STATIC_SCRATCH = -9        /* cotten_attn_bwd_static only: the call needs more than
                                           COTTEN_STATIC_SCRATCH_BYTES of scratch, or the
                                           address of the scratch array could not be obtained */
} cotten_status;

typedef struct cotten_params {
  int dtype;              /* a cotten_dtype                                             */
  float scale;            /* scalar normaliser s; <= 0 selects the default 1/N          */
  float eps;              /* epsilon inside the square root; < 0 selects 1e-6; 0 allowed */
  void* workspace;        /* device buffer, 16-byte aligned; may be NULL when
                             cotten_attn_workspace_bytes() is 0 for the call            */
  size_t workspace_bytes; /* size of `workspace` (ignored when it is NULL)              */
  const float* slice_scale; /* device, [B*H] floats, or NULL.  When given, slice (b,h) uses
                               slice_scale[b*H+h] (finite, > 0) and `scale` is ignored      */
  float* dlog_scale;      /* backward only: device, [B*H] floats, or NULL.  When given it
                             receives sum_i dO_i . O_i of every slice (see above)          */
  int layout;             /* a cotten_layout: applies to Q, K, V, O, dO, dQ, dK and dV     */
  int causal;             /* 0: bidirectional (the paper's model).  1: row i attends only the
                             valid keys j <= i (the variant the paper's model leaves out, "no
                             causal mask"): O_i = scale * qhat_i sum_{j<=i} m_j khat_j^T v_j
                             and its exact gradients.  d_h in {16, 32, 64}; sequences of more
                             than 208 rows need the workspace that
                             cotten_attn_workspace_bytes_ex() reports; dlog_scale is not
                             available (COTTEN_ERR_BAD_PARAM)                              */
  float* saved_state;     /* device, [B*H, d_h, d_h] floats, 16-byte aligned, or NULL.  The state
                             S = sum_j m_j khat_j^T v_j of every slice (row a, column c; without
                             the scale), kept by the caller from the forward call to the
                             backward call of the same K, V, mask and eps, as the chain rule
                             allows (the backward needs S again, nothing else of the forward).
                             Forward: written when given.  Backward: when given, read instead
                             of rebuilding S from K and V (one pass over K, V less); results
                             agree with the rebuilding call to fp32 rounding of S.  The
                             kernels for rows of 256 bytes and more (fp32 d_h = 64, d_h = 128),
                             the 16-bit backward
                             for N <= 208 (its slice sits in LDS, rebuilding costs no memory
                             traffic) and a backward call that also asks for dlog_scale rebuild
                             S all the same; the causal variant has no such state and ignores
                             the field                                                     */
  int feature_map;        /* a cotten_feature_map: what is done to the rows of Q and K    */
} cotten_params;

/* Forward (reordered CosineAttention with scalar normaliser, "Model Description"):
 * O = scale * Qhat (Khat^T V) under the key mask.  fp32 I/O, scale = 1/N, eps = 1e-6.
 * Shapes for which cotten_attn_workspace_bytes() is not 0 need the _ex form. */
int cotten_attn_fwd(const void* Q, const void* K, const void* V, const uint8_t* mask,
                    void* O, int B, int H, int N, int d_h, void* stream);

/* Backward of the same expression: given dO writes dQ, dK, dV (formulas above).
 * fp32 I/O, scale = 1/N, eps = 1e-6.  The state S is rebuilt from K, V; nothing
 * saved by the forward call is needed (cotten_params.saved_state offers the other way).
 * Shapes for which cotten_attn_workspace_bytes() is not 0 need the _ex form. */
int cotten_attn_bwd(const void* Q, const void* K, const void* V, const uint8_t* mask,
                    const void* dO, void* dQ, void* dK, void* dV, int B, int H, int N,
                    int d_h, void* stream);

/* Same operations with explicit dtype, scale, eps and workspace.  `params` must not
 * be NULL. */
int cotten_attn_fwd_ex(const void* Q, const void* K, const void* V, const uint8_t* mask,
                       void* O, int B, int H, int N, int d_h, void* stream,
                       const cotten_params* params);
int cotten_attn_bwd_ex(const void* Q, const void* K, const void* V, const uint8_t* mask,
                       const void* dO, void* dQ, void* dK, void* dV, int B, int H, int N,
                       int d_h, void* stream, const cotten_params* params);

/* For callers that cannot allocate device memory and so cannot bring a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The same
 * operation, arguments and results (bit for bit) as cotten_attn_bwd_ex with a workspace of
 * COTTEN_STATIC_SCRATCH_BYTES, except that the partial states of long sequences go through a scratch array that is part of the library
 * image (a file-scope __device__ array of COTTEN_STATIC_SCRATCH_BYTES bytes; every GPU the
 * library runs on holds its own copy until the process ends) instead of params->workspace,
 * which is ignored together with params->workspace_bytes.  The call allocates, frees and
 * synchronises nothing.  A call that needs more scratch than the array holds
 * (cotten_attn_workspace_bytes(..., is_bwd = 1) > COTTEN_STATIC_SCRATCH_BYTES; fp32: than it
 * also runs in, see Workspace) returns COTTEN_ERR_STATIC_SCRATCH and enqueues nothing; 32 MiB covers, for instance, 64 slices of
 * 4096 rows at d_h = 64 (16 MiB) and every shape that needs no workspace at all.  All calls on
 * one GPU share that GPU's array, which keeps the last call's contents (every element a
 * call reads it has written before, so nothing needs clearing): calls on the same GPU must be
 * ordered on one stream; calls that overlap on one GPU race. */
#define COTTEN_STATIC_SCRATCH_BYTES (32u << 20)
int cotten_attn_bwd_static(const void* Q, const void* K, const void* V, const uint8_t* mask,
                           const void* dO, void* dQ, void* dK, void* dV, int B, int H, int N,
                           int d_h, void* stream, const cotten_params* params);

/* Learnable normaliser 1/n^m of the scaled CosineAttention ("Model Description"), one
 * exponent per head:  slice_scale[b*H+h] = n_b^(-m_h).  m: device, [H] floats.  n: device,
 * [B] int32 with n_b >= 1 (for instance the valid length of each sequence), or NULL for
 * n_b = N, the padded length.  slice_scale: device, [B*H] floats, written. */
int cotten_normaliser_fwd(const float* m, const int32_t* n, float* slice_scale, int B, int H,
                          int N, void* stream);

/* Gradient of the exponents from the backward call's dlog_scale:
 * dm[h] = -sum_b ln(n_b) * dlog_scale[b*H+h], summed in a fixed order.  dm: device, [H]
 * floats, written.  n as above. */
int cotten_normaliser_bwd(const float* dlog_scale, const int32_t* n, float* dm, int B, int H,
                          int N, void* stream);

/* Bytes of workspace the given call would use if it has them (pure host arithmetic; 0 for an
 * unsupported shape).  Grows like B*H*d_h^2 times the number of sequence splits,
 * never like N*d_h or N^2: the method keeps only the d_h x d_h state ("Memory and
 * Compute Complexity"). */
size_t cotten_attn_workspace_bytes(int B, int H, int N, int d_h, int dtype, int is_bwd);

/* The same for a call with these params (dtype, causal and feature_map are looked at): what
 * params->workspace must hold.  Differs from the function above for the causal variant, whose
 * sequences of more than 208 rows pass up to one d x d state per 208 rows and slice through the
 * workspace (two in the backward call).  0 for invalid arguments or params == NULL.  Host
 * only, no device work. */
size_t cotten_attn_workspace_bytes_ex(int B, int H, int N, int d_h, int is_bwd,
                                      const cotten_params* params);

/* Static, NUL-terminated description of a status code. */
const char* cotten_status_string(int status);

/* ---- Gated delta rule -----------------------------------------------------------------------
 *
 * The recurrent form of the causal linear attention above, with a state that can forget and
 * correct itself.  For every slice (b,h), with unit rows xhat = x / sqrt(sum_c x_c^2 + eps)
 * of Q and K as above, a_t = exp(g_t) and the state S (d_h x d_h, row a, column c):
 *
 *     u_t = beta_t * (v_t - a_t * S_{t-1}^T khat_t)        what is still missing of v_t
 *     S_t = a_t * S_{t-1} + khat_t u_t^T                   decay, then write
 *     O_t = scale * S_t^T qhat_t
 *
 * g (log decays, any sign; -inf empties the state) and beta are float, [B, H, N] or, with
 * COTTEN_BNHD, [B, N, H]; Q, K, V, O and their gradients are as above.  A masked token (mask
 * byte 0) leaves the state as it is: a = 1, beta = 0, and its K, V, g and beta are not
 * used, so they may hold anything; O exists for all N rows (queries are not masked).  Gradients of masked K, V, g
 * and beta are exact zeros.  A sequence without a valid token keeps its initial state.
 *
 * States are fp32, [B, H, d_h, d_h].  Sums, states and norms are fp32 or wider whatever the I/O type,
 * and operands of products are not rounded to 16 bits.  A value that is not finite in a row
 * that takes part makes the results of its column not finite from its group of 32 tokens on.
 *
 * Calls enqueue on `stream` only, allocate nothing, and give the same bits for the same
 * arguments.  A call is several launches that pass data through its workspace and `kept`: calls from several host threads
 * need buffers of their own, also on one stream, where the launches of two calls may alternate.
 *
 * d_h in {16, 32, 64, 128}; B * H up to 2^22, and the rows of a slice, or 32 of them if there are fewer, within 2^31 bytes
 * from the first to the last (COTTEN_ERR_BAD_SHAPE beyond).  */
typedef struct cotten_delta_params {
  int dtype;                  /* a cotten_dtype: of Q, K, V, O and their gradients               */
  float scale;                /* factor of O; <= 0 selects 1                                     */
  float eps;                  /* inside the square roots; < 0 selects 1e-6; 0 allowed            */
  int layout;                 /* a cotten_layout                                                 */
  void* workspace;            /* device buffer of cotten_delta_workspace_bytes(), 16-byte aligned;
                                 may be NULL where that is 0 (any forward but those of few and
                                 long sequences without kept)                                    */
  size_t workspace_bytes;
  const float* initial_state; /* device, [B*H, d_h, d_h], or NULL: zeros                         */
  float* final_state;         /* forward: receives the state after row N-1, or NULL.  May be
                                 initial_state itself (a server's state, replaced in place)      */
  const float* dfinal_state;  /* backward: gradient of the final state, or NULL: zeros           */
  float* dinitial_state;      /* backward: receives the gradient of the initial state, or NULL   */
  void* kept;                 /* device buffer of cotten_delta_kept_bytes(), 16-byte aligned, or
                                 NULL.  Forward: receives what the backward of the same inputs
                                 needs of it.  Backward: what that forward wrote (without it the
                                 backward walks the sequence forwards first, in its workspace,
                                 with the same results)                                          */
  size_t kept_bytes;
} cotten_delta_params;

/* `params` must not be NULL.  N = 1 with final_state == initial_state is one step of a server. */
int cotten_delta_fwd(const void* Q, const void* K, const void* V, const float* g, const float* beta,
                     const uint8_t* mask, void* O, int B, int H, int N, int d_h, void* stream,
                     const cotten_delta_params* params);

/* Gradients of all inputs from dO (and params->dfinal_state).  initial_state is read where kept is NULL: it has to hold
 * what the forward call saw. */
int cotten_delta_bwd(const void* Q, const void* K, const void* V, const float* g, const float* beta,
                     const uint8_t* mask, const void* dO, void* dQ, void* dK, void* dV, float* dg,
                     float* dbeta, int B, int H, int N, int d_h, void* stream,
                     const cotten_delta_params* params);

/* Bytes of params->kept, and of params->workspace (with_kept: the call is given params->kept).
 * They grow like N * d_h * (d_h / 32 + 1), a forward's workspace like d_h * d_h.  0 for invalid arguments; host only. */
size_t cotten_delta_kept_bytes(int B, int H, int N, int d_h, int dtype);
size_t cotten_delta_workspace_bytes(int B, int H, int N, int d_h, int dtype, int is_bwd, int with_kept);

/* ---- Decay attention --------------------------------------------------------------------------
 *
 * The causal linear attention with one decay for each head, on the same unit rows: for every slice (b,h), with
 * a = exp(g[h]) and the state S (d_h x d_h, row a, column c),
 *
 *     S_t = a * S_{t-1} + khat_t v_t^T          O_t = scale * S_t^T qhat_t
 *
 * g is float, [H]: log decays of any sign (-inf empties the state at every token).  A masked token (mask byte 0)
 * leaves the state as it is, and its K and V are not used, so they may hold anything; O exists for all N rows (queries
 * are not masked).  Gradients of masked K and V are exact zeros, those of g are summed over the batch in 64 bits.  A
 * sequence without a valid token keeps its initial state.  With g = 0 and no states it is the causal variant above.
 *
 * Types, layouts, states, precision, streams, limits of rows and what calls may share are those of the gated delta rule, but that
 * the products that make rows of 16-bit results keep 16 significant bits of their operands; B * H up to 2^20.  A value that is not finite in a row that takes part makes the results that hang on it not finite from its group
 * of 32 tokens on; so does a growth (g > 0) whose power by the number of the group's tokens that count is above what fp32 holds. */
typedef struct cotten_decay_params {
  int dtype;                  /* a cotten_dtype: of Q, K, V, O and their gradients               */
  float scale;                /* factor of O; <= 0 selects 1                                     */
  float eps;                  /* inside the square roots; < 0 selects 1e-6; 0 allowed            */
  int layout;                 /* a cotten_layout                                                 */
  void* workspace;            /* device buffer of cotten_decay_workspace_bytes(), 16-byte aligned;
                                 may be NULL where that is 0                                     */
  size_t workspace_bytes;
  const float* initial_state; /* device, [B*H, d_h, d_h], or NULL: zeros                         */
  float* final_state;         /* forward: receives the state after row N-1, or NULL.  May be
                                 initial_state itself (a server's state, replaced in place)      */
  const float* dfinal_state;  /* backward: gradient of the final state, or NULL: zeros           */
  float* dinitial_state;      /* backward: receives the gradient of the initial state, or NULL   */
} cotten_decay_params;

/* `params` must not be NULL.  N = 1 with final_state == initial_state is one step of a server. */
int cotten_decay_fwd(const void* Q, const void* K, const void* V, const float* g, const uint8_t* mask, void* O, int B, int H, int N,
                     int d_h, void* stream, const cotten_decay_params* params);
/* Gradients of all inputs from dO (and params->dfinal_state); dg, [H] floats, may be NULL.  Nothing of the forward call is kept:
 * the inputs and initial_state have to hold what it saw. */
int cotten_decay_bwd(const void* Q, const void* K, const void* V, const float* g, const uint8_t* mask, const void* dO, void* dQ,
                     void* dK, void* dV, float* dg, int B, int H, int N, int d_h, void* stream, const cotten_decay_params* params);
/* Bytes of params->workspace (with_dg: dg is given).  0 for invalid arguments; host only. */
size_t cotten_decay_workspace_bytes(int B, int H, int N, int d_h, int dtype, int is_bwd, int with_dg);

/* ---- Embedding of item ids -------------------------------------------------------------------
 *
 * The input of the layers (Cotten4Rec, "Model Description": E_t = s_t + P_t), with a factor:
 *
 *     E[b,n] = scale * W[ids[b,n]] + P[position_offset + n]
 *     dW[i]  = scale * sum of dE[b,n] over the tokens with ids[b,n] = i, in a fixed order
 *     dP[position_offset + n] = sum_b dE[b,n]
 *
 * W is [V, D], P [positions, D] (or NULL: none), E and dE [B, N, D], contiguous, all of one element type;
 * ids [B, N], int32 or int64.  A token with padding_idx, or with an id outside 0 ... V-1, has no row:
 * its E is its position's alone, and it gives dW nothing.  Sums are fp32, rounded once.  dW and dP are
 * dense and written whole, zeros included.  The same arguments give the same bits (sums of more than sixteen tokens are
 * sums of partial sums).
 *
 * The backward needs a workspace of cotten_embed_workspace_bytes() bytes (lists of the tokens sorted by id, and
 * partial sums), which calls from several host threads must not share, as above.  Calls enqueue on `stream` only and allocate nothing.  D up to 65536, V below 2^30, B * N below 2^31
 * (with dW up to 2^29), with dP up to 2^22 positions, and tables and gradients of no more than a launch reaches: a workgroup for
 * 64 KB of zeros, for 64 pieces of up to 16 bytes of dP's columns, or for a row of more than 64 KB, of 2^23 in
 * all (COTTEN_ERR_BAD_SHAPE beyond, before anything is enqueued). */
typedef struct cotten_embed_params {
  int dtype;            /* a cotten_dtype: of W, P, E and their gradients                        */
  int id_bytes;         /* 4 or 8                                                                */
  float scale;          /* as it is (finite)                                                     */
  int padding_idx;      /* -1: none                                                              */
  int positions;        /* rows of P; position_offset + N at most                                */
  int position_offset;
  void* workspace;      /* backward: 16-byte aligned device buffer                               */
  size_t workspace_bytes;
} cotten_embed_params;

int cotten_embed_fwd(const void* ids, const void* W, const void* P, void* E, int B, int N, int D, int V,
                     void* stream, const cotten_embed_params* params);
/* dW or dP may be NULL, not both. */
int cotten_embed_bwd(const void* ids, const void* dE, void* dW, void* dP, int B, int N, int D, int V,
                     void* stream, const cotten_embed_params* params);
/* 0 for invalid arguments; host only. */
size_t cotten_embed_workspace_bytes(int B, int N, int D, int V);

/* ---- Dropout and the seam between two blocks --------------------------------------------------
 *
 * Dropout draws from a counter-based generator, Philox4x32 with ten rounds: the same (seed, offset) and
 * number of an element give the same decision, so no mask is stored, and the backward is the same call on
 * the upstream gradient.  Eight elements, numbered through the tensor, share a counter (number / 8, offset)
 * under the key `seed` and take 16 bits each, in order (of a word the lower half first); an element is
 * dropped where they are below t = floor(65536 p + 1/2), so p counts as t / 65536:
 *
 *     y = x * 65536 / (65536 - t), or 0 where dropped (whatever x holds there)
 *
 * Other offsets are other draws: a program counts its calls.  `step`, a device number that is added to offset,
 * lets a captured graph draw anew in every replay.  The seam, rows of D elements:
 *
 *     Y = X + alpha * gate * drop(N(F; post_weight, post_bias))        H = N(Y; next_weight, next_bias)
 *     N(x; w, b) = w (x - mu) / sqrt(mean (x - mu)^2 + eps) + b        mu = mean x, or 0 (COTTEN_NORM_RMS)
 *
 * Without post_weight F goes in as it is, without next_weight there is no H, without gate it is 1; the number of an
 * element is that in F.  X, F, Y, H and their gradients are [B, N, D], contiguous; weights, biases and
 * the gate are [D], the gate with gate_per_sequence [B, D]; all are of one element type.  Sums are fp32, in a fixed
 * order, every result is rounded once (H comes from the row Y before its rounding).  D up to 8192, B * N below 2^31, up to
 * 2^40 elements for the dropout by itself.  y may be x, Y may be X, and H may be F (no others overlap).  The backward keeps nothing: it makes the rows again from
 * X and F, which have to hold what the forward saw.  A row is one of N = 1 for single tokens. */
typedef enum cotten_norm {
  COTTEN_NORM_RMS = 0,
  COTTEN_NORM_LAYER = 1
} cotten_norm;

typedef struct cotten_dropout_params {
  int dtype;           /* a cotten_dtype                                                         */
  double p;            /* 0 <= p, and below 1 as it counts (COTTEN_ERR_BAD_PARAM)                */
  uint64_t seed;
  uint64_t offset;     /* the number of the call                                                 */
  const int64_t* step; /* device, or NULL: added to offset                                       */
} cotten_dropout_params;

int cotten_dropout(const void* x, void* y, size_t n, void* stream, const cotten_dropout_params* params);

typedef struct cotten_residual_params {
  int dtype;             /* a cotten_dtype                                                       */
  int norm;              /* a cotten_norm: of both norms                                         */
  const void* post_weight;
  const void* post_bias; /* (only with post_weight)                                              */
  const void* gate;
  const void* next_weight;
  const void* next_bias; /* (only with next_weight)                                              */
  int gate_per_sequence;
  float alpha;           /* finite                                                               */
  float eps;             /* < 0 selects 1e-6; 0 allowed                                          */
  double p;              /* of the dropout, as above; 0: none                                    */
  uint64_t seed;
  uint64_t offset;
  const int64_t* step;
  void* workspace;       /* backward: 16-byte aligned device buffer                              */
  size_t workspace_bytes;
} cotten_residual_params;

/* What the backward writes besides dX and dF: each NULL where it is not wanted. */
typedef struct cotten_residual_grads {
  void* post_weight;
  void* post_bias;
  void* gate;
  void* next_weight;
  void* next_bias;
} cotten_residual_grads;

/* H is NULL exactly where next_weight is. */
int cotten_residual_fwd(const void* X, const void* F, void* Y, void* H, int B, int N, int D, void* stream,
                        const cotten_residual_params* params);
/* dY or dH may be NULL (zeros), not both. */
int cotten_residual_bwd(const void* X, const void* F, const void* dY, const void* dH, void* dX, void* dF, int B, int N, int D,
                        void* stream, const cotten_residual_params* params, const cotten_residual_grads* grads);
/* 0 for invalid arguments; host only. */
size_t cotten_residual_workspace_bytes(int B, int N, int D, int gate_per_sequence);

/* ---- A step of a beam search -----------------------------------------------------------------
 *
 * Of every sequence's K beams with their scores (sums of logarithms) and the logits of V items for each, the K
 * best continuations:
 *
 *     total[k, v] = scores[k] + logits[k, v] - log sum_v' exp(logits[k, v'])
 *
 * in falling order, of equal totals the one with the lower k * V + v.  A beam that ended (finished byte not 0)
 * goes on with the item `pad` alone, at its score; its logits are not read.  What else an ended beam could
 * go on with, and everything of a beam whose score, or sum of exponentials, is not finite, has the total -inf (taken
 * where nothing else is left).  A NaN among the logits counts as -inf.  Totals are compared in 64 bits, with sums in fp32 where
 * these decide and in 64 bits where candidates of two beams are nearer than that can tell apart.
 * logits [B, K, V] of one element type, contiguous; scores, new_scores float [B, K] (new_scores may be scores);
 * finished [B, K] bytes or NULL; parents (the beam 0 ... K-1 that is continued) and tokens (the item) int32 [B, K].  K up to 32, B * K
 * below 2^22, V below 2^30.  The workspace holds cotten_beam_workspace_bytes(); calls from several host threads must not share
 * one, as above.
 *
 * cotten_beam_reorder gives beam k what beam parents[k] of its sequence had, in place, for `bytes` bytes of
 * every beam (states of the delta rule or of the decay attention, [B, K, ...]; histories of items; flags): any contiguous tensor [B, K, ...].  Beams that stay
 * are not touched; a parent outside 0 ... K-1 leaves its beam as it is. */
typedef struct cotten_beam_params {
  int dtype;              /* a cotten_dtype: of the logits                                       */
  int pad;                /* 0 ... V-1 where finished is given (COTTEN_ERR_BAD_PARAM)            */
  void* workspace;        /* 16-byte aligned device buffer                                       */
  size_t workspace_bytes;
} cotten_beam_params;

int cotten_beam_select(const void* logits, const float* scores, const uint8_t* finished, float* new_scores, int32_t* parents,
                       int32_t* tokens, int B, int K, int V, void* stream, const cotten_beam_params* params);
int cotten_beam_reorder(void* state, const int32_t* parents, int B, int K, size_t bytes, void* stream);
/* 0 for invalid arguments; host only. */
size_t cotten_beam_workspace_bytes(int B, int K, int V);

#ifdef __cplusplus
}
#endif
#endif /* COTTEN_ATTN_H_ */
