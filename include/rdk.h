/*
 * rdk.h -- C ABI of the MI355X (gfx950) library for Redistributing Drafter Kernels (RDK).
 *
 * The library covers the data-parallel hot path of the method, and beside it what its drafter is trained on and what decodes the same
 * rows without drawing: the teacher's top logits, distillation from them, beam search; and what stands at a model's ends: log
 * probabilities of given tokens and embedding rows, with their gradients.  For a batch of B positions it
 * redistributes a vocabulary-pruned drafter's distribution q (n kept ids) onto the target
 * vocabulary (N ids) through a row-stochastic token-affinity kernel M (Alg. 1 of the paper), and
 * runs the accept / residual / sample step of speculative decoding against the target
 * distribution p (Alg. 4, steps 2 and 4-10).
 *
 * Conventions, valid for every entry point unless stated otherwise
 *  - Every data pointer is a DEVICE pointer owned by the caller (any allocator; 16-byte aligned).
 *    The library allocates no device memory: scratch comes in through `workspace`, whose size is
 *    given by the *_bytes queries.  Descriptor structs and out-parameters such as `size_t*` and
 *    `rdk_kernel_t**` are HOST pointers.
 *  - Work is enqueued on the HIP stream passed as `stream` (a hipStream_t cast to void*; NULL is the
 *    default stream).  Calls do not synchronise, except rdk_build_kernel with `validate != 0`.
 *    The redistribution, verification and sampling calls consist of kernel launches on that stream
 *    only (no copy, no memset, no allocation), so they may be recorded into a HIP graph and replayed;
 *    the seed and the counter offset are then those given at capture time.
 *  - Calls that use distinct workspaces may run concurrently on distinct streams; two calls that
 *    share a workspace must be ordered by the caller.
 *  - Matrices are row-major with a leading dimension given in ELEMENTS (ld >= row length).
 *  - Position b of a batch draws its random numbers from the counter-based generator
 *    Philox4x32-10 with key = seed and counter = (offset + b, 0): four words per position, mapped
 *    to [0,1) as (word >> 8) * 2^-24; word 0 picks the draft token, word 1 decides acceptance,
 *    word 2 picks the residual token, word 3 the bonus token.
 *  - Every function returns an rdk_status_t; nothing is written to outputs on error.
 */
#ifndef RDK_H
#define RDK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RDK_OK = 0,
    RDK_ERR_NULL = 1,           /* a required pointer is NULL */
    RDK_ERR_SHAPE = 2,          /* a size, leading dimension or count is out of range */
    RDK_ERR_DTYPE = 3,          /* unknown input kind / kernel format / mode */
    RDK_ERR_KEPT_IDS = 4,       /* kept ids not strictly ascending or outside [0, N) (validate only) */
    RDK_ERR_NOT_STOCHASTIC = 5, /* a supplied kernel has a negative entry or a row sum off 1 by > 1e-3 (validate only) */
    RDK_ERR_WORKSPACE = 6,      /* workspace or storage smaller than the *_bytes query says */
    RDK_ERR_UNSUPPORTED = 7,    /* combination not offered (e.g. exact redistribution with a sparse kernel) */
    RDK_ERR_HIP = 8,            /* a HIP call failed; see rdk_last_hip_error() */
    RDK_ERR_ALIGN = 9           /* a device pointer is not 16-byte aligned */
} rdk_status_t;

/* How the token-affinity kernel M (n x N, row = kept slot, column = target id) is stored. */
typedef enum {
    RDK_DENSE_F32 = 0,   /* every entry, fp32 */
    RDK_DENSE_BF16 = 1,  /* every entry, rounded to bf16, 16 bits per entry, packed for the matrix cores */
    RDK_SPARSE_TOPK = 2, /* per pruned id its k strongest kept neighbours; per kept id itself only */
    RDK_IDENTITY = 3     /* M = identity on the kept ids: RDK reduces to token-level intersection */
} rdk_kernel_format_t;

/* What a [B, len] input holds. */
typedef enum {
    RDK_PROB_F32 = 0,   /* non-negative fp32 weights (need not be normalised where noted) */
    RDK_LOGIT_F32 = 1,  /* fp32 logits; the softmax is applied on the fly */
    RDK_LOGIT_BF16 = 2  /* bf16 logits (uint16 bit patterns); widened to fp32, then softmax */
} rdk_input_kind_t;

typedef enum {
    RDK_LINEAR_TAYLOR = 0, /* first-order closed form, Eq. 3 of the paper; needs p, no matrix */
    RDK_LINEAR_SPARSE = 1  /* Alg. 1 step 2 with the top-k sparse kernel; O(N k) */
} rdk_linear_mode_t;

typedef struct rdk_kernel rdk_kernel_t; /* opaque host object; points into caller-owned device storage */

/*
 * Inputs of the kernel construction (section 3, "Token-affinity priors", Eq. 2):
 *   M_ij = exp(Omega_ij / tau) / sum_k exp(Omega_ik / tau),  i a kept id, j any target id.
 * Omega is given either through embeddings (Omega_ij = cosine similarity of rows kept_ids[i] and j,
 * the stand-in for the covariance statistics of the paper) or not at all, when the caller brings a
 * finished kernel (dense_M, or the sparse triple).
 *
 * Sparse format (RDK_SPARSE_TOPK): row i keeps the diagonal entry (i, kept_ids[i]) and, for every
 * pruned id j that ranks slot i among its k most similar kept slots (ties: lower slot), the entry
 * (i, j); Eq. 2 is applied over the retained entries, so rows still sum to one.  Its interchange
 * form is keyed by pruned slot u (the u-th id not in kept_ids, ascending):
 *   sparse_idx[u*k + t] = kept slot, sparse_w[u*k + t] = M[slot, id(u)], self_w[i] = M[i, kept_ids[i]].
 */
typedef struct {
    int32_t N;                 /* target vocabulary size |T| */
    int32_t n;                 /* number of kept ids |I|, 1 <= n <= N */
    int32_t d;                 /* embedding width (ignored without embeddings) */
    int32_t k;                 /* neighbours per pruned id, 0 <= k <= min(n, 64); RDK_SPARSE_TOPK only */
    const int32_t *kept_ids;   /* [n] device: the kept target ids, strictly ascending */
    const float *embeddings;   /* [N, d] device, row-major, or NULL */
    const float *dense_M;      /* [n, N] device, row-major, row-stochastic, or NULL (dense formats) */
    const int32_t *sparse_idx; /* [(N-n), k] device or NULL (sparse format) */
    const float *sparse_w;     /* [(N-n), k] device or NULL */
    const float *self_w;       /* [n] device or NULL */
    float tau;                 /* temperature of Eq. 2, > 0 (ignored without embeddings) */
    rdk_kernel_format_t format;
    int32_t validate;          /* != 0: check kept_ids (and a supplied kernel) on the device, then synchronise */
} rdk_kernel_desc_t;

/*
 * Bytes of device storage the finished kernel occupies, and of scratch the build needs.  A top-k kernel takes 8 bytes per
 * neighbour (k rounded up to 16) and, with n <= 20320 and at least 128 KB of those, holds them a second time in the order that
 * larger batches read them in: about 48 N (ceil(k / 8) + 1/2) bytes more, whichever batches it is used for (N = 151936, n = 16384,
 * k = 32: 34.7 MB and 32.8 MB; N = 32000, n = 8000, k = 16: 3.1 MB and 3.8 MB).
 */
rdk_status_t rdk_kernel_storage_bytes(const rdk_kernel_desc_t *desc, size_t *storage_bytes,
                                      size_t *build_workspace_bytes);

/*
 * Token features from data (Sec. 3, "Token-affinity priors": Omega is estimated from data).  z [T, ldz] holds T
 * sampled score rows over the N target ids (target logits, fp32 or bf16, or probabilities); features [N, ldf]
 * receives  F[j, t] = z[t, j] - mean_t z[., j].  Passed as `embeddings` (d = T, row stride T: use ldf = T) to
 * rdk_build_kernel, Omega_ij becomes the correlation of the scores of tokens i and j over the sample, i.e. the
 * covariance matrix of the standardised scores; it is 1 on the diagonal and at most 1 elsewhere, as Eq. 2's
 * evaluation here assumes.  T >= 2; a token whose score never varies has no direction and must not be passed on.
 * No workspace; enqueues on `stream`.
 */
rdk_status_t rdk_features_from_scores(const void *z, rdk_input_kind_t z_kind, int64_t ldz, int32_t T, int32_t N,
                                      float *features, int64_t ldf, void *stream);

/*
 * Build M into `storage` (Eq. 2; a one-off preprocessing step, Sec. 3).  `storage` must stay
 * alive and untouched for the life of the kernel object; `workspace` may be reused once the
 * stream has passed the build.  *out receives the host handle.
 */
rdk_status_t rdk_build_kernel(const rdk_kernel_desc_t *desc, void *storage, size_t storage_bytes,
                              void *workspace, size_t workspace_bytes, void *stream,
                              rdk_kernel_t **out);

/* Frees the host object only; the device storage belongs to the caller. */
rdk_status_t rdk_destroy_kernel(rdk_kernel_t *kernel);

/* Copy a sparse kernel out in the interchange form described above (device buffers). */
rdk_status_t rdk_kernel_get_sparse(const rdk_kernel_t *kernel, int32_t *sparse_idx, float *sparse_w,
                                   float *self_w, void *stream);

/* Copy a dense kernel out as fp32 [n, ldm] (bf16 storage is widened). */
rdk_status_t rdk_kernel_get_dense(const rdk_kernel_t *kernel, float *dense_M, int64_t ldm,
                                  void *stream);

/* Scratch needed by either redistribute call for B positions with this kernel. */
rdk_status_t rdk_workspace_bytes(const rdk_kernel_t *kernel, int32_t B, size_t *bytes);

/*
 * Alg. 1, steps 1-2, exact form:  q_prime[b, :] = M^T TLI(q[b, :]).
 *   q        [B, ldq]  drafter weights or logits over the n kept slots (slot s <-> id kept_ids[s]).
 *            PROB: any non-negative row; step 1 (Eq. 1) divides by its sum.  A row whose sum is zero has no
 *            image under Eq. 1: every redistribution call (exact, both linear forms, the fused call and the
 *            draft draw) returns the zero row for it, so that verification sees alpha = 0, resid_mass = sum(p),
 *            draft_ids = -1, accept = 0, and draws resid_ids from the target row alone.
 *            LOGIT: the softmax over the n slots, which equals Eq. 1 applied to a full softmax; a row of which every
 *            logit is -inf is one whose sum is zero.
 *   q_prime  [B, ldo]  fp32, the redistributed drafter over all N target ids.
 * Kernel format must be DENSE_F32, DENSE_BF16 or IDENTITY.  With DENSE_BF16 the kernel entries are rounded to
 * bf16 and the normalised drafter rows to eleven significant bits (both are fed to the matrix cores as fp16 numbers
 * scaled by 2^15; values below 2^-29 count as zero), products accumulate in fp32 and each output row is rescaled
 * to sum to one: every output is within 2e-3 (relative, plus 1e-7) of the exact product with the kernel as stored.
 */
rdk_status_t rdk_redistribute_exact(const rdk_kernel_t *kernel, const void *q,
                                    rdk_input_kind_t q_kind, int64_t ldq, int32_t B,
                                    float *q_prime, int64_t ldo, void *workspace,
                                    size_t workspace_bytes, void *stream);

/*
 * Alg. 1, steps 1-2, linear-time forms.
 *   RDK_LINEAR_TAYLOR (Eq. 3): theta = p^T q', pt_j = (N q'_j + theta p_j) / (N + p_j),
 *     q_prime = pt / sum(pt), with q' = TLI(q) scattered to the kept ids.  Needs p [B, ldp]
 *     (PROB rows must sum to one); uses only kept_ids of the kernel (any format).
 *   RDK_LINEAR_SPARSE: q_prime = M^T q' with the top-k sparse kernel (format RDK_SPARSE_TOPK or
 *     RDK_IDENTITY); p is ignored and may be NULL.
 */
rdk_status_t rdk_redistribute_linear(const rdk_kernel_t *kernel, rdk_linear_mode_t mode,
                                     const void *p, rdk_input_kind_t p_kind, int64_t ldp,
                                     const void *q, rdk_input_kind_t q_kind, int64_t ldq,
                                     int32_t B, float *q_prime, int64_t ldo, void *workspace,
                                     size_t workspace_bytes, void *stream);

/* Verification of a batch (Alg. 4, steps 2 and 4-10). */
typedef struct {
    int32_t B;            /* positions */
    int32_t N;            /* target vocabulary size */
    int32_t gamma;        /* draft tokens per sequence; 0 = no per-sequence scan; else B % gamma == 0 */
    int32_t sample_draft; /* != 0: draw d ~ q_prime into draft_ids; 0: draft_ids holds the caller's tokens */
    uint64_t seed;        /* Philox key */
    uint64_t offset;      /* Philox counter of position 0 */
} rdk_verify_desc_t;

/* With 1 <= gamma <= 63 the size holds 16 bytes per position for the per-sequence scan (steps 4-10) to run inside the
 * last kernel.  A workspace of the size for gamma = 0 is enough for any gamma: the scan is then a launch of its own. */
rdk_status_t rdk_verify_workspace_bytes(const rdk_verify_desc_t *desc, size_t *bytes);

/*
 * Per position b, with q' = q_prime[b, :] and p = the target row:
 *   alpha[b]      = sum_j min(p_j, q'_j)                                  (Def. 2.1)
 *   resid_mass[b] = sum_j max(0, p_j - q'_j)                              (denominator of Alg. 4 step 8)
 *   draft_ids[b]  = smallest j with prefix_j(q') > u0 * sum(q')           (step 2; only if sample_draft)
 *   accept[b]     = 1 iff u1 * q'_d < p_d, d = draft_ids[b]               (step 6; d outside [0,N) -> 0)
 *   resid_ids[b]  = smallest j with prefix_j(max(0, p - q')) > u2 * resid_mass, or -1 if resid_mass = 0
 * and per sequence s of gamma consecutive positions (steps 4-10), when gamma > 0:
 *   n_accepted[s] = length of the accepted prefix,
 *   out_tokens[s, 0..gamma] = accepted drafts, then the residual token of the first rejected position,
 *                             then -1 (no bonus token is drawn here: that needs one more target row).
 * q_prime == NULL draws only the bonus token t ~ p (step 8, else-branch) into resid_ids with u3;
 * then alpha = 0, accept = 0, resid_mass = sum(p), draft_ids is untouched, gamma must be 0.
 * p: PROB_F32 rows are used as given; LOGIT kinds go through the softmax.  Any of alpha,
 * resid_mass, n_accepted, out_tokens may be NULL.  Sums run in fp32 per 1024-id block and in
 * fp64 across blocks; token ids can differ from an exact evaluation only where the threshold lies
 * within rounding (about 1e-6 of the total) of a prefix-sum step.
 */
rdk_status_t rdk_verify_sample(const rdk_verify_desc_t *desc, const void *p, rdk_input_kind_t p_kind,
                               int64_t ldp, const float *q_prime, int64_t ldq, int32_t *draft_ids,
                               uint8_t *accept, float *alpha, float *resid_mass, int32_t *resid_ids,
                               int32_t *n_accepted, int32_t *out_tokens, void *workspace,
                               size_t workspace_bytes, void *stream);

/*
 * rdk_verify_sample for callers that can neither allocate device memory nor hand in a workspace (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): same arguments without the workspace, same
 * kernels, same outputs bit for bit.  The scratch (the per-block sums, and the softmax statistics of logit rows) lives
 * in a device array inside the library, 4 MiB per GPU, held until the process ends; the call allocates and frees
 * nothing.  A batch whose scratch need (rdk_verify_workspace_bytes with gamma = 0 minus its 256 bytes of slack, about
 * 12 * B * ceil(N / 1024) bytes) exceeds 4 MiB is refused with RDK_ERR_WORKSPACE and nothing is launched.  All calls
 * on one GPU share the one array: calls that overlap on one GPU (different streams, or different threads) race and
 * must be ordered by the caller; nothing in it needs clearing between calls.  Runs on the current device.
 */
rdk_status_t rdk_verify_sample_static(const rdk_verify_desc_t *desc, const void *p, rdk_input_kind_t p_kind,
                                      int64_t ldp, const float *q_prime, int64_t ldq, int32_t *draft_ids,
                                      uint8_t *accept, float *alpha, float *resid_mass, int32_t *resid_ids,
                                      int32_t *n_accepted, int32_t *out_tokens, void *stream);

/*
 * Alg. 1 steps 1-2 and Alg. 4 steps 2, 4-10 in one call: the outputs of rdk_redistribute_linear(mode)
 * followed by rdk_verify_sample on its result, without the round trip of q' through HBM.  The
 * redistributed rows are produced tile by tile, summed against p on the spot, and re-computed for the
 * two blocks in which the sampled ids fall.  q_prime may be NULL (then it is never written); otherwise
 * it receives the same rows rdk_redistribute_linear writes.  Block sums run over 64 ids (sparse) or
 * 1024 ids (Eq. 3), so fp32 rounding, and with it an id that sits on a prefix-sum step, can differ
 * from the two-call path within the tolerance stated at rdk_verify_sample.  desc->N must equal the
 * kernel's N; draft_ids is required (in/out as in rdk_verify_sample).  RDK_LINEAR_SPARSE needs a
 * RDK_SPARSE_TOPK kernel (k = 0 included: token-level intersection).
 */
rdk_status_t rdk_redistribute_verify_workspace_bytes(const rdk_kernel_t *kernel, rdk_linear_mode_t mode,
                                                     const rdk_verify_desc_t *desc, size_t *bytes);
rdk_status_t rdk_redistribute_verify(const rdk_kernel_t *kernel, rdk_linear_mode_t mode,
                                     const rdk_verify_desc_t *desc, const void *p, rdk_input_kind_t p_kind,
                                     int64_t ldp, const void *q, rdk_input_kind_t q_kind, int64_t ldq,
                                     float *q_prime, int64_t ldo, int32_t *draft_ids, uint8_t *accept,
                                     float *alpha, float *resid_mass, int32_t *resid_ids, int32_t *n_accepted,
                                     int32_t *out_tokens, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Alg. 4 step 2 on the drafter's side, before any target row exists: the draft token of every position is drawn
 * from the redistributed row q' = M^T TLI(q), out-of-vocabulary ids included (the use Sec. 1 and Sec. 3 name:
 * sampling tokens the drafter's vocabulary does not hold):
 *   draft_ids[b] = smallest j with prefix_j(q'_b) > u0 * sum_j q'_b(j),  u0 = word 0 of Philox(seed, offset + b)
 * -- the draw rdk_verify_sample and rdk_redistribute_verify make when sample_draft = 1, so verifying later with
 * sample_draft = 0 and these ids gives what the fused call gives.  q_draft (optional, [B]) receives q'_b(draft_ids[b]).
 *   RDK_SPARSE_TOPK kernel: q' is summed per 64-id block as it is produced and only the block of the
 *     crossing is re-computed; q_prime (optional, [B, ldo]) receives the rows if given.
 *   any other kernel (identity, dense fp32 / bf16): the rows are produced by the matching redistribution
 *     into q_prime, which is then required, and drawn from there.
 * draft_ids[b] = -1 (and q_draft[b] = 0) for a row without mass.  Workspace: rdk_sample_draft_workspace_bytes.
 * Errors as rdk_redistribute_linear.
 */
rdk_status_t rdk_sample_draft_workspace_bytes(const rdk_kernel_t *kernel, int32_t B, size_t *bytes);
rdk_status_t rdk_sample_draft(const rdk_kernel_t *kernel, const void *q, rdk_input_kind_t q_kind, int64_t ldq, int32_t B,
                              uint64_t seed, uint64_t offset, int32_t *draft_ids, float *q_draft, float *q_prime,
                              int64_t ldo, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Verification of several candidates per position.  The paper's introduction (Sec. 1) names multi-candidate / tree
 * verification among the related work; the steps are those of the method cited there (multi-step speculative
 * sampling) with the redistributed drafter q' in the drafter's place, per position b:
 *   r <- p_b;  for i = 0 .. C-1:  candidate x_i;  keep x_i when  u * q'_b(x_i) < r(x_i)  and stop;
 *              otherwise  r <- max(0, r - q'_b) / sum_j max(0, r(j) - q'_b(j));
 *   no candidate kept:  t drawn from r by the inverse CDF (smallest j whose prefix exceeds u * total).
 * With C = 1 this is rdk_verify_sample for one position (same draft, same decision, same residual token).  The
 * emitted token follows p_b exactly whatever q'_b is.
 *   sample_candidates = 1: the C candidates are drawn from q'_b by the inverse CDF and written to cand_ids;
 *   sample_candidates = 0: cand_ids [B, C] is input; an id >= N is a candidate that is never kept, a negative id
 *     ends the list of the position (fewer than C candidates; none at all: the token is drawn from p_b).
 * Uniforms: the m-th uniform of position b is word m % 4 of Philox4x32-10 with key = seed and counter
 * (offset + b as two words, m / 4, 0);  m = i for the draw of candidate i, C + i for its test, 2C for the final draw.
 * Outputs (device): accepted [B] = index of the kept candidate, or C; token [B] = the emitted id (-1 when the last
 * residual is empty); resid_mass [B, C] (optional) = sum_j max(0, r(j) - q'_b(j)) after each rejection, 0 for rounds
 * that were not reached.  p [B, ldp] of kind p_kind, q_prime [B, ldq] fp32; 1 <= C <= 16, N <= 2 097 152.
 * A call with less workspace than it asks for, but enough for the softmax partials of logit rows, takes a form that is slower for few
 * long rows, with the same results.
 * Errors: RDK_ERR_NULL, RDK_ERR_SHAPE (B, N, C, strides), RDK_ERR_DTYPE, RDK_ERR_ALIGN (p, q_prime or the workspace not 16-byte
 * aligned; the rows may lie at any stride),
 * RDK_ERR_UNSUPPORTED (N or C above the limits), RDK_ERR_WORKSPACE, RDK_ERR_HIP.
 */
typedef struct {
    int32_t B, N, C;            /* positions, target ids, candidates per position */
    uint64_t seed, offset;      /* Philox key and counter base */
    int sample_candidates;      /* 1: draw the candidates from q_prime; 0: cand_ids is input */
} rdk_multi_desc_t;
rdk_status_t rdk_verify_multi_workspace_bytes(const rdk_multi_desc_t *desc, rdk_input_kind_t p_kind, size_t *bytes);
rdk_status_t rdk_verify_multi(const rdk_multi_desc_t *desc, const void *p, rdk_input_kind_t p_kind, int64_t ldp,
                              const float *q_prime, int64_t ldq, int32_t *cand_ids, int32_t *accepted, int32_t *token,
                              float *resid_mass, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Verification of token trees (the other variant Sec. 1 names among the related work), in two calls: rdk_verify_multi
 * on every node with the tokens of its children as the node's candidates (position s * nodes + v = node v of tree s,
 * node 0 the root; p and q' of a node are the target and the redistributed drafter distribution after the prefix that
 * ends at the node), then this walk: from the root, emit token[.] of the node; if its verification kept candidate i
 * (accepted[.] = i < C) go on to child_node[., i], else stop -- the token was the residual draw, or the draw from p at
 * a leaf.  A chain of nodes is Alg. 4 steps 4-10 on one sequence.
 *   child_node [S, nodes, C] (device): node index of the child behind candidate slot i (> the node's own index).
 *   accepted, token [S * nodes] (device): outputs of rdk_verify_multi.
 *   n_accepted [S]: candidates kept along the path; out_tokens [S, nodes]: the emitted ids, -1 beyond them.
 * Integer work only (bit-exact).  Errors: RDK_ERR_NULL, RDK_ERR_SHAPE, RDK_ERR_HIP.
 */
rdk_status_t rdk_tree_walk(int32_t S, int32_t nodes, int32_t C, const int32_t *child_node, const int32_t *accepted,
                           const int32_t *token, int32_t *n_accepted, int32_t *out_tokens, void *stream);

/*
 * The k largest entries of every row and the logarithm of its normaliser: what is kept of a teacher's rows (rdk_distill_*), or of
 * redistributed rows.  Per row b of x [B, ldx] over N ids:
 *   ids[b, :]    = the ids of the k largest unmasked entries, descending, equal entries by ascending id; a logit of -inf and a weight of 0
 *                  are masked; -1 where fewer than k are left.  A NaN counts as larger than any number.
 *   values[b, :] = the entries themselves (logits are not divided by the temperature), widened to fp32; -inf (logits) or 0 (weights) beside -1.
 *   lse[b]       = log sum_j exp(x_bj / temperature) for logits, log sum_j x_bj for weights (temperature 1); -inf for a row that is
 *                  masked altogether; NaN for a row with a NaN or a logit of +inf.  May be NULL.
 * ids and values are [B, k] without gaps.  1 <= k <= min(N, 128), B < 2^24, temperature a positive normal number.  The ids and values are exact, whatever the
 * input; sums run in fp32.  Rows that crowd out the fast way (thousands of entries that tie with the k-th) take a slower one.
 * Errors: RDK_ERR_NULL, RDK_ERR_SHAPE (B, N, k, ldx, temperature), RDK_ERR_DTYPE, RDK_ERR_ALIGN (x or the workspace),
 * RDK_ERR_UNSUPPORTED (k above 128, N above 2^30, B from 2^24 on; weights with a temperature other than 1), RDK_ERR_WORKSPACE, RDK_ERR_HIP.
 */
typedef struct {
    int32_t B, N, k;            /* rows, ids, entries kept per row */
    float temperature;          /* of lse */
} rdk_topk_desc_t;
rdk_status_t rdk_topk_workspace_bytes(const rdk_topk_desc_t *desc, rdk_input_kind_t x_kind, size_t *bytes);
rdk_status_t rdk_topk(const rdk_topk_desc_t *desc, const void *x, rdk_input_kind_t x_kind, int64_t ldx, int32_t *ids, float *values,
                      float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Distillation of a drafter from its teacher's top logits.  Per position b the drafter has logits z [B, ldz] over its n kept slots (fp32
 * or bf16) and the teacher K entries: top_ids [B, K] target ids and top_logits [B, K] fp32 (rdk_topk writes both).  `kernel` (any
 * format) says which slot a target id has; with NULL the ids are slots themselves.  An entry counts if its id lies in the drafter's vocabulary
 * and its logit is above -inf; others (id -1, pruned ids) are passed over.  The ids of a row that count are distinct.  With T = temperature,
 * s = softmax(z_b / T), A = the slots of the entries that count and w = weight[b] (NULL: 1):
 *   teacher_lse == NULL: the teacher is renormalised over A (Eq. 1 of the paper on its own rows),  t_k = exp(v_k / T) / sum_A exp(v / T):
 *     loss[b] = w sum_A t (log t - log s),   dz[b, j] = w / T (s_j - t_j);      both 0 if A is empty.
 *   teacher_lse [B] = log sum exp(v / T) over the teacher's whole row (rdk_topk's lse at this temperature):  t_k = exp(v_k / T - lse), and what
 *     remains, r = max(0, 1 - sum_A t), is held against the drafter's remainder rho = sum_{j not in A} s_j:
 *     loss[b] = w (sum_A t (log t - log s) + r (log r - log rho)),
 *     dz[b, j] = w / T (s_j - t_j) on A,  w / T s_j (1 - r / rho) elsewhere;    without a slot outside A as if teacher_lse were NULL.
 * A row of weight 0 has loss 0 and gradient 0 whatever its logits hold (they are not read).  Masked logits (-inf) have s = 0: the loss is +inf
 * where the teacher has mass on them, and only there (finite logits, however far apart, give what the formulas give).  A drafter row that is masked
 * altogether has s = 0 everywhere.  NaN in a row that counts shows in its loss.
 *   rdk_distill_loss       forward: loss [B] and stats [B, 4] fp32, which the backward call reads (contents not part of the interface).
 *   rdk_distill_grad       backward: dz [B, ldd] of z's type from stats; weight is what comes from above (d / d loss[b], times whatever
 *                          weight the forward call had: a row whose weight was 0 there has 0 here).  Same z, top_ids, top_logits and temperature as in the forward call.  No workspace.
 *   rdk_distill_loss_grad  both at once, for weights known beforehand; z is read once where a row fits the registers.  stats may be NULL.
 * dz may be z itself (same stride), else they must not overlap.  Sums and statistics are held in fp32; a bf16 gradient is rounded once.
 * 1 <= K <= 128, B < 2^22, temperature a positive normal number; top_ids and top_logits without gaps.
 * Errors: RDK_ERR_NULL, RDK_ERR_SHAPE (B, n, K, strides, temperature, n other than the kernel's), RDK_ERR_DTYPE, RDK_ERR_ALIGN (z, dz, workspace),
 * RDK_ERR_UNSUPPORTED (K above 128, B from 2^22 on; rows of probabilities), RDK_ERR_WORKSPACE, RDK_ERR_HIP.
 */
typedef struct {
    int32_t B, n, K;            /* positions, drafter slots, teacher entries per position */
    float temperature;
} rdk_distill_desc_t;
rdk_status_t rdk_distill_workspace_bytes(const rdk_distill_desc_t *desc, rdk_input_kind_t z_kind, size_t *bytes);
rdk_status_t rdk_distill_loss(const rdk_distill_desc_t *desc, const rdk_kernel_t *kernel, const void *z, rdk_input_kind_t z_kind, int64_t ldz,
                              const int32_t *top_ids, const float *top_logits, const float *teacher_lse, const float *weight, float *loss,
                              float *stats, void *workspace, size_t workspace_bytes, void *stream);
rdk_status_t rdk_distill_grad(const rdk_distill_desc_t *desc, const rdk_kernel_t *kernel, const void *z, rdk_input_kind_t z_kind, int64_t ldz,
                              const int32_t *top_ids, const float *top_logits, const float *stats, const float *weight, void *dz, int64_t ldd,
                              void *stream);
rdk_status_t rdk_distill_loss_grad(const rdk_distill_desc_t *desc, const rdk_kernel_t *kernel, const void *z, rdk_input_kind_t z_kind,
                                   int64_t ldz, const int32_t *top_ids, const float *top_logits, const float *teacher_lse, const float *weight,
                                   float *loss, float *stats, void *dz, int64_t ldd, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Beam search's selection over beams and vocabulary.  G requests of W beams; x [G W, ldx] the next-token rows of the beams (logits, or weights
 * such as redistributed rows), scores [G, W] their scores (summed log-probabilities).  Candidates of a request:
 *   a live beam w: every unmasked id j, with  scores[w] + log softmax(x_w)_j  (weights: log(x_wj / sum x_w)), formed in fp32 as
 *     scores[w] + ((x_wj - max x_w) - log sum exp(x_w - max x_w));
 *   a beam with finished[w] != 0: the id eos alone, with scores[w];   a beam of score -inf: none.  Rows of such beams are not read.
 * The K best by descending score, equal scores by ascending beam, then id (of a beam only its K largest entries are candidates, equal entries by
 * ascending id): scores_out, parent (beam 0 .. W-1), token, finished_out (the beam was finished, or token == eos), all [G, K]; score -inf,
 * parent -1, token -1, finished 0 where there are fewer.  NaN and +inf in a live row make its scores NaN, which rank first.
 * finished and finished_out may be NULL; eos = -1: no id ends a beam (finished must be NULL then).  Outputs must not overlap the inputs.
 * 1 <= W <= 64, 1 <= K <= 128, N <= 2^30, W N < 2^31, G W < 2^24.
 * Errors: RDK_ERR_NULL, RDK_ERR_SHAPE (G, W, N, K, ldx, eos, an output that overlaps its input), RDK_ERR_DTYPE, RDK_ERR_ALIGN (x, workspace),
 * RDK_ERR_UNSUPPORTED (limits), RDK_ERR_WORKSPACE, RDK_ERR_HIP.
 */
typedef struct {
    int32_t G, W, N, K;         /* requests, beams per request, ids, candidates kept per request */
    int32_t eos;                /* id that ends a beam, or -1 */
} rdk_beam_desc_t;
rdk_status_t rdk_beam_select_workspace_bytes(const rdk_beam_desc_t *desc, rdk_input_kind_t x_kind, size_t *bytes);
rdk_status_t rdk_beam_select(const rdk_beam_desc_t *desc, const void *x, rdk_input_kind_t x_kind, int64_t ldx, const float *scores,
                             const uint8_t *finished, float *scores_out, int32_t *parent, int32_t *token, uint8_t *finished_out,
                             void *workspace, size_t workspace_bytes, void *stream);

/*
 * The states of the beams after a selection: row i of request g in dst becomes row parent[g, i] of request g in src, for `count` states at once
 * (`states` is a HOST array of device buffers: key-value caches, token histories, recurrent states).  parent [G, K] (device) holds beams
 * 0 .. W-1; a row whose parent is -1 (or not a beam) is left as it is.  src has G W rows, dst G K rows.  A row is `segments` pieces of segment_bytes, *_pitch
 * bytes apart (the filled part of a cache with room for more), rows are *_stride bytes apart; any alignment (fastest where everything is a
 * multiple of 16).  dst == src with the same strides reorders in place (K must be W), rows that keep their beam are then not touched; otherwise
 * src and dst must not overlap.  Segments of a state must not overlap one another, nor states.  Copies are exact.
 * 1 <= W, K <= 64; no workspace.
 * Errors: RDK_ERR_NULL, RDK_ERR_SHAPE (sizes, strides, overlap, K other than W in place), RDK_ERR_UNSUPPORTED (W or K above 64), RDK_ERR_HIP.
 */
typedef struct {
    const void *src;            /* device */
    void *dst;                  /* device */
    int64_t src_stride, dst_stride;   /* bytes from one beam's row to the next */
    int64_t segments, segment_bytes;  /* pieces of a row, and their size */
    int64_t src_pitch, dst_pitch;     /* bytes from one piece to the next (ignored for one piece) */
} rdk_state_t;
rdk_status_t rdk_beam_reorder(int32_t G, int32_t W, int32_t K, const int32_t *parent, const rdk_state_t *states, int32_t count, void *stream);

/*
 * Log probabilities of given tokens, with the row's entropy and its top alternatives, and the gradient of these: scoring a text, what a server returns
 * beside its tokens, candidates held against redistributed rows, training on tokens.  Per row b of x [B, ldx] (logits, or weights such as redistributed
 * rows) with y_j = x_j / temperature (weights: log x_j, temperature 1) and s = softmax(y):
 *   logprob[b, c] = log s at tokens[b, c];  0 for a negative token (padding: nothing was asked); -inf for one that the row masks (a logit of -inf, a weight
 *                   of 0) or does not hold (an id from N on; with `kernel` a pruned id).
 *   rank[b, c]    = how many entries come before it in the order of rdk_topk (larger, or equal at a lower place); -1 beside a log probability of -inf
 *                   or NaN and for a negative token.  May be NULL.
 *   entropy[b]    = - sum_j s_j log s_j;  0 for a row that is masked altogether.  May be NULL.
 *   top_ids, top_logprobs [B, k] = rdk_topk's entries with their log probabilities (-1, -inf where fewer are unmasked); not touched with k = 0.
 *   stats [B, 4] fp32 = what the backward call reads (contents not part of the interface).  May be NULL.
 * `kernel` (any format): the rows are over its n kept slots (N = n) and tokens, top_ids are target ids; NULL: ids are places in the row.
 * A row with a NaN or a logit of +inf has log probabilities and an entropy of NaN (masked tokens -inf).  A row that is sure of an entry keeps the entropy and the
 * log probability of that entry to their own last bits.  Tokens may repeat.  1 <= C <= 16, 0 <= k <= min(N, 128), N <= 2^30, B < 2^24.
 *   rdk_logprobs_grad  dx [B, ldd] of x's type:  sum_c d_logprob[b, c] d logprob[b, c] / dx + d_entropy[b] d entropy[b] / dx
 *       = 1 / T (sum_{c: token c at j} g_c - s_j (G + h (log s_j + entropy))),  g = d_logprob, h = d_entropy, G = sum of g over the tokens that the row holds;
 *     tokens it does not hold add nothing, d_logprob or d_entropy may be NULL (0).  A row whose g (of tokens it holds) and h are all 0 has gradient 0 whatever its
 *     logits hold (they are not read), and so has a row that is masked altogether.  No workspace.
 *   rdk_logprobs_step  forward and backward at once, for d_logprob and d_entropy known beforehand; x is read once where a row fits the registers.
 *     No ranks and no alternatives (k = 0).
 * Gradients are of rows of logits only, at temperatures from 2^-40 on, B < 2^22 and B ceil(N / 16384) < 2^24 (fp32: N / 8192).  dx may be x itself (same
 * stride), else they must not overlap.  Sums are held in fp32, a bf16 gradient is rounded once.
 * Errors: RDK_ERR_NULL, RDK_ERR_SHAPE (B, N, C, k, strides, temperature, N other than the kernel's n, an overlap), RDK_ERR_DTYPE, RDK_ERR_ALIGN (x, dx, stats,
 * workspace), RDK_ERR_UNSUPPORTED (limits; weights with a temperature other than 1; gradients of weights or at lower temperatures; rdk_logprobs_step with k > 0), RDK_ERR_WORKSPACE, RDK_ERR_HIP.
 */
typedef struct {
    int32_t B, N, C, k;         /* rows, entries of a row, given tokens per row, alternatives per row */
    float temperature;
} rdk_logprobs_desc_t;
rdk_status_t rdk_logprobs_workspace_bytes(const rdk_logprobs_desc_t *desc, rdk_input_kind_t x_kind, size_t *bytes);
rdk_status_t rdk_logprobs(const rdk_logprobs_desc_t *desc, const rdk_kernel_t *kernel, const void *x, rdk_input_kind_t x_kind, int64_t ldx,
                          const int32_t *tokens, float *logprob, int32_t *rank, float *entropy, int32_t *top_ids, float *top_logprobs, float *stats,
                          void *workspace, size_t workspace_bytes, void *stream);
rdk_status_t rdk_logprobs_grad(const rdk_logprobs_desc_t *desc, const rdk_kernel_t *kernel, const void *x, rdk_input_kind_t x_kind, int64_t ldx,
                               const int32_t *tokens, const float *stats, const float *d_logprob, const float *d_entropy, void *dx, int64_t ldd,
                               void *stream);
rdk_status_t rdk_logprobs_step(const rdk_logprobs_desc_t *desc, const rdk_kernel_t *kernel, const void *x, rdk_input_kind_t x_kind, int64_t ldx,
                               const int32_t *tokens, const float *d_logprob, const float *d_entropy, float *logprob, float *entropy, float *stats,
                               void *dx, int64_t ldd, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Rows of an embedding table for a batch of tokens, and the table's gradient.  table [V, ldt], out [B, ldo], each fp32 or bf16:
 *   rdk_embed       out[b, :] = scale * table[ids[b], :], rounded once; zeros for an id that the table does not hold (negative, from V on).
 *   rdk_embed_grad  d_table[v, :] = scale * sum_{b: ids[b] = v} d_out[b, :]  (accumulate != 0: added to what d_table holds, and rows that no token names
 *     are left as they are; accumulate = 0: these are set to 0), summed in fp32 and rounded once, in an order that depends on ids, B, V, d and types alone:
 *     the same call gives the same bits.
 * `kernel` (any format): the table has a row for each of its n kept slots (V = n) and ids are target ids, pruned ones are not held; NULL: ids are rows.
 * Data of a row d elements wide; rows may lie at any stride.  Inputs and outputs must not overlap.  1 <= B < 2^24, 1 <= V <= 2^29, 1 <= d <= 2^20, scale finite.
 * Errors: RDK_ERR_NULL, RDK_ERR_SHAPE (B, V, d, strides, scale, V other than the kernel's n, an overlap), RDK_ERR_DTYPE, RDK_ERR_ALIGN (table, out,
 * d_table, d_out, workspace), RDK_ERR_UNSUPPORTED (limits), RDK_ERR_WORKSPACE, RDK_ERR_HIP.
 */
typedef enum {
    RDK_F32 = 1,
    RDK_BF16 = 2
} rdk_float_t;
typedef struct {
    int32_t B, V, d;            /* tokens, rows of the table, width */
    float scale;
} rdk_embed_desc_t;
rdk_status_t rdk_embed(const rdk_embed_desc_t *desc, const rdk_kernel_t *kernel, const int32_t *ids, const void *table, rdk_float_t table_type,
                       int64_t ldt, void *out, rdk_float_t out_type, int64_t ldo, void *stream);
rdk_status_t rdk_embed_grad_workspace_bytes(const rdk_embed_desc_t *desc, size_t *bytes);
rdk_status_t rdk_embed_grad(const rdk_embed_desc_t *desc, const rdk_kernel_t *kernel, const int32_t *ids, const void *d_out, rdk_float_t out_type,
                            int64_t ldo, void *d_table, rdk_float_t table_type, int64_t ldt, int32_t accumulate, void *workspace,
                            size_t workspace_bytes, void *stream);

/* The four Philox words of `count` consecutive positions, [count, 4] uint32 on the device (for
 * checking the random stream against an independent implementation). */
rdk_status_t rdk_philox_words(uint64_t seed, uint64_t offset, int32_t count, uint32_t *words,
                              void *stream);

/*
 * Kernel timing for benchmarks.  After rdk_timing_select(name) every launch of the library kernel
 * of that name ("*" = every kernel of the redistribute / verify calls, NULL or "" = none) is
 * bracketed by two HIP events on the launch stream; "name/8" brackets every eighth launch only
 * (an event pair costs the host and the stream several microseconds, which a short step would
 * otherwise show).  rdk_timing_read(name, ...) waits for the
 * recorded events of that kernel, returns how many launches were recorded and their summed
 * elapsed time in milliseconds, and forgets them.  Both take HOST strings.  Names:
 * row_stats_kernel, row_block_sums_kernel, verify_stream_kernel, verify_finalize_kernel, draft_finalize_kernel,
 * sequence_scan_kernel, taylor_stats_kernel, taylor_write_kernel, taylor_row_kernel, taylor_whole_kernel, tli_scatter_kernel,
 * tree_walk_kernel, verify_multi_kernel, verify_multi_round_kernel,
 * q_transpose_kernel, sparse_product_kernel, prep_a_split_kernel, exact_f32_split_kernel,
 * exact_reduce_kernel, prep_a_bf16_kernel, exact_bf16_kernel, topk_part_kernel, topk_merge_kernel, beam_merge_kernel, beam_reorder_kernel,
 * distill_row_kernel, distill_loop_kernel, distill_part_kernel, distill_finish_kernel, distill_grad_kernel,
 * logprob_part_kernel, logprob_finish_kernel, logprob_grad_kernel, logprob_row_kernel,
 * embed_kernel, embed_grad_few_kernel, embed_sort_kernel, embed_count_kernel, embed_scan_kernel, embed_place_kernel, embed_grad_sum_kernel,
 * embed_grad_join_kernel.
 */
rdk_status_t rdk_timing_select(const char *kernel_name);
rdk_status_t rdk_timing_read(const char *kernel_name, int64_t *launches, double *total_ms);

const char *rdk_status_string(rdk_status_t status);

/* Text of the last HIP error seen by the calling thread ("" if none). */
const char *rdk_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* RDK_H */
