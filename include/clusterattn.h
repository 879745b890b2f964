/*
 * clusterattn.h - C ABI of the ClusterAttention hot path on MI355X (gfx950).
 *
 * ClusterAttention replaces bidirectional softmax attention, per head, by four
 * steps (paper: Method, Overview; Preliminaries, motivation for sparse
 * attention):
 *   1. ca_cluster            split queries and keys into clusters of a fixed
 *                            power-of-two size (Method: Clustering), and form
 *                            the permuted Q/K/V and the cluster centroids;
 *   2. ca_select             score every query cluster against every key
 *                            cluster by centroid dot products and keep the top-k
 *                            key clusters (Method: Cluster assignment);
 *   3. ca_block_sparse_attn  softmax attention of each query cluster onto the
 *                            keys of its selected clusters, returning the output
 *                            and the softmax denominator (Method: Overview);
 *   4. ca_compensate         striped mean-compensation: every skipped key
 *                            cluster enters through its centroid key and value
 *                            weighted by its size, merged with step 3, and the
 *                            rows restored to the original token order
 *                            (Preliminaries: error in sparse attention; App. A).
 * ca_attn_compensated computes steps 3 and 4 in one pass (bf16): the same
 * result without the intermediate op/lse arrays.
 *
 * Conventions shared by every call
 * --------------------------------
 * - All data pointers are DEVICE pointers (hipMalloc'd or equivalent) on the
 *   current HIP device. The caller owns every buffer; the library never
 *   allocates, frees or synchronises. Work is enqueued on `stream` (a
 *   hipStream_t; NULL = the default stream) and buffers must stay alive until
 *   the stream has passed it.
 * - Q/K/V and the final output use the problem's layout (ca_layout) with the
 *   last dimension contiguous. Every other array is dense, row-major, with the
 *   shape given in its comment; BH = batch * heads, heads vary fastest.
 * - Derived sizes: nqc = ceil(nq/cq), nkc = ceil(nk/ck), nq_pad = nqc*cq,
 *   nk_pad = nkc*ck. Clusters hold exactly cq (ck) tokens except the last one,
 *   which holds the remainder; its missing rows are zero-filled padding that
 *   never influences a result.
 * - Every call validates its arguments before touching the GPU. On any status
 *   other than CA_OK nothing has been enqueued. CA_E_DEVICE means a HIP launch
 *   error after validation; ca_last_error() then gives the HIP error text.
 *   No C++ exception crosses this interface.
 * - Every output element is written (including padding rows). Outputs must not
 *   alias inputs. Results are deterministic: two identical calls give
 *   bit-identical outputs.
 * - Non-finite inputs (NaN/Inf) are not checked by the steps: the calls stay
 *   memory-safe but the results are unspecified. Checked mode is the separate
 *   call ca_check_finite, which flags them on the device.
 * - Calls on different streams may run concurrently if their outputs and
 *   workspaces do not overlap.
 */
#ifndef CLUSTERATTN_H_
#define CLUSTERATTN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define CA_ABI_VERSION 8

#if defined(__GNUC__) || defined(__clang__)
#define CA_API __attribute__((visibility("default")))
#else
#define CA_API
#endif

typedef enum {
  CA_OK = 0,
  CA_E_INVALID = 1,     /* bad argument: null pointer, size out of range, c not a power of two, k not in [1, nkc] */
  CA_E_UNSUPPORTED = 2, /* valid but not built: e.g. bf16 attention with d not in {64, 128} */
  CA_E_WORKSPACE = 3,   /* workspace smaller than ca_workspace_size() */
  CA_E_DEVICE = 4,      /* HIP reported an error while enqueueing */
  CA_E_NONFINITE = 5    /* checked mode: an input holds NaN or Inf (reported by the caller's
                           read of ca_check_finite's flags; no call returns it itself, since
                           the library never synchronises) */
} ca_status;

typedef enum { CA_F32 = 0, CA_BF16 = 1 } ca_dtype;

/* Space in which the recursive split is done (Method: Transforms).
 *   CA_XF_NONE:   the raw coordinates.
 *   CA_XF_PCA:    principal coordinates of the raw vectors (diagonalized
 *                 splitting without the attention-aware metrics).
 *   CA_XF_METRIC: keys in the query-induced metric Q^T Q / n, queries through
 *                 r(q) = q S_k / |q S_k| with S_k S_k^T = the key covariance
 *                 (top-k representation, App. B.2), each side then on its own
 *                 principal coordinates. This is the evaluated method.
 *   CA_XF_ADAPTIVE: keys as CA_XF_METRIC; queries through the unnormalised
 *                 r(q) = q S_k (the metric K_c^T K_c / n of the centred keys,
 *                 Method: query clustering for adaptive assignment; App. B.1),
 *                 on its principal coordinates. For use with the adaptive
 *                 (attention-mass) selection of ca_select_hist.
 *   CA_XF_RANDOM: the random-cluster control (Experiments: baselines, random
 *                 clusters routed by centroid scores): tokens are split on
 *                 pseudo-random coordinates y[i][j] = (splitmix64 output
 *                 number c, top 24 bits) / 2^24 with c = (((2 bh + side) <<
 *                 22 | i) << 7) | j (bh = b * heads + h, side 0 queries / 1
 *                 keys; splitmix64 as published by S. Vigna, started at state
 *                 0), which partitions them into clusters at random. */
typedef enum {
  CA_XF_NONE = 0,
  CA_XF_PCA = 1,
  CA_XF_METRIC = 2,
  CA_XF_ADAPTIVE = 3,
  CA_XF_RANDOM = 4
} ca_transform;

/* Recursive split algorithm (Method: Recursive splitting).
 *   CA_SPLIT_DIAG:  diagonalized splitting (the evaluated method): at each node
 *                   the global principal coordinate of highest variance on a
 *                   subsample (see ca_cluster).
 *   CA_SPLIT_BASIC: basic splitting, a variation of principal direction
 *                   divisive partitioning: at each node the first principal
 *                   direction of the subsample's centred covariance by 8
 *                   power iterations, warm-started from the mean of the
 *                   parent's direction and random normal noise rescaled to its
 *                   norm; every member is projected on it and the split is
 *                   made on the projections. Supported with CA_XF_NONE and
 *                   CA_XF_METRIC (the metric root space without principal
 *                   axes: keys k S_q, queries q S_k / |q S_k|, no
 *                   eigendecomposition). Arithmetic (fp32, fixed order, no
 *                   fused multiply-add): mean mu = (sum of the m subsample
 *                   rows in order) / m; rows centred; per iteration t_j =
 *                   sum_k (x_jk - mu_k) v_k, w_k = sum_j t_j (x_jk - mu_k),
 *                   v = w / sqrt(sum_k w_k^2) (a zero w keeps v); start v0 =
 *                   noise at the root, else (v_p + r sqrt(|v_p|^2) /
 *                   sqrt(|r|^2)) / 2; projections sum_k y_ik v_k. Noise of
 *                   the node at slot s of level l of head bh, side (0 queries,
 *                   1 keys), coordinate k: (sum over u < 12 of the top 24 bits
 *                   of splitmix64 output 16 c + u) / 2^24 - 6 (fp64, rounded
 *                   once to fp32), c = ((((2 bh + side) << 5 | l) << 20 | s)
 *                   << 7) | k. */
typedef enum { CA_SPLIT_DIAG = 0, CA_SPLIT_BASIC = 1 } ca_split;

/* Layout of Q, K, V and the final output: BHND = [B][H][N][d],
 * BNHD = [B][N][H][d] (the usual activation layout of a transformer), both
 * dense; STRIDED = any element strides given in the problem (for instance
 * views of a fused QKV projection, [B][N][3][H][d], with the output in a
 * tensor of its own). In every layout the last dimension is contiguous. */
typedef enum { CA_LAYOUT_BHND = 0, CA_LAYOUT_BNHD = 1, CA_LAYOUT_STRIDED = 2 } ca_layout;

typedef struct {
  int32_t batch, heads;  /* >= 1 */
  int32_t nq, nk;        /* real query / key tokens per head, >= 1 */
  int32_t d;             /* head dimension, 1..128 (attention: see below) */
  int32_t cq, ck;        /* cluster sizes, powers of two in [1, 256] */
  int32_t dtype;         /* ca_dtype of Q/K/V, permuted copies and output */
  int32_t transform;     /* ca_transform (ca_cluster only) */
  int32_t layout;        /* ca_layout of Q/K/V/out */
  int32_t split;         /* ca_split (ca_cluster only) */
  /* CA_LAYOUT_STRIDED only (ignored by the dense layouts): element strides
   * {batch, head, token} of q, k, v and the output; element (b, h, i, t) of
   * q sits at q + b q_stride[0] + h q_stride[1] + i q_stride[2] + t. Each
   * stride is >= 0 and a multiple of 16 bytes' worth of elements (8 for
   * bf16, 4 for fp32), and the tensors' base pointers are 16-byte aligned,
   * so that rows can be read and written in 16-byte pieces. The output's
   * rows must not overlap one another or any input (not checked). */
  int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3];
} ca_problem;

/* Outputs of ca_cluster. Required unless marked optional. */
typedef struct {
  int32_t* perm_q;   /* [BH][nq]  original query index at each cluster-ordered position */
  int32_t* perm_k;   /* [BH][nk]  same for keys */
  int32_t* cid_q;    /* [BH][nq]  cluster of original query i (optional, may be NULL) */
  int32_t* cid_k;    /* [BH][nk]  cluster of original key i (optional, may be NULL) */
  int32_t* count_q;  /* [BH][nqc] real members per query cluster */
  int32_t* count_k;  /* [BH][nkc] real members per key cluster */
  float* cent_q;     /* [BH][nqc][d] fp32 mean of the ORIGINAL query vectors of each cluster */
  float* cent_k;     /* [BH][nkc][d] same for keys */
  float* cent_v;     /* [BH][nkc][d] same for values (values follow the key clusters);
                        optional: NULL (with v == NULL) skips values */
  void* qp;          /* [BH][nq_pad][d] dtype: queries in cluster order, pad rows zero */
  void* kp;          /* [BH][nk_pad][d] dtype: keys in cluster order, pad rows zero */
  void* vp;          /* [BH][nkc][d][ck] dtype: value tiles. For every key cluster the ck value
                        rows in cluster order, stored transposed (dimension-major, ck
                        contiguous), pad columns zero. This is the operand layout of the
                        value product in the attention calls. Optional: NULL with v. */
  float* yq_dbg;     /* [BH][nq][d] optional: the query split coordinates (original order) */
  float* yk_dbg;     /* [BH][nk][d] optional: the key split coordinates (original order) */
} ca_cluster_out;

/* ABI version compiled into the library (CA_ABI_VERSION). */
CA_API int ca_abi_version(void);

/* Static text for a status code. */
CA_API const char* ca_status_str(int status);

/* Detail of the last non-OK status returned on the calling thread ("" if none). */
CA_API const char* ca_last_error(void);

/* Bytes of workspace ca_cluster, ca_select and ca_compensate need for this
 * problem with k kept key clusters (k is only used for validation; the size
 * does not depend on it). Host-only; enqueues nothing. Workspace must be
 * 256-byte aligned. */
CA_API int ca_workspace_size(const ca_problem* p, int32_t k, size_t* bytes);

/* Step 1: clustering (Method: Clustering, Recursive splitting - diagonalized
 * variant; Transforms).
 *
 * Per head, queries and keys are each mapped to their split space (transform)
 * and recursively split: at a node of s > c tokens, a subsample of
 * m = min(d, s) members at positions floor((2j+1)s/(2m)) of the node (in
 * ascending original-index order) picks the coordinate of highest fp64
 * population variance (two-pass, sequential, ties to the lower coordinate);
 * the node's c*floor(ceil(s/c)/2) members with the smallest (coordinate value,
 * original index) go left, the rest right, both keeping index order; leaves
 * are numbered left to right. This is deterministic: given the split
 * coordinates (exported through yq_dbg / yk_dbg) the permutation is exact.
 *
 * q, k: [B,H,nq|nk,d] in the problem layout and dtype. v: same shape as k, or
 * NULL to skip the value outputs. ws: device workspace of ws_bytes >=
 * ca_workspace_size(). */
CA_API int ca_cluster(const ca_problem* p, const void* q, const void* k, const void* v,
               const ca_cluster_out* out, void* ws, size_t ws_bytes, void* stream);

/* Step 2: assignment (Method: Cluster assignment - scoring and top-k
 * selection). scores[a][b] = cent_q[a] . cent_k[b] (fp32, the mean pairwise
 * logit up to the 1/sqrt(d) factor; for bf16 problems with d = 64 or 128 and
 * 16-byte aligned centroids they are formed on the matrix cores from a
 * three-term bf16 split of the fp32 centroids, about 2^-16 relative per
 * product); lists[a] = the k key clusters with the largest scores, ties to
 * the lower index, in ascending order.
 *
 * cent_q: [BH][nqc][d], cent_k: [BH][nkc][d] fp32. scores_in: optional
 * [BH][nqc][nkc] fp32 scores to rank instead of computing them (NULL:
 * compute). scores_out: optional [BH][nqc][nkc] export of the ranked scores.
 * lists: [BH][nqc][k] int32 output. 1 <= k <= nkc. */
CA_API int ca_select(const ca_problem* p, const float* cent_q, const float* cent_k,
              const float* scores_in, float* scores_out, int32_t k, int32_t* lists,
              void* ws, size_t ws_bytes, void* stream);

/* Step 2, histogram variant (Method: Cluster assignment - selection, the
 * two-pass histogram). For query cluster a, with S = the centroid scores of
 * its row: a 16384-step grid over [min S, max S] (coarse bins of 128 steps,
 * each refined into 128), g_b = min(16383, floor((S_b - min S) * (16384 /
 * (max S - min S)))) in fp32; the estimated attention mass of key cluster b,
 * count_k[b] * exp(scale * (S_b - max S)), in fixed point (2^-32 units, fp64
 * arithmetic, exact integer sums); need = ceil(mass_recall * total mass).
 * The coarse histogram finds the highest coarse bin whose lower edge keeps
 * at least min_count clusters and at least `need` mass; its 128 fine bins
 * find the highest such edge G inside it; every b with g_b >= G is selected.
 * If all scores are equal, or min_count >= nkc, every cluster is selected.
 *   top-k through the histogram: min_count = k, mass_recall = 0 (at least k
 *   clusters: the ties inside the edge's fine bin are kept);
 *   adaptive assignment: min_count = 16, mass_recall in (0, 1].
 *
 * cent_q, cent_k, scores_in, scores_out: as ca_select. count_k: [BH][nkc].
 * min_count >= 1; mass_recall in [0, 1]; scale <= 0 selects 1/sqrt(d).
 * lists: [BH][nqc][nkc] int32 output, lens[a] ascending cluster indices in
 * row a (the rest of the row is not written); lens: [BH][nqc] int32 output,
 * each in [1, nkc]. Pass lists with list stride k = nkc and lens to the
 * attention and compensation calls. ws: as ca_select. */
CA_API int ca_select_hist(const ca_problem* p, const float* cent_q, const float* cent_k,
                   const int32_t* count_k, const float* scores_in, float* scores_out,
                   int32_t min_count, float mass_recall, float scale, int32_t* lists,
                   int32_t* lens, void* ws, size_t ws_bytes, void* stream);

/* Step 3: block-sparse attention (Method: Overview - attention over the
 * selected clusters, returning the softmax denominator).
 *
 * For query row p of cluster a (permuted order), over the real keys j of the
 * clusters in lists[a]:  s_j = scale * qp[p] . kp[j],
 *   op[p]  = sum_j e^{s_j - m} vp[j] / sum_j e^{s_j - m},
 *   lse[p] = m + ln sum_j e^{s_j - m}   (natural log; m = max_j s_j).
 * Key rows past count_k[b] in a cluster are padding and are excluded.
 *
 * qp: [BH][nq_pad][d], kp: [BH][nk_pad][d], vp: [BH][nkc][d][ck] value tiles
 * as written by ca_cluster (all dtype), count_k: [BH][nkc], each in [1, ck],
 * lists: [BH][nqc][k] with entries in [0, nkc) (not checked on the device;
 * out-of-range entries are clamped), lens: optional [BH][nqc] list lengths
 * (NULL: every list has k entries; otherwise row a uses its first lens[a]
 * entries, clamped to [1, k] on the device), op: [BH][nq_pad][d] dtype, lse:
 * [BH][nq_pad] fp32. scale <= 0 selects 1/sqrt(d). Padding query rows get
 * defined values that callers ignore. bf16: d in {64, 128}, cq and ck in
 * {64, 128}; fp32: d % 4 == 0, any cq, ck.
 *
 * ws: optional device workspace of ws_bytes >= ca_workspace_size(). With
 * lens given (lists of different lengths) the bf16 path uses it to schedule
 * the query clusters: they are cut into eight contiguous ranges of about
 * equal work, one per XCD, and each range runs longest list first. With ws
 * NULL (ws_bytes 0) the query clusters run in index order. The results are
 * the same either way: only the order in which workgroups start changes. */
CA_API int ca_block_sparse_attn(const ca_problem* p, const void* qp, const void* kp, const void* vp,
                         const int32_t* count_k, const int32_t* lists, const int32_t* lens,
                         int32_t k, float scale, void* op, float* lse, void* ws,
                         size_t ws_bytes, void* stream);

/* Step 4: striped mean-compensation and un-permutation (Preliminaries: error
 * in sparse attention; App. A).
 *
 * For query row p of cluster a: every key cluster b NOT in lists[a] adds the
 * logit t_b = scale * qp[p] . cent_k[b] + ln count_k[b] with value cent_v[b];
 *   lse_c = ln sum_b e^{t_b},  o_c = sum_b e^{t_b - lse_c} cent_v[b],
 *   lse   = ln(e^{lse[p]} + e^{lse_c}),
 *   out   = e^{lse[p] - lse} op[p] + e^{lse_c - lse} o_c,
 * written to out[perm_q[p]] (original token order, problem layout). With
 * enable == 0, or when every cluster is selected, out = op[p], lse = lse[p].
 *
 * qp, op: [BH][nq_pad][d] dtype; cent_k, cent_v: [BH][nkc][d] fp32; count_k:
 * [BH][nkc]; lists: [BH][nqc][k], lens: optional list lengths as in
 * ca_block_sparse_attn; lse: [BH][nq_pad] fp32; perm_q: [BH][nq];
 * out: [B,H,nq,d] in the problem layout and dtype; lse_out: optional
 * [BH][nq] fp32 in original order. ws: device workspace of ws_bytes >=
 * ca_workspace_size(), where the bf16 path stages the centroids as bf16
 * tiles; required only for bf16 with enable != 0 and either k < nkc or lens
 * given (otherwise it may be NULL with ws_bytes 0). Compensation keeps a
 * selection bitmap of the key clusters per query cluster: with enable != 0
 * and either k < nkc or lens given, more than 65536 key clusters return
 * CA_E_UNSUPPORTED (enable == 0, or every cluster kept, has no such limit). */
CA_API int ca_compensate(const ca_problem* p, const void* qp, const float* cent_k, const float* cent_v,
                  const int32_t* count_k, const int32_t* lists, const int32_t* lens, int32_t k,
                  float scale,
                  int32_t enable, const void* op, const float* lse, const int32_t* perm_q,
                  void* out, float* lse_out, void* ws, size_t ws_bytes, void* stream);

/* Steps 3 and 4 in one pass (bf16 problems; Method: Overview; Preliminaries:
 * error in sparse attention; App. A).
 *
 * The result of ca_block_sparse_attn followed by ca_compensate on the same
 * arguments, up to rounding: each query cluster runs one online softmax over
 * the keys of its selected clusters and then over the centroid keys of the
 * unselected clusters, the logit of centroid b being
 * scale * qp[p] . cent_k[b] + ln count_k[b]. Combining the two parts inside
 * one softmax gives the merged output and lse directly (ln of the sum of both
 * parts' exponentials), so op and lse are never formed or rounded, and the
 * rows go straight to out[perm_q[p]].
 *
 * Arguments as in ca_block_sparse_attn (qp, kp, vp, count_k, lists, lens, k,
 * scale) and ca_compensate (cent_k, cent_v, enable, perm_q, out, lse_out).
 * ws: device workspace of ws_bytes >= ca_workspace_size(); required when
 * enable != 0 and either k < nkc or lens is given (the centroids are staged
 * there as bf16 tiles) and used for the launch schedule when lens is given;
 * otherwise it may be NULL with ws_bytes 0. Returns CA_E_UNSUPPORTED for fp32
 * problems and for more than 65536 key clusters. */
CA_API int ca_attn_compensated(const ca_problem* p, const void* qp, const void* kp, const void* vp,
                               const float* cent_k, const float* cent_v, const int32_t* count_k,
                               const int32_t* lists, const int32_t* lens, int32_t k, float scale,
                               int32_t enable, const int32_t* perm_q, void* out, float* lse_out,
                               void* ws, size_t ws_bytes, void* stream);

/* Checked mode (the method is defined for finite query, key and value
 * vectors; Method: Overview). Scans q, k and v (v may be NULL) in the
 * problem's layout and writes flags[0] on the stream: bit 0 if q holds a NaN
 * or an infinity, bit 1 for k, bit 2 for v; 0 when all are finite. flags: one
 * device int32, cleared by this call before the scan (no memset is
 * recorded); read it once the stream has passed the call, and treat a
 * non-zero value as CA_E_NONFINITE. Reads each input once (an HBM pass over
 * q, k and v). */
CA_API int ca_check_finite(const ca_problem* p, const void* q, const void* k, const void* v,
                           int32_t* flags, void* stream);

/* ca_attn_compensated without a workspace, for callers that cannot allocate
 * device memory: code under HIP graph capture, serving loops and harnesses
 * that forbid allocation. Same arguments and result as ca_attn_compensated
 * (bit for bit; the same kernels run), minus ws and ws_bytes.
 *
 * The centroid tiles (compensation with unselected clusters:
 * BH * ceil(nkc/128) * 128 * (4 d + 4) bytes, rounded up to 256) and the
 * launch schedule (lens given: (16 + 8 * floor((5 * BH * nqc + 31) / 32)) * 4
 * bytes) go to a scratch array that the library holds on every device it
 * runs on: 32 MiB (33554432 bytes), part of the library's code object, kept
 * until the process ends. Returns CA_E_WORKSPACE, with nothing enqueued,
 * when a problem needs more; ca_attn_compensated with a workspace has no
 * such limit. This call allocates nothing: no hipMalloc and no allocating
 * library routine (the array's device address is looked up once per device,
 * on the first call with that device current).
 *
 * All calls on one device share that device's array, which keeps the last
 * call's contents. Calls that overlap in time on one device (on different
 * streams, or from host threads without ordering between them) race and give
 * wrong results; calls ordered on one stream are safe. */
CA_API int ca_attn_compensated_noalloc(const ca_problem* p, const void* qp, const void* kp,
                                       const void* vp, const float* cent_k, const float* cent_v,
                                       const int32_t* count_k, const int32_t* lists,
                                       const int32_t* lens, int32_t k, float scale,
                                       int32_t enable, const int32_t* perm_q, void* out,
                                       float* lse_out, void* stream);

/* ---- Sequence operators ------------------------------------------------------
 *
 * What stands around the attention layer of a video, sequence or table model:
 * rotary positions of several axes, attention with a sliding window and sinks
 * with its gradients, and a paged key-value cache with the attention of one
 * new token over it. The conventions above hold (device pointers, the
 * caller's buffers, validation before anything is enqueued, deterministic
 * results), with these additions:
 *
 * - Tensors of rows of d are given by element strides (the last dimension is
 *   contiguous): each >= 0 and a multiple of 16 bytes' worth of elements, bases
 *   16-byte aligned. A stride of 0 repeats an input; rows of an output must not
 *   overlap (outputs with a stride of 0 over more than one row are refused),
 *   nor an output another tensor of the call, but for ca_rope in place and
 *   ca_paged_chunk_attn, whose out may be q (base and strides the same).
 * - Query head h of `heads` reads key head h / (heads / heads_k); heads_k
 *   divides heads.
 * - Head dimensions: bf16 64 or 128, fp32 any multiple of 4 up to 128 (rotary:
 *   any multiple of 16 bytes up to 128).
 * - Attention adds up probabilities times values in fp32 and divides at the end:
 *   finite values have to stay below 2^96 in size.
 * - Every call can be captured into a graph: it allocates nothing, keeps
 *   nothing from one call for the next and records kernels only. */

/* Rotary positions of up to four axes (time, height, width of a video's
 * tokens; rows and columns of an image; the place in a text).
 *
 * The head's first 2 * npairs dims form npairs = sum of section[] pairs, the
 * first section[0] pairs belonging to axis 0, the next section[1] to axis 1,
 * and so on. Pair i turns by t = x * freq[i], x the token's position on the
 * pair's axis (product, and reduction by multiples of pi/2, in 64 bits):
 *   (u, w) -> (u cos t - w sin t, u sin t + w cos t)
 * in fp32, rounded once. Pairs are dims (2 i, 2 i + 1), or with halves != 0
 * dims (i, i + npairs); the dims from 2 * npairs on are copied. inverse != 0
 * turns by -t: the transposed map, which takes the gradients of the turned
 * rows to those of the rows.
 *
 * Positions: positions[b pos_stride[0] + a pos_stride[1] + i pos_stride[2]]
 * for axis a of token i of batch entry b (device int32; any sign; a stride of
 * 0 repeats). With positions NULL, token i is element i of a row-major grid
 * grid[0] x .. x grid[axes - 1] (n is at most their product), shifted by
 * start[]. */
typedef struct {
  int32_t batch, heads, heads_k; /* heads_k = 0: no keys (k, k_out NULL); need not divide heads */
  int32_t n, d, dtype;           /* tokens per head, head dimension, ca_dtype */
  int32_t axes;                  /* 1..4 */
  int32_t section[4];            /* pairs per axis, >= 0; 2 * their sum in [2, d] */
  int32_t halves;                /* halves: npairs a multiple of 16 bytes' worth of elements */
  int32_t inverse;
  int32_t grid[4], start[4];     /* positions NULL only */
  int64_t pos_stride[3];         /* {batch, axis, token}, positions given */
  int64_t q_stride[3], k_stride[3], q_out_stride[3], k_out_stride[3]; /* {batch, head, token} */
  double freq[64];               /* radians per position, at most 2^20 */
} ca_rope_desc;

/* q_out and k_out may be q and k themselves (with the same strides): the rows
 * then turn in place. Other overlaps are not allowed. */
CA_API int ca_rope(const ca_rope_desc* p, const void* q, const void* k, const int32_t* positions,
                   void* q_out, void* k_out, void* stream);

/* Attention with a sliding window and sinks.
 *
 * Query i of batch entry b sits at p = i + len_k[b] - len_q[b] (the last query
 * beside the last key) and sees key j < len_k[b] where
 *   (j < sinks  or  p - left <= j <= p + right)  and  (not causal  or  j <= p);
 * a negative left or right is no limit. len_q, len_k: optional device int32
 * [batch], clamped to [0, nq] and [0, nk] (NULL: nq, nk).
 *   out = sum_j e^{s_j - lse} v_j, lse = ln sum_j e^{s_j}, s_j = scale q . k_j
 * over the keys it sees (scale <= 0 selects 1/sqrt(d)). A query that sees no
 * key, and every row at or past len_q, has out = 0 and lse = -inf. What rows at
 * or past the lengths hold, and what a key or value that a query does not see
 * holds (infinities and NaN too), does not reach its output; a query
 * that sees a value that is not finite has an output that is not. (The backward
 * pass promises this for rows past the lengths only: a NaN or an infinity
 * in a token reaches the gradients of its neighbours, up to 127 tokens away.) */
typedef struct {
  int32_t batch, heads, heads_k;
  int32_t nq, nk, d, dtype;      /* 1..2^22 queries and keys */
  int32_t left, right, sinks, causal;
  float scale;
  int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3]; /* {batch, head, token} */
  /* ca_window_attn_backward only */
  int64_t dout_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} ca_window;

/* bf16: token strides of at most 2^23 elements (also of dout in the backward
 * pass), and batch * heads * (blocks of 128 tokens) below 2^22.
 * out: strides out_stride; lse: optional dense fp32 [batch][heads][nq]. ws:
 * workspace (long keys for few queries are cut into parts and joined). */
CA_API int ca_window_attn(const ca_window* p, const void* q, const void* k, const void* v,
                          const int32_t* len_q, const int32_t* len_k, void* out, float* lse,
                          void* ws, size_t ws_bytes, void* stream);

/* Bytes of workspace of ca_window_attn (backward 0; may be 0 bytes) or
 * ca_window_attn_backward (backward 1), 256-byte aligned. Host-only. */
CA_API int ca_window_workspace_size(const ca_window* p, int32_t backward, size_t* bytes);

/* Gradients of ca_window_attn: from out and lse as it wrote them (same
 * arguments) and dout, with P = e^{s - lse} and D = row sums of dout * out,
 *   dv = P^T dout,  dS = P (dout v^T - D),  dq = scale dS k,  dk = scale dS^T q,
 * dk and dv summed over the query heads that share the key head. Rows at or
 * past the lengths have zero gradients. */
CA_API int ca_window_attn_backward(const ca_window* p, const void* q, const void* k, const void* v,
                                   const void* out, const float* lse, const void* dout,
                                   const int32_t* len_q, const int32_t* len_k, void* dq, void* dk,
                                   void* dv, void* ws, size_t ws_bytes, void* stream);

/* A paged key-value cache: `pages` pages of `page` tokens in two pools, and per
 * sequence a row of the page table (device int32 [batch][max_pages], rows
 * table_stride apart): token j of sequence b is token j % page of page
 * table[b][j / page]. lens: device int32 [batch], tokens of each sequence,
 * clamped to [0, max_pages * page]. Table entries outside [0, pages) hold no
 * tokens; entries that no visible token needs are not read. */
typedef struct {
  int32_t batch, heads, heads_k, d, dtype;
  int32_t page, pages, max_pages; /* >= 1; max_pages * page < 2^30 */
  int32_t left, sinks;            /* ca_paged_attn: as in ca_window, negative left: the whole cache */
  float scale;
  int64_t table_stride;
  int64_t k_stride[3], v_stride[3]; /* pools: {page, token, head} */
  int64_t q_stride[2], out_stride[2];         /* ca_paged_attn: {batch, head} */
  int32_t n_new;                              /* ca_cache_append: new tokens per sequence */
  int64_t k_new_stride[3], v_new_stride[3];   /* ca_cache_append: {batch, token, head} */
} ca_paged;

/* Writes n_new new keys and values of each sequence at its places lens[b] -
 * n_new .. lens[b] - 1 (lens counts them already; places before 0, past the
 * table or on pages outside the pool are left out). Everything else in the
 * pools stays as it is. Sequences must not write the same place of a page. */
CA_API int ca_cache_append(const ca_paged* p, const void* k, const void* v, void* k_pages,
                           void* v_pages, const int32_t* table, const int32_t* lens, void* stream);

/* Bytes of workspace of ca_paged_attn (256-byte aligned; may be 0). The lengths
 * are on the device, so it goes with the table's width (partial results of up to
 * max_pages * page visible keys for every sequence and head). Host-only. */
CA_API int ca_paged_workspace_size(const ca_paged* p, size_t* bytes);

/* Attention of one query per sequence and head, its last token (position
 * lens[b] - 1), over the sequence's cache: the keys j with j < sinks or
 * j >= lens[b] - 1 - left. Keys that it does not see are not read, so pages that
 * hold no visible token may be gone. A sequence that sees no key has out = 0,
 * lse = -inf. q, out: q_stride, out_stride; lse: optional dense fp32
 * [batch][heads]. */
CA_API int ca_paged_attn(const ca_paged* p, const void* q, const void* k_pages,
                         const void* v_pages, const int32_t* table, const int32_t* lens, void* out,
                         float* lse, void* ws, size_t ws_bytes, void* stream);

/* ---- Chunks of new tokens over the paged cache --------------------------------
 *
 * A step of a serving program takes any number of new tokens of each of its
 * sequences: one where a sequence goes on, a few where drafted tokens are checked,
 * a frame of a video, all of a prompt. The new tokens lie packed, one sequence
 * after the other: those of sequence b are rows starts[b] .. starts[b + 1] - 1 of
 * arrays of `tokens` rows (starts: device int32 [batch + 1], ascending from 0; the
 * rows from starts[batch] on are room for more). lens[b] counts the sequence's
 * tokens, the new ones, its last, included.
 *
 * ca_cache_grow finds pages for the new tokens and says where they go,
 * ca_cache_write puts their keys and values there, ca_paged_chunk_attn attends,
 * ca_cache_release gives pages back.
 *
 * The pages that no sequence holds are free_pages[0 .. state[0] - 1], a stack:
 * device int32 free_pages[pages], the next page to be taken last. state: device
 * int32 [3]: the number of free pages; pages that the last ca_cache_grow lacked;
 * new tokens for which it had no rows. A free page must not stand twice in the
 * stack, nor in a table. A page may stand in several rows of the table (a common
 * beginning) if it is full: ca_cache_grow leaves an entry that holds a page as it
 * is, so sequences that go on inside a shared page would write over each other
 * (copy such a page to one of its own first). */
typedef struct {
  int32_t batch, page, pages, max_pages; /* as in ca_paged; max_pages * page < 2^30 */
  int32_t tokens;                        /* ca_cache_grow: rows of slots and positions, >= 1 */
  int32_t left, sinks;                   /* ca_cache_release */
  int64_t table_stride;                  /* >= max_pages where batch > 1 */
} ca_pages;

/* Pages for the new tokens of a step, and where they go. n_new: device int32
 * [batch], how many of the lens[b] tokens are new (clamped to [0, lens[b]]; lens to
 * [0, max_pages * page]).
 *
 * Every entry of the table that a new token lies on (those of places lens[b] -
 * n_new[b] .. lens[b] - 1) and that holds no page (a value outside [0, pages)) gets
 * one: the first such entry, by sequence and place, the last of the stack, and so
 * on. Entries that hold one stay, so a call repeated changes nothing. Where the
 * stack runs short the later entries stay as they are and state[1] says how
 * many; it is 0 else. Their tokens have no slot and are not written: for this step's
 * attention they are not there, and a later step has to bring them again (a page
 * found for them then holds nothing of theirs).
 *
 * starts[b] = the sum of n_new[0 .. b - 1], at most `tokens` (state[2] says how many
 * tokens are beyond). slots (device int64 [tokens]): the place of a row's token in
 * the pools, page * (its table entry) + place in the page, -1 where there is no
 * page and in rows from starts[batch] on. positions (device int32 [tokens]): the
 * token's place in its sequence (as ca_rope reads it), 0 in rows from
 * starts[batch] on.
 *
 * Where state[2] > 0 a sequence has rows for the first of its new tokens only, or
 * for none, and lens[b] counts tokens that are not written in this step:
 * ca_paged_chunk_attn, whose rows are a sequence's last tokens, would take its rows
 * for later ones and read places without a token. ca_cache_grow_seen also says how
 * far the rows go, seen (device int32 [batch]): lens[b] less the new tokens of b that
 * have no row (lens[b], as clamped, where all have one). Calls that take seen for
 * lens are right whatever n_new was, and the tokens left out are the next step's
 * first ones. */
CA_API int ca_cache_grow(const ca_pages* p, const int32_t* lens, const int32_t* n_new,
                         int32_t* table, int32_t* free_pages, int32_t* state, int32_t* starts,
                         int64_t* slots, int32_t* positions, void* stream);
CA_API int ca_cache_grow_seen(const ca_pages* p, const int32_t* lens, const int32_t* n_new,
                              int32_t* table, int32_t* free_pages, int32_t* state,
                              int32_t* starts, int64_t* slots, int32_t* positions, int32_t* seen,
                              void* stream);

/* Gives back the pages that hold no token which the next one of its sequence sees:
 * an entry i of row b keeps its page where a token j of its places (i * page <= j <
 * (i + 1) * page) has j < lens[b] and, with left >= 0, j < sinks or j >= lens[b] -
 * left. All others in [0, pages) go to the stack, the first one, by sequence and
 * place, on top (what ca_cache_grow took goes back as it came), and become -1.
 * lens[b] = 0 gives back all of a finished sequence, a smaller length than before
 * the pages of rejected tokens, left and sinks those behind a window. A page that
 * stands in several rows (a common beginning) must not go back from two of them, nor
 * from one while another holds it.
 * ws: workspace (ca_cache_release_workspace_size, 256-byte aligned). */
CA_API int ca_cache_release(const ca_pages* p, const int32_t* lens, int32_t* table,
                            int32_t* free_pages, int32_t* state, void* ws, size_t ws_bytes,
                            void* stream);
CA_API int ca_cache_release_workspace_size(const ca_pages* p, size_t* bytes);

/* Attention of the new tokens, and what ca_cache_write writes */
typedef struct {
  int32_t batch, heads, heads_k, d, dtype; /* ca_cache_write: heads_k, d and dtype only */
  int32_t page, pages, max_pages;          /* ca_cache_write: page and pages only */
  int32_t tokens;                          /* rows of q and out (of k and v), 1..2^24 */
  int32_t left, right, sinks, causal;      /* as in ca_window */
  float scale;
  int64_t table_stride;
  int64_t k_stride[3], v_stride[3];         /* pools: {page, token, head} */
  int64_t q_stride[2], out_stride[2];       /* {token, head} */
  int64_t k_new_stride[2], v_new_stride[2]; /* ca_cache_write: {token, head} */
} ca_chunk;

/* Writes row t of k and v to place slots[t] (device int64 [tokens]) of the pools:
 * token slots[t] % page of page slots[t] / page. Rows whose slot lies outside
 * [0, pages * page) are left out. No two rows may have the same slot. */
CA_API int ca_cache_write(const ca_chunk* p, const void* k, const void* v, void* k_pages,
                          void* v_pages, const int64_t* slots, void* stream);

/* Attention of packed queries over the cache of their sequences. Query i of the
 * lq = starts[b + 1] - starts[b] of sequence b sits at p = i + lens[b] - lq (the last
 * one beside the last key) and sees the keys that ca_window_attn shows it: j <
 * lens[b] where (j < sinks or p - left <= j <= p + right) and (not causal or j <= p).
 * out, lse as there: 0 and -inf where a query sees no key. Keys on entries outside
 * [0, pages) are not there; what keys and values that a query does not see
 * hold does not reach it. starts are clamped to [0, tokens], lens to
 * [0, max_pages * page]. Rows of out and lse (optional, dense fp32 [tokens][heads])
 * before starts[0] and from starts[batch] on are left as they were. ws: workspace. */
CA_API int ca_paged_chunk_attn(const ca_chunk* p, const void* q, const void* k_pages,
                               const void* v_pages, const int32_t* table, const int32_t* lens,
                               const int32_t* starts, void* out, float* lse, void* ws,
                               size_t ws_bytes, void* stream);

/* Bytes of workspace of ca_paged_chunk_attn (256-byte aligned; may be 0). Host-only. */
CA_API int ca_paged_chunk_workspace_size(const ca_chunk* p, size_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* CLUSTERATTN_H_ */
