/*
 * vs_softmax.h -- C ABI of the softmax operators over the rows of an index (libvs_softmax.so).
 *
 * A search (vs.h) returns the k best rows for a query; the operators here weigh all rows by the
 * softmax of their scores: log-probabilities of given rows with their gradients, for training the
 * vectors that an index holds and for answering with them, and attention over the compressed vectors of a
 * 4-bit IVF-PQ index with its gradient, for reading an index as a memory.
 *
 * Conventions are those of vs.h (device pointers, row-major and contiguous arrays, work enqueued on
 * `hip_stream`, VS_OK or a negative error code, nothing thrown), and:
 *   - The calls allocate and synchronise nothing: work space is the caller's (`workspace`, 256-byte
 *     aligned, at least what the *_workspace_bytes function of the same arguments returns).  Its contents need not be kept
 *     between calls.  Calls that may run at the same time, and captured graphs that may, take a work space each.
 *   - Vectors are fp32, fp16 or bf16 (`dtype`), 16-byte aligned.  Scores, normalisers and sums are fp32.
 *   - Results do not depend on the order in which workgroups run: equal calls give equal bits.
 */
#ifndef VS_SOFTMAX_H_
#define VS_SOFTMAX_H_

#include "vs.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { VS_FP32 = 0, VS_FP16 = 1, VS_BF16 = 2 };
#define VS_MAX_TOP 64     /* largest k of vs_flat_logprob */
#define VS_MAX_ROW 65536 /* largest d of vs_flat_logprob */

/*
 * Log-probabilities under the softmax of exact inner products:
 *   s_ij = scale <q_i, x_j> + bias_j,  lse_i = log sum_j exp(s_ij),  logp_ij = s_ij - lse_i.
 *   x           [nb, d], q [nq, d]: the rows and the queries, both of `dtype`.  nb < 2^31, nq < 2^31.
 *   bias        [nb] fp32 or NULL (zeros).  A row whose bias is -inf does not exist: it has probability 0
 *               whatever it holds, infinities and NaN included.
 *   targets     [nq, nt] int64 or NULL (nt = 0): rows whose log-probability is asked for.  Entries outside
 *               [0, nb) are skipped (their log-probability is 0).
 *   out_logp    [nq, nt] fp32; -inf for a row that does not exist.
 *   out_lse     [nq] fp32;  out_entropy [nq] fp32: -sum_j p_ij logp_ij.
 *   out_top_logp, out_top_ids [nq, k] fp32, int64: the k largest log-probabilities and their rows, best first,
 *               ties to the smaller row; slots without a row: -inf and -1.  k = 0: none (NULL).
 * A query without any row (nb = 0, or every bias -inf): lse -inf, entropy 0, logp -inf, no alternatives.
 * A score of +inf or NaN makes its query's lse, entropy and log-probabilities NaN.
 * Scores are fp32 sums of products; these are exact (fp32: rounded) up to 64 queries and for fp16 and bf16 rows of a multiple
 * of 64 components.  Otherwise rows are multiplied from copies relative to the largest component of their row: 16-bit
 * components lose at most 2^-39 of it (nothing above 2^-31 of it); fp32 ones, two fp16 parts each, at most 2^-24 of themselves
 * or 2^-39 of it, and a score at most 2^-21 |q||x| that way.  Order among scores closer than their rounding may differ from
 * the exact one; rows that are equal go by number.
 * Errors: null pointers (with nq > 0), d outside [1, VS_MAX_ROW], nb or nq outside [0, 2^31), nt < 0, k outside [0, VS_MAX_TOP], unknown
 * dtype, scale not finite, misaligned vectors or work space, a work space that is too small.  nq = 0 is a no-op.
 */
VS_API int64_t vs_flat_logprob_workspace_bytes(int64_t nb, int64_t nq, int32_t d, int32_t dtype, int32_t k);
VS_API int vs_flat_logprob(const void* x, int64_t nb, const void* q, int64_t nq, int32_t d, int32_t dtype, float scale,
                    const float* bias, const int64_t* targets, int32_t nt, int32_t k, float* out_logp, float* out_lse,
                    float* out_entropy, float* out_top_logp, int64_t* out_top_ids, void* workspace,
                    int64_t workspace_bytes, void* hip_stream);

/*
 * Gradients of vs_flat_logprob for the queries, the rows and the bias; the probabilities are computed again
 * from lse.  With g_logp, g_lse and g_entropy the gradients of a loss for its outputs (the alternatives' gradient goes through
 * targets), the gradient of the loss for a score is
 *   G_ij = p_ij (g_lse_i - sum_t g_logp_it) - g_entropy_i p_ij (logp_ij + entropy_i) + sum_{t: target_it = j} g_logp_it,
 * 0 for rows that do not exist, and
 *   dq_i = scale sum_j G_ij x_j,  dx_j = scale sum_i G_ij q_i,  dbias_j = sum_i G_ij.
 *   lse         [nq] fp32 as returned by vs_flat_logprob; entropy [nq] fp32 likewise, read if g_entropy is given.
 *   g_logp [nq, nt], g_lse [nq], g_entropy [nq]: fp32, each may be NULL (zeros); a target listed twice counts twice.
 *   out_dq [nq, d], out_dx [nb, d] of `dtype`, out_dbias [nb] fp32: each may be NULL (not wanted).
 * A query whose g_logp, g_lse or g_entropy is infinite or NaN: NaN in its dq and in dx and dbias of the rows that exist.
 * One for which all three are 0 takes no part, whatever it holds.
 * The scores are computed as vs_flat_logprob does beyond 64 queries.  G is held in fp16 relative to a bound of its row (for
 * fp32 vectors in two parts, together 22 bits), 2^-11 of a value or 2^-38 of the bound.  The vectors that it multiplies are
 * held likewise, relative to the largest component of their column: column t of dq with x_jt over the rows that exist, column
 * t of dx with bound_i q_it over the queries; 2^-24 (fp32) or nothing (16 bits) of a component is lost, and at most 2^-39 of that
 * largest one.  Sums are fp32.
 * Errors: as vs_flat_logprob; entropy missing where g_entropy is given; VS_ERR_UNSUPPORTED beyond 2^23 tiles of 128 rows or
 * components by 64 queries.  nq = 0 sets out_dx and out_dbias to zero.
 */
VS_API int64_t vs_flat_logprob_grad_workspace_bytes(int64_t nb, int64_t nq, int32_t d, int32_t dtype);
VS_API int vs_flat_logprob_grad(const void* x, int64_t nb, const void* q, int64_t nq, int32_t d, int32_t dtype, float scale,
                         const float* bias, const int64_t* targets, int32_t nt, const float* lse, const float* entropy,
                         const float* g_logp, const float* g_lse, const float* g_entropy, void* out_dq, void* out_dx,
                         float* out_dbias, void* workspace, int64_t workspace_bytes, void* hip_stream);

/*
 * Attention over the vectors of a 4-bit IVF-PQ index (VS_METRIC_IP): every stored vector x'_j = centroid of its list
 * + its codewords is a key in its components [0, dk) and a value in its components [v0, d):
 *   s_ij = scale <q_i, x'_j[0:dk]>,  out_i = sum_j softmax_j(s_ij) x'_j[v0:d],  lse_i = log sum_j exp(s_ij).
 * dk = d, v0 = 0: the vectors are their own values; dk = v0: a key and a value side by side; both whole
 * sub-quantizers (multiples of d / M).
 *   q        [nq, dk] of `dtype`; heads that share a memory are queries of one call.
 *   nprobe   0: over all stored vectors.  Otherwise over the nprobe lists that vs_ivfpq_coarse returns for the query
 *            with zeros behind its dk components (all lists where nprobe >= nlist).
 *   limits   [nq] int64 or NULL: query i sees the vectors whose id is below limits[i] (positions up to its own).
 *   out      [nq, d - v0] of `dtype`, out_lse [nq] fp32 (may be NULL).  A query that sees nothing: zeros and -inf.
 * Scores, weights and sums are fp32, in one of two forms by the size of the call: sums of look-ups in fp32 tables, or, for many
 * queries over all lists, products of fp16 parts of codewords and queries.  These keep 2^-24 of a component or 2^-39 of the
 * largest codeword in it (components more than 2^24 smaller than the largest one: 2^-63 of that), as long as the centroids are
 * less than 2^40 of it; the weights are then held in 22 bits, for fp16 and bf16 queries in 11.
 * The index is not written.  With 0 < nprobe < nlist the coarse quantizer uses the index's own work space, as
 * vs_ivfpq_search does: such calls on one index must not overlap in time, the first of a size allocates, and a stream under
 * capture is refused (VS_ERR_UNSUPPORTED).  A captured call holds the addresses of the index's storage: its graph must not be
 * replayed once vectors have been added to the index, or the index is destroyed.
 * Errors: null pointers (with nq > 0), an index with another metric or with 8-bit codes (VS_ERR_UNSUPPORTED), dk or v0
 * outside their range or inside a sub-quantizer, nprobe outside [0, VS_MAX_K], scale not finite, misaligned vectors or work space, a
 * work space that is too small, an index of another device than the current one; VS_ERR_UNSUPPORTED where the tables of a
 * query exceed the on-chip memory: with sub-quantizers of up to 8 components, M <= 256 fits where dk = d and v0 = 0 and
 * M <= 400 where dk = v0 = d / 2, of the gradient M <= 128 and M <= 256.
 */
VS_API int64_t vs_ivfpq_attend_workspace_bytes(const vs_ivfpq* ix, int64_t nq, int32_t dk, int32_t v0, int32_t dtype,
                                               int32_t nprobe);
VS_API int vs_ivfpq_attend(const vs_ivfpq* ix, const void* q, int64_t nq, int32_t dk, int32_t v0, int32_t dtype,
                    int32_t nprobe, float scale, const int64_t* limits, void* out, float* out_lse, void* workspace,
                    int64_t workspace_bytes, void* hip_stream);

/*
 * Gradient of vs_ivfpq_attend for the queries (the index is a memory that is not trained); the probabilities are
 * computed again from lse:
 *   dp_ij = <g_out_i, x'_j[v0:d]>,  dq_i = scale sum_j p_ij (dp_ij - sum_j p_ij dp_ij + g_lse_i) x'_j[0:dk].
 *   lse [nq] fp32 as returned by vs_ivfpq_attend with the same index, queries, nprobe, scale and limits;
 *   g_out [nq, d - v0] of `dtype`; g_lse [nq] fp32 or NULL;  out_dq [nq, dk] of `dtype`.
 * Errors: as vs_ivfpq_attend.
 */
VS_API int64_t vs_ivfpq_attend_grad_workspace_bytes(const vs_ivfpq* ix, int64_t nq, int32_t dk, int32_t v0,
                                                    int32_t dtype, int32_t nprobe);
VS_API int vs_ivfpq_attend_grad(const vs_ivfpq* ix, const void* q, int64_t nq, int32_t dk, int32_t v0, int32_t dtype,
                         int32_t nprobe, float scale, const int64_t* limits, const float* lse, const void* g_out,
                         const float* g_lse, void* out_dq, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* Message of the calling thread's most recent error in a function of this header ("" if none). */
VS_API const char* vs_softmax_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* VS_SOFTMAX_H_ */
