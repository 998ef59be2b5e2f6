/*
 * mra_exact.h — C ABI of libmra_exact: exact softmax attention, its gradients
 * and a learned position bias on AMD Instinct MI355X (gfx950), the operators
 * that MRA-2 (mra.h) approximates, for the calls it does not take: any length,
 * padded batches, causal rows, shared key heads, single tokens.
 *
 * For batch b, query head h and query i, which stands at position
 * p = q_start[b] + i (default n_k - n_q + i, so that the last query stands at
 * the last key), over the keys j that count for it,
 *
 *   S_ij = scale q_i . k_j + bias[bucket_map[clamp(j - p, -far, far) + far]][h]
 *   L_i  = ln sum_j exp(S_ij)
 *   Z_i  = sum_j exp(S_ij - L_i) v_j
 *
 * (Sec. 2.1 eq. softmax-attention of the paper, arXiv 2207.10284, with scale
 * 1/sqrt(d) and no bias). A key counts if j < lengths[b], key_mask[b][j] != 0
 * and, in causal problems, j <= p; each of the three only where given. A query
 * for which no key counts has Z_i = 0 and L_i = -infinity. Query head h reads
 * key head h / (H / H_kv).
 *
 * Conventions
 * -----------
 * - Status codes, element types, the stream argument, 16-byte alignment, and
 *   that the library never allocates, frees or synchronises: as in mra.h.
 * - Tensors are DEVICE pointers with three strides in elements and dense rows
 *   (the d elements of a row are consecutive). Every stride is >= 0 and a
 *   multiple of 16 bytes. Input strides may be 0 (a broadcast axis). Outputs
 *   must not overlap themselves or another argument.
 * - d is 32, 64 or 128; 0 <= n_q, n_k <= 2^26; row strides below 2^25 bytes. A
 *   pass has below 2^24 workgroups: B H ceil(n_q / 128), and in the backward
 *   B H_kv ceil(n_k / 128); a forward with r = n_q H / H_kv <= 64 rows per key head
 *   has B H_kv ceil(r / 32) instead.
 * - A bias below -2^14 (-infinity and the usual masks of -1e9, -1e30 or a type's
 *   lowest value among them) takes its distances out: such a key does not count.
 *   One above 2^14 is taken as 2^14: its keys outweigh all others, and among
 *   each other weigh as if such entries were equal. None is NaN.
 * - What lies at a key that does not count for any query of its batch
 *   (j >= lengths[b], key_mask[b][j] == 0) may be anything, also NaN. Results
 *   for other non-finite inputs are unspecified.
 * - Device values are taken within their range: lengths[b] within [0, n_k],
 *   q_start[b] within [-2^29, 2^29]; a bucket_map entry outside [0, buckets)
 *   adds no bias and takes no gradient.
 * - Products accumulate in float32; bfloat16 inputs feed bfloat16 matrix
 *   products with the softmax weights (and, backward, the logit gradients)
 *   rounded to bfloat16 before their products; float32 operands enter as sums
 *   of three bfloat16 values, as in mra.h. Results are rounded once. L is one
 *   float32, so the probabilities formed from it are off by about |L| 2^-23.
 * - Results of a call do not change from run to run: no sum depends on the
 *   order in which workgroups run.
 */
#ifndef MRA_EXACT_H_
#define MRA_EXACT_H_

#include "mra.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MRA_EXACT_MAX_FAR 512
#define MRA_EXACT_MAX_BUCKETS 1024

typedef struct {
  int B, H, H_kv;             /* batches, query heads, key heads; H a multiple of H_kv */
  int n_q, n_k, d;
  mra_dtype_t dtype;          /* of q, k, v, out and their gradients */
  float scale;                /* 2^-64 to 2^64 */
  int causal;                 /* 0 or 1 */
  const int32_t* lengths;     /* device [B], or NULL: every key */
  const int32_t* q_start;     /* device [B], or NULL: n_k - n_q */
  const uint8_t* key_mask;    /* device, n_k bytes per batch, or NULL: every key */
  int64_t key_mask_stride;    /* bytes from one batch's mask to the next, >= 0 */
  const void* bias;           /* device [buckets][H] of bias_dtype, or NULL: none */
  mra_dtype_t bias_dtype;
  int buckets;                /* 1 .. MRA_EXACT_MAX_BUCKETS with bias */
  const int32_t* bucket_map;  /* device [2 far + 1]: bucket of each distance key - position */
  int far;                    /* 0 .. MRA_EXACT_MAX_FAR; distances beyond take the outer entries */
} mra_exact_problem_t;

/* A tensor [B][heads][rows][d]: element strides of the three outer axes. */
typedef struct {
  void* data;
  int64_t stride_b, stride_h, stride_n;
} mra_strided_t;

/*
 * mra_exact_forward_workspace_bytes — device workspace of mra_exact_forward
 * (partial results of rows whose keys several workgroups share; 0 if there are
 * none, and for invalid or unsupported problems).
 */
size_t mra_exact_forward_workspace_bytes(const mra_exact_problem_t* p);

/*
 * mra_exact_forward — Z and, if lse_out is not NULL, L.
 *   q, out    : [B][H][n_q][d]; k, v : [B][H_kv][n_k][d].
 *   lse_out   : [B][H][n_q] float32, dense, or NULL.
 *   workspace : at least mra_exact_forward_workspace_bytes(p) bytes; may be NULL
 *               where that is 0. Contents on entry are ignored.
 * B, H, n_q may be 0 (nothing to compute); with n_k = 0 no key counts and k, v
 * are not read.
 */
mra_status_t mra_exact_forward(const mra_exact_problem_t* p, const mra_strided_t* q,
                               const mra_strided_t* k, const mra_strided_t* v,
                               const mra_strided_t* out, float* lse_out, void* workspace,
                               size_t workspace_bytes, void* stream);

/*
 * mra_exact_backward_workspace_bytes — device workspace of mra_exact_backward;
 * 0 for empty, invalid or unsupported problems.
 */
size_t mra_exact_backward_workspace_bytes(const mra_exact_problem_t* p);

/*
 * mra_exact_backward — the gradients, with the probabilities formed again from
 * the log normalisers (P = exp(S - L)): for the gradient G of Z,
 *   dV_j = sum_i P_ij G_i,   D_ij = P_ij (G_i . v_j - G_i . Z_i)  (dS)
 *   dQ_i = scale sum_j D_ij k_j,   dK_j = scale sum_i D_ij q_i,
 *   dbias[c][h] = sum of D_ij over batches, queries and keys with bucket c.
 * dK and dV sum over the query heads of a key head; they are 0 for keys that
 * do not count.
 *   out, lse : as mra_exact_forward wrote them for the same problem.
 *   dout     : [B][H][n_q][d], the gradient of out.
 *   dq, dk, dv : outputs with the shapes of q, k, v.
 *   dbias    : [buckets][H] of bias_dtype, or NULL to skip; NULL without bias. Over
 *              many keys per distance of the map, where D's terms cancel, its D is
 *              held to sum to 0 over a query's keys (bfloat16).
 */
mra_status_t mra_exact_backward(const mra_exact_problem_t* p, const mra_strided_t* q,
                                const mra_strided_t* k, const mra_strided_t* v,
                                const mra_strided_t* out, const mra_strided_t* dout,
                                const float* lse, const mra_strided_t* dq,
                                const mra_strided_t* dk, const mra_strided_t* dv, void* dbias,
                                void* workspace, size_t workspace_bytes, void* stream);

/* hipError_t of the calling thread's last MRA_ERR_HIP from this library. */
int mra_exact_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif  /* MRA_EXACT_H_ */
