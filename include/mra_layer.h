/*
 * mra_layer.h — C ABI of libmra_layer: what stands around attention in a
 * decoder's layer, on AMD Instinct MI355X (gfx950): rotary positions, norms of
 * queries and keys per head in the same pass, a paged cache of keys and values
 * in 4 bits, and attention over that cache.
 *
 * Conventions
 * -----------
 * - Status codes, element types, the stream argument, 16-byte alignment, and
 *   that the library never allocates, frees or synchronises: as in mra.h.
 * - Tensors [B][heads][rows][d] are given as in mra_exact.h (mra_strided_t): three
 *   strides in elements, dense rows of d elements, each stride >= 0 and a multiple of 16
 *   bytes. Input strides may be 0. Outputs must not overlap themselves or, where
 *   not said otherwise, another argument.
 * - d is 32, 64 or 128; rotary calls have below 2^27 tokens (B n); writing and reading the
 *   cache, sequences times key heads times tiles of 64 tokens, (n + 62) / 64 + 1, are below 2^24; attention has at most
 *   2^30 rows (B H n_q) and below 2^23 row tiles (16 rows of a key head up to 64 of them, else 128);
 *   heads are at most 2^16.
 * - Everything is computed in float32 (angles in float64)
 *   and rounded once, if not said otherwise.
 * - Results do not change from run to run.
 */
#ifndef MRA_LAYER_H_
#define MRA_LAYER_H_

#include "mra_exact.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * Rotary positions and head norms
 *
 * A row x of d elements of a query or key head, at position p. With a weight w
 * its norm is taken first, x_i <- x_i w_i / sqrt(mean(x^2) + eps). Then pair
 * (a, b) of the first `rot` elements, of frequency f = freqs[i], becomes
 *
 *   a' = m (a cos(p f) - b sin(p f))     b' = m (b cos(p f) + a sin(p f))
 *
 * Pair i is the elements i and i + rot/2, or 2i and 2i + 1 (interleaved). The elements
 * from rot on stay as they are.
 *
 * The angle p f is taken in turns, in float64, and its whole turns leave it before it is rounded; cosine and sine are
 * float32, off by some 2^-23 at every position, far or near. Of rows with a
 * norm the mean square is within float32's range.
 */
typedef struct {
  int B, H, H_kv, n, d;       /* H or H_kv may be 0: no queries, no keys */
  int rot;                    /* a multiple of 16, 0 to d */
  mra_dtype_t dtype;
  int interleaved;            /* 0 or 1 */
  float magnitude;            /* m, finite */
  float eps;                  /* > 0, finite; of the norms */
  const double* freqs;        /* device [rot / 2], radians a position; NULL with rot 0 */
  const int32_t* positions;   /* device, n per batch, or NULL: token i stands at i */
  int64_t positions_stride;   /* elements from one batch's positions to the next, >= 0 */
  const void* q_weight;       /* device [d] of weight_dtype, or NULL: no norm */
  const void* k_weight;
  mra_dtype_t weight_dtype;
} mra_rotary_problem_t;

/*
 * mra_rotary_forward — q [B][H][n][d] to q_out, k [B][H_kv][n][d] to k_out. An
 * output may be its input (same data and strides): then it is changed in place.
 */
mra_status_t mra_rotary_forward(const mra_rotary_problem_t* p, const mra_strided_t* q,
                                const mra_strided_t* k, const mra_strided_t* q_out,
                                const mra_strided_t* k_out, void* stream);

/* Device workspace of mra_rotary_backward (partial sums of the weights' gradients). */
size_t mra_rotary_backward_workspace_bytes(const mra_rotary_problem_t* p);

/*
 * mra_rotary_backward — gradients, for those of the results (dq_out, dk_out): with
 * g the result's gradient rotated back, r = 1 / sqrt(mean(x^2) + eps), y = r x,
 *   no weight: dx = g;  else h = w g, dx = r (h - y mean(h y)),
 *   dw = sum of g y over batches, heads and tokens.
 * q, k are read where they have a weight (may be NULL otherwise). dq may be dq_out
 * (same data and strides), dk dk_out. dq_weight, dk_weight: [d] of weight_dtype, or NULL
 * to skip; NULL without that weight. They are 0 where there are no rows.
 */
mra_status_t mra_rotary_backward(const mra_rotary_problem_t* p, const mra_strided_t* q,
                                 const mra_strided_t* k, const mra_strided_t* dq_out,
                                 const mra_strided_t* dk_out, const mra_strided_t* dq,
                                 const mra_strided_t* dk, void* dq_weight, void* dk_weight,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * A paged cache of keys and values in 4 bits
 *
 * 32 consecutive channels of a token of one head share a step s = 2^e, the
 * smallest power of two with max |x| <= 7 s, -125 <= e <= 125. x / s (exact) is
 * rounded to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, ties
 * to the even one in this order, to 6 beyond it. So no value is off by more than half the
 * distance of its neighbours (s beyond 6 s; beyond 7 2^125, infinity included, it is 6 2^125), all that
 * the cache holds is exact in bfloat16, and every way to evaluate the above gives the same. What is held
 * for a block with a NaN is unspecified, and finite.
 *
 * The bytes of one page of one head, page_size tokens of d channels (4 bits: codes
 * 0 to 7 in the order above, 8 more for negative ones; e is held as e + 127):
 *   keys, values           [page_size][d/2] each; channel 2j low, 2j + 1 high
 *   key and value steps    [page_size][d/32] each
 *
 * A sequence's tokens lie in the pages of its row of `table`: token t in page
 * table[b][t / page_size], place t % page_size. Sequences may share pages. An entry
 * outside [0, pages) is no page: what would be written there is not, and nothing is
 * read there.
 */
typedef struct {
  int pages, H_kv, d;
  int page_size;              /* a power of two, 32 to 1024 */
  void* data;                 /* device [pages][H_kv][mra_fp4_page_bytes(page_size, d)], 16-byte aligned */
  const int32_t* table;       /* device [B][max_pages] */
  int B, max_pages;           /* max_pages page_size <= 2^26 */
} mra_fp4_cache_t;

/* page_size (d + d / 16); 0 for sizes that are not supported. */
size_t mra_fp4_page_bytes(int page_size, int d);

/*
 * mra_fp4_cache_write — token i < counts[b] of sequence b, keys k and values v
 * [B][H_kv][n][d] of dtype, to place starts[b] + i.
 *   starts, counts : device [B], or NULL: 0, n. Taken within [0, max_pages page_size]
 *                    and [0, n].
 * Only the bytes of the tokens written change. Two sequences that write to one
 * place leave either's values, or a mix.
 */
mra_status_t mra_fp4_cache_write(const mra_fp4_cache_t* cache, const mra_strided_t* k,
                                 const mra_strided_t* v, int n, mra_dtype_t dtype,
                                 const int32_t* starts, const int32_t* counts, void* stream);

/*
 * mra_fp4_cache_read — the values held at places starts[b] + i to row i < counts[b]
 * of k_out and v_out [B][H_kv][n][d]; 0 in the other rows and where there is no page.
 */
mra_status_t mra_fp4_cache_read(const mra_fp4_cache_t* cache, const mra_strided_t* k_out,
                                const mra_strided_t* v_out, int n, mra_dtype_t dtype,
                                const int32_t* starts, const int32_t* counts, void* stream);

/* ---------------------------------------------------------------------------
 * Attention over that cache
 *
 * For query i of sequence b, at position p = q_start[b] + i (default lengths[b] - n_q
 * + i), over the tokens j < lengths[b] (causal: j <= p) that have a page,
 *
 *   S_ij = scale q_i . k_j    L_i = ln sum_j exp(S_ij)    Z_i = sum_j exp(S_ij - L_i) v_j
 *
 * Query head h reads key head h / (H / H_kv). A query without keys has Z = 0, L = -infinity.
 * One that has a key and holds a NaN or an infinity has NaN in all of Z and in L; other queries are as without it.
 * Products accumulate in float32; the cache's values enter them exactly, bfloat16 queries as they are with the
 * weights rounded to bfloat16; float32 queries and their weights as sums of three bfloat16 values.
 */
typedef struct {
  int H, n_q;                 /* H a multiple of the cache's H_kv */
  mra_dtype_t dtype;          /* of q and out */
  float scale;                /* 2^-64 to 2^64 */
  int causal;                 /* 0 or 1 */
  const int32_t* lengths;     /* device [B]; taken within [0, max_pages page_size] */
  const int32_t* q_start;     /* device [B], taken within [-2^29, 2^29], or NULL */
} mra_fp4_attention_t;

/* Device workspace of mra_fp4_attention (0: none). */
size_t mra_fp4_attention_workspace_bytes(const mra_fp4_cache_t* cache, const mra_fp4_attention_t* p);

/*
 * mra_fp4_attention — Z to out [B][H][n_q][d] and, if lse_out is not NULL, L
 * (float32 [B][H][n_q], dense).
 */
mra_status_t mra_fp4_attention(const mra_fp4_cache_t* cache, const mra_fp4_attention_t* p,
                               const mra_strided_t* q, const mra_strided_t* out, float* lse_out,
                               void* workspace, size_t workspace_bytes, void* stream);

/* hipError_t of the calling thread's last MRA_ERR_HIP from this library. */
int mra_layer_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif  /* MRA_LAYER_H_ */
