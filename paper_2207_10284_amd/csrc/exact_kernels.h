// Launchers of the exact-attention kernels (internal; the public interface is
// mra_exact.h). Every launcher only enqueues on `stream` and returns
// hipGetLastError(). Arguments are assumed validated by the caller (exact_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mra_exact.h"

namespace mra {

// A tensor as the kernels take it: strides in bytes.
struct Rows {
  char* p;
  long long sb, sh, sn;
};

// What every kernel of a call shares.
struct ExactArgs {
  Rows q, k, v, out;
  int B, H, Hkv, group, nq, nk;
  int causal;
  float scale, scale_log2;                // scale, and scale log2(e)
  const int32_t* lengths;
  const int32_t* q_start;
  const uint8_t* key_mask;
  long long mask_stride;
  const void* bias;
  int bias_bf16, buckets, far;
  const int32_t* map;
};

// Few rows per key head: `splits` workgroups share the keys of each 32 rows and
// leave partial results (see exact_split_kernel) in the workspace.
struct SplitPlan {
  bool use;                               // the split kernel at all
  int splits, mtiles;                     // workgroups per 32 rows; groups of 32 rows per key head
  size_t bytes;                           // workspace (0 for one split)
};
SplitPlan exact_split_plan(const mra_exact_problem_t& p);

hipError_t launch_exact_forward(const ExactArgs& a, int d, int dtype, float* lse, const SplitPlan& plan, void* ws,
                                hipStream_t stream);

struct ExactGrads {
  Rows dout, dq, dk, dv;
  const float* lse;
  float* delta;                           // [B, H, n_q]: G . Z per query
  float* diag;                            // [H, B, blocks, slots, window]: sums of dS over diagonals; null: not asked for
  int slots;                              // parts of the dQ pass, and one of exact_centre_kernel
  float* row_sums;                        // [parts, B, H, n_q, 4]: see exact_centre_kernel; null: it does not run
  void* dbias;
  float *part_q, *part_k, *part_v;        // [parts, B, heads, n, d]: see BackwardPlan
};

// How many workgroups share a block of the passes, and the floats of their partial sums.
struct BackwardPlan {
  int dq_parts, dkv_parts;
  bool centre;                            // exact_centre_kernel, where dbias is asked for
  size_t q_floats, k_floats;              // of dq; of dk, and of dv (0: one part)
};
BackwardPlan exact_backward_plan(const mra_exact_problem_t& p);
// Workgroups whose diagonal sums a query block has.
inline int exact_slots(const BackwardPlan& b) { return b.dq_parts + (b.centre ? 1 : 0); }
// Query blocks of the dQ pass per head and floats of a block's diagonal sums.
int exact_dq_blocks(int nq);
int exact_window(int far);
hipError_t launch_exact_backward(const ExactArgs& a, const ExactGrads& g, const BackwardPlan& plan, int d, int dtype,
                                 hipStream_t stream);

}  // namespace mra
