// Launchers of libmra_layer's kernels (internal; the public interface is mra_layer.h).
// Every launcher only enqueues on `stream` and returns hipGetLastError(). Arguments are
// assumed validated by the caller (layer_api.cpp).
#pragma once

#include "exact_kernels.h"
#include "mra_layer.h"

namespace mra {

// One side (queries or keys) of a rotary call.
struct RotarySide {
  Rows x, y;                              // forward: input, result; backward: input (with a weight), dx
  Rows g;                                 // backward: the result's gradient
  const void* w;
  int heads;
  int head_fast;                          // a token's heads lie closer than a head's tokens
};

struct RotaryArgs {
  RotarySide side[2];
  int n, rot, weight_bf16;
  long long tokens;                       // B n
  const double* freqs;
  const int32_t* positions;
  long long positions_stride;
  float magnitude, eps;
  float* part;                            // backward: [workgroups][2][d] sums of the weights' gradients, or null
};

// Workgroups of the backward, whose partial sums the workspace holds.
int rotary_backward_groups(long long tokens);
hipError_t launch_rotary_forward(const RotaryArgs& a, int d, int dtype, int interleaved, hipStream_t stream);
hipError_t launch_rotary_backward(const RotaryArgs& a, int d, int dtype, int interleaved, void* dq_weight,
                                  void* dk_weight, hipStream_t stream);

// The cache as the kernels take it.
struct CacheArgs {
  char* data;
  long long head_bytes;                   // of one page of one head
  const int32_t* table;
  int pages, Hkv, page_log2, max_pages;
  int cap;                                // max_pages << page_log2
};

struct CacheRowsArgs {
  CacheArgs c;
  Rows k, v;
  int B, n;
  const int32_t *starts, *counts;
};

// Workgroups of one head: tiles of tokens that n neighbouring ones can touch.
int cache_row_tiles(int n);
hipError_t launch_cache_write(const CacheRowsArgs& a, int d, int dtype, hipStream_t stream);
hipError_t launch_cache_read(const CacheRowsArgs& a, int d, int dtype, hipStream_t stream);

struct CacheAttentionArgs {
  CacheArgs c;
  Rows q, out;
  int B, H, group, nq, causal;
  float scale_log2;
  const int32_t *lengths, *q_start;
  float* lse;
};

// Row tiles per key head, and the workgroups that share the keys of one.
struct CachePlan {
  bool few;                               // fp4_token_kernel
  int splits, mtiles;
  size_t bytes;                           // workspace (0 for one split)
};
CachePlan cache_plan(int B, int Hkv, long long rows, int cap, int d, int dtype);
hipError_t launch_cache_attention(const CacheAttentionArgs& a, int d, int dtype, const CachePlan& plan, void* ws,
                                  hipStream_t stream);

}  // namespace mra
