// C ABI of libmra_layer (declared in mra_layer.h): argument validation, workspace
// layout and dispatch. Every check runs before the first HIP call, so a rejected
// call has enqueued nothing.
#include "mra_layer.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "layer_kernels.h"

namespace {

thread_local int g_last_hip_error = 0;

constexpr int kMaxLen = 1 << 26;
constexpr long long kMaxRows = 1LL << 30;         // row indices, rounded up to a tile, are 32-bit integers
constexpr long long kMaxGroups = (1LL << 32) / 256 - 1;   // a launch has below 2^32 threads per dimension, 256 a workgroup
constexpr int64_t kMaxRowStride = 1 << 25;        // bytes
constexpr int kMaxHeads = 1 << 16;

#define MRA_TRY(expr)                 \
  do {                                \
    const mra_status_t st_ = (expr);  \
    if (st_ != MRA_OK) return st_;    \
  } while (0)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

mra_status_t hip_status(hipError_t e) {
  if (e == hipSuccess) return MRA_OK;
  g_last_hip_error = (int)e;
  return MRA_ERR_HIP;
}

mra_status_t check_dtype(mra_dtype_t dt) { return (dt == MRA_F32 || dt == MRA_BF16) ? MRA_OK : MRA_ERR_UNSUPPORTED; }

bool known_width(int d) { return d == 32 || d == 64 || d == 128; }

mra_status_t check_tensor(const mra_strided_t* t, mra_dtype_t dt) {
  if (t == nullptr || t->data == nullptr) return MRA_ERR_INVALID_ARG;
  if (t->stride_b < 0 || t->stride_h < 0 || t->stride_n < 0) return MRA_ERR_INVALID_ARG;
  if (!aligned16(t->data)) return MRA_ERR_MISALIGNED;
  const int64_t per = dt == MRA_BF16 ? 8 : 4;
  if (t->stride_b % per || t->stride_h % per || t->stride_n % per) return MRA_ERR_MISALIGNED;
  return t->stride_n < kMaxRowStride / (16 / per) ? MRA_OK : MRA_ERR_UNSUPPORTED;
}

mra::Rows rows_of(const mra_strided_t* t, mra_dtype_t dt) {
  const long long e = dt == MRA_BF16 ? 2 : 4;
  return {static_cast<char*>(t->data), t->stride_b * e, t->stride_h * e, t->stride_n * e};
}

mra_status_t check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return MRA_OK;
  if (ws == nullptr) return MRA_ERR_INVALID_ARG;
  if (!aligned16(ws)) return MRA_ERR_MISALIGNED;
  return have < need ? MRA_ERR_WORKSPACE : MRA_OK;
}

// ---- rotary positions and head norms

mra_status_t check_rotary(const mra_rotary_problem_t* p) {
  if (p == nullptr) return MRA_ERR_INVALID_ARG;
  if (p->B < 0 || p->H < 0 || p->H_kv < 0 || p->n < 0 || p->d <= 0 || p->rot < 0) return MRA_ERR_INVALID_ARG;
  if (p->interleaved != 0 && p->interleaved != 1) return MRA_ERR_INVALID_ARG;
  if (!std::isfinite(p->magnitude)) return MRA_ERR_INVALID_ARG;
  if (!known_width(p->d)) return MRA_ERR_UNSUPPORTED;
  if (p->rot > p->d) return MRA_ERR_INVALID_ARG;
  if (p->rot % 16) return MRA_ERR_UNSUPPORTED;
  MRA_TRY(check_dtype(p->dtype));
  if (p->q_weight != nullptr || p->k_weight != nullptr) {
    MRA_TRY(check_dtype(p->weight_dtype));
    if (!(p->eps > 0.0f) || !std::isfinite(p->eps)) return MRA_ERR_INVALID_ARG;
  }
  if (p->positions != nullptr && p->positions_stride < 0) return MRA_ERR_INVALID_ARG;
  if (p->n > kMaxLen || p->H > kMaxHeads || p->H_kv > kMaxHeads) return MRA_ERR_UNSUPPORTED;
  // a workgroup for 8 tokens, where they are many
  if ((long long)p->B * p->n > 8 * kMaxGroups) return MRA_ERR_UNSUPPORTED;
  return MRA_OK;
}

bool rotary_side(const mra_rotary_problem_t& p, int heads) { return p.B > 0 && p.n > 0 && heads > 0; }

mra::RotaryArgs rotary_args(const mra_rotary_problem_t& p) {
  mra::RotaryArgs a{};
  a.n = p.n;
  a.rot = p.rot;
  a.tokens = (long long)p.B * p.n;
  a.freqs = p.freqs;
  a.positions = p.positions;
  a.positions_stride = p.positions_stride;
  a.magnitude = p.magnitude;
  a.eps = p.eps;
  a.weight_bf16 = p.weight_dtype == MRA_BF16;
  a.side[0].w = p.q_weight;
  a.side[1].w = p.k_weight;
  return a;
}

// Rows of one side are taken as they lie: `t` is what its loads go by. (Single tokens, whose stride is 0, are taken head by
// head over the batches.)
void order(mra::RotarySide& s, const mra::Rows& t, int heads) {
  s.heads = heads;
  s.head_fast = t.sh < t.sn;
}

// ---- the cache

int log2_of(int x) {
  int l = 0;
  while ((1 << l) < x) ++l;
  return l;
}

bool known_page(int size) { return size >= 32 && size <= 1024 && (size & (size - 1)) == 0; }

mra_status_t check_cache(const mra_fp4_cache_t* c) {
  if (c == nullptr) return MRA_ERR_INVALID_ARG;
  if (c->pages < 0 || c->H_kv < 0 || c->B < 0 || c->max_pages < 0 || c->d <= 0 || c->page_size <= 0)
    return MRA_ERR_INVALID_ARG;
  if (!known_width(c->d) || !known_page(c->page_size) || c->H_kv > kMaxHeads) return MRA_ERR_UNSUPPORTED;
  return (long long)c->max_pages * c->page_size <= kMaxLen ? MRA_OK : MRA_ERR_UNSUPPORTED;
}

// What a call that reaches into the cache needs of it.
mra_status_t check_cache_memory(const mra_fp4_cache_t* c) {
  if (c->pages > 0 && c->data == nullptr) return MRA_ERR_INVALID_ARG;
  if (c->max_pages > 0 && c->table == nullptr) return MRA_ERR_INVALID_ARG;
  return aligned16(c->data) ? MRA_OK : MRA_ERR_MISALIGNED;
}

mra::CacheArgs cache_args(const mra_fp4_cache_t& c) {
  mra::CacheArgs a{};
  a.data = static_cast<char*>(c.data);
  a.head_bytes = (long long)mra_fp4_page_bytes(c.page_size, c.d);
  a.table = c.table;
  a.pages = c.pages;
  a.Hkv = c.H_kv;
  a.page_log2 = log2_of(c.page_size);
  a.max_pages = c.max_pages;
  a.cap = c.max_pages * c.page_size;
  return a;
}

// A write (`read` false) or a read.
mra_status_t cache_rows(const mra_fp4_cache_t* cache, const mra_strided_t* k, const mra_strided_t* v, int n,
                        mra_dtype_t dtype, const int32_t* starts, const int32_t* counts, void* stream, bool read) {
  MRA_TRY(check_cache(cache));
  MRA_TRY(check_dtype(dtype));
  if (n < 0) return MRA_ERR_INVALID_ARG;
  if (n > kMaxLen) return MRA_ERR_UNSUPPORTED;
  if ((long long)cache->B * cache->H_kv > kMaxGroups / mra::cache_row_tiles(n)) return MRA_ERR_UNSUPPORTED;
  if (cache->B == 0 || cache->H_kv == 0 || n == 0) return MRA_OK;
  if (!read && (cache->pages == 0 || cache->max_pages == 0)) return MRA_OK;
  MRA_TRY(check_cache_memory(cache));
  MRA_TRY(check_tensor(k, dtype));
  MRA_TRY(check_tensor(v, dtype));
  mra::CacheRowsArgs a{cache_args(*cache), rows_of(k, dtype), rows_of(v, dtype), cache->B, n, starts, counts};
  auto launch = read ? mra::launch_cache_read : mra::launch_cache_write;
  return hip_status(launch(a, cache->d, (int)dtype, static_cast<hipStream_t>(stream)));
}

mra_status_t check_attention(const mra_fp4_cache_t* c, const mra_fp4_attention_t* p) {
  MRA_TRY(check_cache(c));
  if (p == nullptr) return MRA_ERR_INVALID_ARG;
  if (p->H < 0 || p->n_q < 0) return MRA_ERR_INVALID_ARG;
  if (p->H > 0 && (c->H_kv == 0 || p->H % c->H_kv != 0)) return MRA_ERR_INVALID_ARG;
  if (p->H == 0 && c->H_kv != 0) return MRA_ERR_INVALID_ARG;
  if (!(p->scale >= 0x1p-64f && p->scale <= 0x1p64f)) return MRA_ERR_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return MRA_ERR_INVALID_ARG;
  MRA_TRY(check_dtype(p->dtype));
  if (p->n_q > kMaxLen || p->H > kMaxHeads) return MRA_ERR_UNSUPPORTED;
  const long long heads = (long long)c->B * p->H;
  if (p->n_q > 0 && heads > kMaxRows / p->n_q) return MRA_ERR_UNSUPPORTED;
  return MRA_OK;
}

bool no_rows(const mra_fp4_cache_t& c, const mra_fp4_attention_t& p) { return c.B == 0 || p.H == 0 || p.n_q == 0; }

mra::CachePlan attention_plan(const mra_fp4_cache_t& c, const mra_fp4_attention_t& p) {
  return mra::cache_plan(c.B, c.H_kv, (long long)p.n_q * (p.H / c.H_kv), c.max_pages * c.page_size, c.d,
                         (int)p.dtype);
}

// Workgroups have up to 512 threads. (The join has fewer: splits are several only below two workgroups a CU.)
mra_status_t check_attention_grid(const mra_fp4_cache_t& c, const mra::CachePlan& plan) {
  return (long long)c.B * c.H_kv * plan.mtiles <= kMaxGroups / 2 / plan.splits ? MRA_OK : MRA_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

mra_status_t mra_rotary_forward(const mra_rotary_problem_t* p, const mra_strided_t* q, const mra_strided_t* k,
                                const mra_strided_t* q_out, const mra_strided_t* k_out, void* stream) {
  MRA_TRY(check_rotary(p));
  mra::RotaryArgs a = rotary_args(*p);
  const mra_strided_t *in[2] = {q, k}, *out[2] = {q_out, k_out};
  const int heads[2] = {p->H, p->H_kv};
  bool some = false;
  for (int x = 0; x < 2; ++x) {
    if (!rotary_side(*p, heads[x])) continue;
    some = true;
    MRA_TRY(check_tensor(in[x], p->dtype));
    MRA_TRY(check_tensor(out[x], p->dtype));
    a.side[x].x = rows_of(in[x], p->dtype);
    a.side[x].y = rows_of(out[x], p->dtype);
    order(a.side[x], a.side[x].x, heads[x]);
  }
  if (!some) return MRA_OK;
  if (p->rot > 0 && p->freqs == nullptr) return MRA_ERR_INVALID_ARG;
  return hip_status(mra::launch_rotary_forward(a, p->d, (int)p->dtype, p->interleaved, static_cast<hipStream_t>(stream)));
}

size_t mra_rotary_backward_workspace_bytes(const mra_rotary_problem_t* p) {
  if (check_rotary(p) != MRA_OK || (p->q_weight == nullptr && p->k_weight == nullptr)) return 0;
  const long long tokens = (long long)p->B * p->n;
  return tokens == 0 ? 0 : (size_t)mra::rotary_backward_groups(tokens) * 2 * p->d * sizeof(float);
}

mra_status_t mra_rotary_backward(const mra_rotary_problem_t* p, const mra_strided_t* q, const mra_strided_t* k,
                                 const mra_strided_t* dq_out, const mra_strided_t* dk_out, const mra_strided_t* dq,
                                 const mra_strided_t* dk, void* dq_weight, void* dk_weight, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  MRA_TRY(check_rotary(p));
  if ((dq_weight != nullptr && p->q_weight == nullptr) || (dk_weight != nullptr && p->k_weight == nullptr))
    return MRA_ERR_INVALID_ARG;
  if (!aligned16(dq_weight) || !aligned16(dk_weight)) return MRA_ERR_MISALIGNED;
  mra::RotaryArgs a = rotary_args(*p);
  const mra_strided_t *in[2] = {q, k}, *g[2] = {dq_out, dk_out}, *out[2] = {dq, dk};
  const int heads[2] = {p->H, p->H_kv};
  bool some = false;
  for (int x = 0; x < 2; ++x) {
    if (!rotary_side(*p, heads[x])) continue;
    some = true;
    if (a.side[x].w != nullptr) {
      MRA_TRY(check_tensor(in[x], p->dtype));
      a.side[x].x = rows_of(in[x], p->dtype);
    }
    MRA_TRY(check_tensor(g[x], p->dtype));
    MRA_TRY(check_tensor(out[x], p->dtype));
    a.side[x].g = rows_of(g[x], p->dtype);
    a.side[x].y = rows_of(out[x], p->dtype);
    order(a.side[x], a.side[x].g, heads[x]);
  }
  if (some && p->rot > 0 && p->freqs == nullptr) return MRA_ERR_INVALID_ARG;
  const bool weights = dq_weight != nullptr || dk_weight != nullptr;
  if (!some && !weights) return MRA_OK;
  if (weights && some) {
    MRA_TRY(check_workspace(workspace, workspace_bytes, mra_rotary_backward_workspace_bytes(p)));
    a.part = static_cast<float*>(workspace);
  }
  if (!some) a.tokens = 0;
  return hip_status(mra::launch_rotary_backward(a, p->d, (int)p->dtype, p->interleaved, dq_weight, dk_weight,
                                                static_cast<hipStream_t>(stream)));
}

size_t mra_fp4_page_bytes(int page_size, int d) {
  return known_page(page_size) && known_width(d) ? (size_t)page_size * (d + d / 16) : 0;
}

mra_status_t mra_fp4_cache_write(const mra_fp4_cache_t* cache, const mra_strided_t* k, const mra_strided_t* v, int n,
                                 mra_dtype_t dtype, const int32_t* starts, const int32_t* counts, void* stream) {
  return cache_rows(cache, k, v, n, dtype, starts, counts, stream, false);
}

mra_status_t mra_fp4_cache_read(const mra_fp4_cache_t* cache, const mra_strided_t* k_out, const mra_strided_t* v_out,
                                int n, mra_dtype_t dtype, const int32_t* starts, const int32_t* counts, void* stream) {
  return cache_rows(cache, k_out, v_out, n, dtype, starts, counts, stream, true);
}

size_t mra_fp4_attention_workspace_bytes(const mra_fp4_cache_t* cache, const mra_fp4_attention_t* p) {
  if (check_attention(cache, p) != MRA_OK || no_rows(*cache, *p)) return 0;
  const mra::CachePlan plan = attention_plan(*cache, *p);
  return check_attention_grid(*cache, plan) == MRA_OK ? plan.bytes : 0;
}

mra_status_t mra_fp4_attention(const mra_fp4_cache_t* cache, const mra_fp4_attention_t* p, const mra_strided_t* q,
                               const mra_strided_t* out, float* lse_out, void* workspace, size_t workspace_bytes,
                               void* stream) {
  MRA_TRY(check_attention(cache, p));
  if (no_rows(*cache, *p)) return MRA_OK;
  const mra::CachePlan plan = attention_plan(*cache, *p);
  MRA_TRY(check_attention_grid(*cache, plan));
  if (p->lengths == nullptr) return MRA_ERR_INVALID_ARG;
  MRA_TRY(check_cache_memory(cache));
  MRA_TRY(check_tensor(q, p->dtype));
  MRA_TRY(check_tensor(out, p->dtype));
  if (lse_out != nullptr && !aligned16(lse_out)) return MRA_ERR_MISALIGNED;
  MRA_TRY(check_workspace(workspace, workspace_bytes, plan.bytes));
  mra::CacheAttentionArgs a{};
  a.c = cache_args(*cache);
  a.q = rows_of(q, p->dtype);
  a.out = rows_of(out, p->dtype);
  a.B = cache->B;
  a.H = p->H;
  a.group = p->H / cache->H_kv;
  a.nq = p->n_q;
  a.causal = p->causal;
  a.scale_log2 = (float)((double)p->scale * 1.4426950408889634);
  a.lengths = p->lengths;
  a.q_start = p->q_start;
  a.lse = lse_out;
  return hip_status(mra::launch_cache_attention(a, cache->d, (int)p->dtype, plan, workspace, static_cast<hipStream_t>(stream)));
}

int mra_layer_last_hip_error(void) { return g_last_hip_error; }

}  // extern "C"
