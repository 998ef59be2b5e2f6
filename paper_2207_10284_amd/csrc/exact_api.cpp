// C ABI of libmra_exact (declared in mra_exact.h): argument validation, workspace
// layout and dispatch. Every check runs before the first HIP call, so a rejected
// call has enqueued nothing.
#include "mra_exact.h"

#include <hip/hip_runtime.h>

#include <cstdint>

#include "exact_kernels.h"

namespace {

thread_local int g_last_hip_error = 0;

constexpr int kMaxLen = 1 << 26;
constexpr long long kMaxIndex = 2147483647LL;     // block and row indices are 32-bit integers
constexpr long long kMaxGroups = (1LL << 32) / 256 - 1;   // a launch has below 2^32 threads per dimension, 256 a workgroup
constexpr int64_t kMaxRowStride = 1 << 25;        // bytes: 64 rows within 32 bits

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

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

mra_status_t check_problem(const mra_exact_problem_t* p) {
  if (p == nullptr) return MRA_ERR_INVALID_ARG;
  if (p->B < 0 || p->H < 0 || p->H_kv < 0 || p->n_q < 0 || p->n_k < 0 || p->d <= 0) return MRA_ERR_INVALID_ARG;
  if (p->H > 0 && (p->H_kv == 0 || p->H % p->H_kv != 0)) return MRA_ERR_INVALID_ARG;
  if (p->H == 0 && p->H_kv != 0) return MRA_ERR_INVALID_ARG;
  if (!(p->scale >= 0x1p-64f && p->scale <= 0x1p64f)) return MRA_ERR_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return MRA_ERR_INVALID_ARG;
  if (p->d != 32 && p->d != 64 && p->d != 128) return MRA_ERR_UNSUPPORTED;
  if (p->n_q > kMaxLen || p->n_k > kMaxLen) return MRA_ERR_UNSUPPORTED;
  MRA_TRY(check_dtype(p->dtype));
  if (p->key_mask != nullptr && p->key_mask_stride < 0) return MRA_ERR_INVALID_ARG;
  if (p->bias != nullptr) {
    MRA_TRY(check_dtype(p->bias_dtype));
    if (p->buckets < 1 || p->far < 0 || p->bucket_map == nullptr) return MRA_ERR_INVALID_ARG;
    if (p->buckets > MRA_EXACT_MAX_BUCKETS || p->far > MRA_EXACT_MAX_FAR) return MRA_ERR_UNSUPPORTED;
  }
  // blocks of 128 rows of all heads, and rows
  const long long longest = p->n_q > p->n_k ? p->n_q : p->n_k;
  const long long heads = (long long)p->B * p->H, blocks = (longest + 127) / 128;
  if (blocks > 0 && heads > kMaxIndex / blocks) return MRA_ERR_UNSUPPORTED;
  const long long rows = heads * p->n_q;
  if (rows > kMaxIndex) return MRA_ERR_UNSUPPORTED;
  return MRA_OK;
}

bool empty(const mra_exact_problem_t& p) { return p.B == 0 || p.H == 0 || p.n_q == 0; }

// Whether every launch of a call fits; those not named have fewer workgroups (the join: splits are
// several only below two workgroups a CU; the parts' sums: only where a pass has at most eight).
mra_status_t check_forward_grid(const mra_exact_problem_t& p, const mra::SplitPlan& plan) {
  const long long groups = plan.use ? (long long)p.B * p.H_kv * plan.mtiles * plan.splits
                                    : (long long)p.B * p.H * ((p.n_q + 127) / 128);
  return groups <= kMaxGroups ? MRA_OK : MRA_ERR_UNSUPPORTED;
}

mra_status_t check_backward_grid(const mra_exact_problem_t& p) {
  const long long dq = (long long)p.B * p.H * mra::exact_dq_blocks(p.n_q), dkv = (long long)p.B * p.H_kv * mra::exact_dq_blocks(p.n_k);
  const long long bias = p.bias != nullptr ? p.H : 0;
  return dq <= kMaxGroups && dkv <= kMaxGroups && bias <= kMaxGroups ? MRA_OK : MRA_ERR_UNSUPPORTED;
}

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

mra::ExactArgs args_of(const mra_exact_problem_t& p) {
  mra::ExactArgs a{};
  a.B = p.B;
  a.H = p.H;
  a.Hkv = p.H_kv;
  a.group = p.H_kv > 0 ? p.H / p.H_kv : 1;
  a.nq = p.n_q;
  a.nk = p.n_k;
  a.causal = p.causal;
  a.scale = p.scale;
  a.scale_log2 = (float)((double)p.scale * 1.4426950408889634);
  a.lengths = p.lengths;
  a.q_start = p.q_start;
  a.key_mask = p.key_mask;
  a.mask_stride = p.key_mask_stride;
  a.bias = p.bias;
  a.bias_bf16 = p.bias_dtype == MRA_BF16;
  a.buckets = p.bias != nullptr ? p.buckets : 0;
  a.far = p.bias != nullptr ? p.far : 0;
  a.map = p.bucket_map;
  return a;
}

// Workspace of the backward: delta per query, the diagonal sums (with a bias), the queries'
// sums (exact_centre_kernel), the partial sums of dq, dk and dv.
struct WsBackward {
  mra::BackwardPlan plan;
  size_t diag, rows, q, k, v, total;
};

WsBackward ws_backward(const mra_exact_problem_t& p) {
  WsBackward w{};
  w.plan = mra::exact_backward_plan(p);
  size_t off = align256((size_t)p.B * p.H * p.n_q * sizeof(float));
  w.diag = off;
  if (p.bias != nullptr)
    off += align256((size_t)p.B * p.H * mra::exact_dq_blocks(p.n_q) * mra::exact_slots(w.plan) * mra::exact_window(p.far) *
                    sizeof(float));
  w.rows = off;
  if (w.plan.centre) off += align256((size_t)w.plan.dq_parts * p.B * p.H * p.n_q * 4 * sizeof(float));
  w.q = off; off += align256(w.plan.q_floats * sizeof(float));
  w.k = off; off += align256(w.plan.k_floats * sizeof(float));
  w.v = off; off += align256(w.plan.k_floats * sizeof(float));
  w.total = off;
  return w;
}

mra_status_t check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return MRA_OK;
  if (ws == nullptr) return MRA_ERR_INVALID_ARG;
  if (!aligned16(ws)) return MRA_ERR_MISALIGNED;
  return have < need ? MRA_ERR_WORKSPACE : MRA_OK;
}

}  // namespace

extern "C" {

size_t mra_exact_forward_workspace_bytes(const mra_exact_problem_t* p) {
  if (check_problem(p) != MRA_OK || empty(*p)) return 0;
  const mra::SplitPlan plan = mra::exact_split_plan(*p);
  return check_forward_grid(*p, plan) == MRA_OK ? plan.bytes : 0;
}

mra_status_t mra_exact_forward(const mra_exact_problem_t* p, const mra_strided_t* q, const mra_strided_t* k,
                               const mra_strided_t* v, const mra_strided_t* out, float* lse_out, void* workspace,
                               size_t workspace_bytes, void* stream) {
  MRA_TRY(check_problem(p));
  if (empty(*p)) return MRA_OK;
  const mra::SplitPlan plan = mra::exact_split_plan(*p);
  MRA_TRY(check_forward_grid(*p, plan));
  MRA_TRY(check_tensor(q, p->dtype));
  MRA_TRY(check_tensor(out, p->dtype));
  if (p->n_k > 0) {
    MRA_TRY(check_tensor(k, p->dtype));
    MRA_TRY(check_tensor(v, p->dtype));
  }
  if (lse_out != nullptr && !aligned16(lse_out)) return MRA_ERR_MISALIGNED;
  MRA_TRY(check_workspace(workspace, workspace_bytes, plan.bytes));
  mra::ExactArgs a = args_of(*p);
  a.q = rows_of(q, p->dtype);
  a.out = rows_of(out, p->dtype);
  if (p->n_k > 0) {
    a.k = rows_of(k, p->dtype);
    a.v = rows_of(v, p->dtype);
  }
  return hip_status(mra::launch_exact_forward(a, p->d, (int)p->dtype, lse_out, plan, workspace,
                                              static_cast<hipStream_t>(stream)));
}

size_t mra_exact_backward_workspace_bytes(const mra_exact_problem_t* p) {
  if (check_problem(p) != MRA_OK || check_backward_grid(*p) != MRA_OK || empty(*p)) return 0;
  return ws_backward(*p).total;
}

mra_status_t mra_exact_backward(const mra_exact_problem_t* p, const mra_strided_t* q, const mra_strided_t* k,
                                const mra_strided_t* v, const mra_strided_t* out, const mra_strided_t* dout,
                                const float* lse, const mra_strided_t* dq, const mra_strided_t* dk,
                                const mra_strided_t* dv, void* dbias, void* workspace, size_t workspace_bytes,
                                void* stream) {
  MRA_TRY(check_problem(p));
  MRA_TRY(check_backward_grid(*p));
  if (dbias != nullptr && p->bias == nullptr) return MRA_ERR_INVALID_ARG;
  if (dbias != nullptr && !aligned16(dbias)) return MRA_ERR_MISALIGNED;
  const bool rows = !empty(*p), keys = p->B > 0 && p->H > 0 && p->n_k > 0;
  mra::ExactArgs a = args_of(*p);
  mra::ExactGrads g{};
  if (rows) {
    for (const mra_strided_t* t : {q, out, dout, dq}) MRA_TRY(check_tensor(t, p->dtype));
    if (lse == nullptr) return MRA_ERR_INVALID_ARG;
    if (!aligned16(lse)) return MRA_ERR_MISALIGNED;
    a.q = rows_of(q, p->dtype);
    a.out = rows_of(out, p->dtype);
    g.dout = rows_of(dout, p->dtype);
    g.dq = rows_of(dq, p->dtype);
    g.lse = lse;
  }
  if (keys) {
    for (const mra_strided_t* t : {k, v, dk, dv}) MRA_TRY(check_tensor(t, p->dtype));
    a.k = rows_of(k, p->dtype);
    a.v = rows_of(v, p->dtype);
    g.dk = rows_of(dk, p->dtype);
    g.dv = rows_of(dv, p->dtype);
  }
  mra::BackwardPlan plan{1, 1, false, 0, 0};
  if (rows) {
    const WsBackward w = ws_backward(*p);
    MRA_TRY(check_workspace(workspace, workspace_bytes, w.total));
    plan = w.plan;
    auto at = [&](size_t off) { return reinterpret_cast<float*>(static_cast<char*>(workspace) + off); };
    g.delta = at(0);
    if (dbias != nullptr) {
      g.diag = at(w.diag);
      g.slots = mra::exact_slots(plan);
      if (plan.centre) g.row_sums = at(w.rows);
    }
    g.part_q = at(w.q);
    g.part_k = at(w.k);
    g.part_v = at(w.v);
  }
  g.dbias = dbias;
  if (!rows && !keys && (dbias == nullptr || p->H == 0)) return MRA_OK;
  return hip_status(mra::launch_exact_backward(a, g, plan, p->d, (int)p->dtype, static_cast<hipStream_t>(stream)));
}

int mra_exact_last_hip_error(void) { return g_last_hip_error; }

}  // extern "C"
