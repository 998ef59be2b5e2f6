// The running softmax of a wave's query rows, and the sum of partial rows, shared by the
// forward kernels of exact attention and of attention over the 4-bit cache.
#pragma once

#include "exact_tile.h"

namespace mra {

// Reference of a query's weights exp2(S - ref) (log2 units), as in tile.hip: any
// works that keeps weights and sums finite. It is the max of the first tile that
// has a key plus kMargin. A tile whose weights sum to more than kCap in some lane
// moves the references of its queries to its own max plus kMargin and forms its
// weights again, so an ordinary tile has no max, no exchange between lanes and no
// rescaling. No weight exceeds 1, so the accumulators overflow only where the sum of |v|
// does, and the largest weight of a query stays above 2^-(kMargin + 1).
constexpr float kMargin = 16.0f;
constexpr float kCap = 1.0f;

template <int NP, int D>
struct FwdRow {
  static constexpr int NT = D / 32, KC = D / 16;
  u32x4 qf[NP][KC];
  f32x16 o[NT];
  float ref, sum;

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = splat16(0.0f);
    ref = -INFINITY;
    sum = 0.0f;
  }

  // weights exp2(s mul + c) and their sum (bfloat16: of the rounded weights)
  __device__ __forceinline__ float weights(const f32x16& s, float mul, float c, Packed<NP>& w) const {
    float p[16], t = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, c));
    w = pack_weights<NP>(p);
    if constexpr (NP == 1) {
      const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          t = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)w.w[0][u][e]), ones, t, false);
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) t += p[r];
    }
    return t;
  }

  // Moves the reference to this tile's max, if that is larger.
  __device__ __forceinline__ void move(const f32x16& s, float mul, float add) {
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = __builtin_elementwise_maximum(mx, s[r]);
    mx = fmaf(halves_max(mx), mul, add);
    const float next = mx > ref ? mx + kMargin : ref;
    const float f = next == ref ? 1.0f : __builtin_amdgcn_exp2f(ref - next);
#pragma unroll
    for (int x = 0; x < NT; ++x) o[x] *= f;
    sum *= f;
    ref = next;
  }
};

// Weights of the scores s of R tiles of as many rows (log2 logits s mul + add; -inf:
// does not count) and their sums; references that a tile outgrows are moved. The
// second turn of the loop, not a branch, forms the weights again: with a branch the
// accumulators were copied to other registers and back on every tile.
template <int NP, int D, int R>
__device__ __forceinline__ void tile_weights(FwdRow<NP, D> (&row)[R], const f32x16 (&s)[R], const float (&mul)[R],
                                             const float (&add)[R], Packed<NP> (&w)[R]) {
  float t[R];
  bool again = false;
  while (true) {
    bool fits = true;
#pragma unroll
    for (int x = 0; x < R; ++x) {
      // moved and still without a key: every s or the bias is -inf
      t[x] = row[x].weights(s[x], mul[x], again && row[x].ref == -INFINITY ? add[x] : add[x] - row[x].ref, w[x]);
      fits = fits && t[x] <= kCap;                 // not so for a query's first tile (ref -inf)
    }
    if (again || __ballot(!fits) == 0) break;
#pragma unroll
    for (int x = 0; x < R; ++x) row[x].move(s[x], mul[x], add[x]);
    again = true;
  }
#pragma unroll
  for (int x = 0; x < R; ++x) row[x].sum += t[x];
}

namespace {                                        // each library has a kernel of its own, also in a program that links both

// Adds the partial rows of `splits` workgroups. D / 4 threads go across a row's columns
// and `groups` (a power of two) across its splits, at most eight for a thread; the
// groups' sums are added in their order. Rows of few splits share a workgroup (6144 rows of
// 2 splits: 4.1 us, 9.2 with a workgroup each).
constexpr int kJoin = 8;
template <int NP, int D>
__global__ __launch_bounds__(256) void exact_join_kernel(ExactArgs a, float* __restrict__ lse, int splits, int groups,
                                                         const float* __restrict__ part_o,
                                                         const float* __restrict__ part_l) {
  constexpr int L = D / 4;
  __shared__ __attribute__((aligned(16))) f32x4 zs[256];
  __shared__ float tops[256], ls[256];
  const int rows = a.nq * a.group, tid = threadIdx.x, c = tid % L, grp = tid / L % groups;
  const long long all = (long long)a.B * a.Hkv * rows;
  const long long row = (long long)blockIdx.x * (256 / (L * groups)) + tid / (L * groups), pr = min(row, all - 1);
  f32x4 o[kJoin];
  float ref[kJoin], l[kJoin];
#pragma unroll
  for (int x = 0; x < kJoin; ++x) {
    const int s = grp + x * groups;
    const long long at = (s < splits ? s : 0) * all + pr;
    o[x] = *reinterpret_cast<const f32x4*>(part_o + at * D + 4 * c);
    ref[x] = part_l[2 * at];
    l[x] = part_l[2 * at + 1];
    if (s >= splits) {
      ref[x] = -INFINITY;
      l[x] = 0.0f;
    }
  }
  float top = ref[0], sum = 0.0f;
#pragma unroll
  for (int x = 1; x < kJoin; ++x) top = fmaxf(top, ref[x]);
  f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [](const f32x4& o, float l, float ref, float top, f32x4& z, float& sum) {
    if (l == 0.0f) return;                         // no key (a part whose scores are NaN has no reference either)
    const float f = __builtin_amdgcn_exp2f(ref - top);
    sum = fmaf(l, f, sum);
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = fmaf(o[e], f, z[e]);
  };
#pragma unroll
  for (int x = 0; x < kJoin; ++x) add(o[x], l[x], ref[x], top, z, sum);
  if (groups > 1) {
    zs[tid] = z;
    tops[tid] = top;
    ls[tid] = sum;
    __syncthreads();
    if (grp == 0) {
      float all_top = top;
      for (int x = 1; x < groups; ++x) all_top = fmaxf(all_top, tops[tid + x * L]);
      z = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      sum = 0.0f;
      for (int x = 0; x < groups; ++x) add(zs[tid + x * L], ls[tid + x * L], tops[tid + x * L], all_top, z, sum);
      top = all_top;
    }
  }
  if (grp != 0 || row >= all) return;
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  const long long bk = pr / rows;
  const int m = (int)(pr - bk * rows), i = m / a.group, b = (int)(bk / a.Hkv);
  const int h = (int)(bk - (long long)b * a.Hkv) * a.group + (m - i * a.group);
  const float out[4] = {z[0] * inv, z[1] * inv, z[2] * inv, z[3] * inv};
  store4<NP>(a.out.p + b * a.out.sb + h * a.out.sh + i * a.out.sn + 4 * c * (NP == 1 ? 2 : 4), out);
  if (lse != nullptr && c == 0)
    lse[((long long)b * a.H + h) * a.nq + i] = sum == 0.0f ? -INFINITY : (log2f(sum) + top) * kLn2;
}

// Enqueues the join of `splits` partial rows (at most 64).
template <int NP, int D>
inline void launch_join(const ExactArgs& a, float* lse, int splits, const float* part_o, const float* part_l,
                        hipStream_t stream) {
  const long long rows = (long long)a.B * a.Hkv * a.nq * a.group;
  int groups = 1;                                  // at most 64 splits: at most eight, of at most 32 threads
  while (groups * kJoin < splits) groups *= 2;
  const int per = 256 / (D / 4 * groups);
  exact_join_kernel<NP, D><<<(unsigned)((rows + per - 1) / per), 256, 0, stream>>>(a, lse, splits, groups, part_o, part_l);
}

}  // namespace

}  // namespace mra
