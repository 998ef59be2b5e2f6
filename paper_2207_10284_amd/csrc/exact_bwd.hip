// Gradients of exact softmax attention (mra_exact.h). The probabilities are formed
// again from the forward's log normalisers, P_ij = exp(S_ij - L_i), in two passes that
// each own what they sum, so no sum depends on the order of workgroups:
//
// exact_dq_kernel: a wave owns 32 queries of one head and walks the keys:
//   delta_i = G_i . Z_i (also written for the second pass), D_ij = P_ij (G_i . v_j - delta_i),
//   dQ_i = scale sum_j D_ij k_j; with a position bias the sums of D over the diagonals.
//   S^T = K Q^T and V G^T leave a lane 16 keys of one query, the B operand of
//   dQ^T += K^T D^T.
// exact_dkv_kernel: a wave owns 32 keys of one key head and walks the queries of its
//   heads: S = Q K^T and G V^T leave a lane 16 queries of one key, the B operands of
//   dV^T += G^T P and dK^T += Q^T D.
// S and dP are formed in both: seven products instead of five, but no atomic sums
// and no partial dQ of n_k / 32 times the size. Where a pass has few blocks, several
// workgroups share each and exact_sum_kernel adds their sums.
//
// exact_centre_kernel: bfloat16 over many keys, takes from dbias what roundings of Z leave in D.
//
// exact_bias_kernel: the diagonal sums of a head's blocks, added by bucket in a fixed
// order.
#include "exact_tile.h"

namespace mra {

constexpr int kDqRows = kExactWaves * 32;
// floats of a wave's skewed tile (32 rows of 64: see exact_dq_kernel)
constexpr int kSkew = 32 * 64;
// D of the tiles beyond the bias window, per wave: a double each below and above it. A lane's float32 sums
// go there every kFarStages stages: over a query's keys D cancels, and one float32 sum over
// 10^5 keys would keep roundings of the sums on the way (dbias, 64 queries x 150000 keys x 64 float32: 3.3e-5 ->
// 2.3e-5 in 2-norm; 2^20 keys whose D rise and fall: 39% -> 5e-6). Doubles in the lanes' registers
// instead would spill (32 heads x 2048 x 128 bfloat16, training: 391 -> 425 us).
constexpr int kFarStages = 16;
constexpr size_t kFarBytes = kExactWaves * 2 * sizeof(double);

// Adds the 16 numbers of a lane (row lane % 32 a query, 16 of its keys) of a 32 x 32 tile to a wave's
// diagonal sums, `at` those of the tile's 63: row query, column key - query + 31 of the skewed tile,
// so the diagonals are columns, a lane each.
__device__ __forceinline__ void add_diagonals(float* skew, const float (&x)[16], float* at) {
  const int lane = lane_id();
  float* to = skew + 63 * (lane & 31) + 31 + 4 * (lane >> 5);
#pragma unroll
  for (int r = 0; r < 16; ++r) to[reg_row(r)] = x[r];
  wave_lds_sync();
  float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int q = 0; q < 32; ++q) t[q & 3] += skew[64 * q + lane];
  at[lane] += (t[0] + t[1]) + (t[2] + t[3]);
  wave_lds_sync();
}

int exact_dq_blocks(int nq) { return (nq + kDqRows - 1) / kDqRows; }
// the window's entries, then the sums of the tiles below and above it
int exact_window(int far) { return window_entries(far) + 2; }

// bfloat16, D = 128: registers for two waves a SIMD (shorter stages, addresses and operand
// chunks one at a time, delta subtracted by the vector ALU) rather than one with all in
// flight: 16 heads x 16384 x 128 causal: 1.99 -> 1.52 ms
template <int NP, int D>
constexpr bool kDqTwo = NP == 1 && D == 128;
template <int NP, int D>
constexpr int kDqStageRows = kDqTwo<NP, D> ? 32 : kStageRows<NP, D>;

// A workgroup's diagonal sums, those of its waves added in their order, to slot `slot` of its block.
__device__ __forceinline__ void store_diagonals(const ExactGrads& g, long long block, int slot, int entries, const float* acc,
                                                const double* far_sums) {
  const int tid = threadIdx.x;
  float* out = g.diag + (block * g.slots + slot) * (entries + 2);
  for (int x = tid; x < entries; x += kExactThreads) {
    float t = 0.0f;
#pragma unroll
    for (int p = 0; p < kExactWaves; ++p) t += acc[p * entries + x];
    out[x] = t;
  }
  if (tid < 2) out[entries + tid] = (float)((far_sums[tid] + far_sums[2 + tid]) + (far_sums[4 + tid] + far_sums[6 + tid]));
}

// RT: 32-row tiles of queries per wave
template <int NP, int D, int RT, bool BIAS>
__global__ __launch_bounds__(kExactThreads, (kDqTwo<NP, D> || RT == 2 ? 2 : 1)) void exact_dq_kernel(ExactArgs a, ExactGrads g, int qblocks) {
  constexpr int KT = kDqStageRows<NP, D>, TILES = KT / 32, KC = D / 16, NT = D / 32;
  using St = Stage<NP, D, KT, kExactThreads>;
  constexpr int STEP = TILES * kTileBytes<D>, ROWS = kDqRows * RT;
  static_assert(RT == 1 || (!BIAS && NP == 1), "one bias, one plane");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* win = reinterpret_cast<float*>(smem + 4 * St::kBytes);
  const int entries = BIAS ? window_entries(a.far) : 0;
  float* acc = win + entries;                      // a window of diagonal sums per wave
  const int tid = threadIdx.x, lane = lane_id(), w = wave_uniform(tid / kWave), hf = lane >> 5;
  const HeadBlock hb = head_block(blockIdx.x, a.B * a.H, qblocks, a.causal);
  const int bh = hb.head, qb = qblocks - 1 - hb.block;             // causal: the longest first
  const int part = blockIdx.y, parts = gridDim.y;
  const int b = bh / a.H, h = bh - b * a.H, hk = h / a.group;
  const int row0 = qb * ROWS + w * 32 * RT, i0 = row0 + (lane & 31);      // this lane's query of tile y: i0 + 32 y
  const int limit = key_limit(a, b), start = first_position(a, b);
  const int kend = a.causal ? min(limit, start + min((qb + 1) * ROWS, a.nq)) : limit;
  const int all_stages = kend > 0 ? (kend + KT - 1) / KT : 0;
  // this workgroup's part of them
  const int begin = parts == 1 ? 0 : (int)((long long)all_stages * part / parts);
  const int stages = parts == 1 ? all_stages : (int)((long long)all_stages * (part + 1) / parts);
  const char* kp = a.k.p + b * a.k.sb + hk * a.k.sh;
  const char* vp = a.v.p + b * a.v.sb + hk * a.v.sh;
  const int pos0 = start + row0;

  TileAddr<D, kDqTwo<NP, D>> at;
  at.init(smem);
  u32x4 qf[RT][NP][KC], gf[RT][NP][KC];
  f32x16 dq[RT][NT];
  float delta[RT], nl[RT];
#pragma unroll
  for (int y = 0; y < RT; ++y) {
    const int i = i0 + 32 * y, ic = min(i, a.nq - 1);
#pragma unroll
    for (int t = 0; t < NT; ++t) dq[y][t] = splat16(0.0f);
    load_operand<NP, D>(a.q.p + b * a.q.sb + h * a.q.sh + ic * a.q.sn, i < a.nq, qf[y]);
    constexpr int LB = NP == 1 ? KC : 2 * KC;
    const int half = hf * (D / 2) * (NP == 1 ? 2 : 4);
    const u32x4* gr = reinterpret_cast<const u32x4*>(g.dout.p + b * g.dout.sb + h * g.dout.sh + ic * g.dout.sn + half);
    const u32x4* zr = reinterpret_cast<const u32x4*>(a.out.p + b * a.out.sb + h * a.out.sh + ic * a.out.sn + half);
    // of Z as stored: the rounding of a bfloat16 Z is one number for all keys of the query (dbias: see
    // exact_centre_kernel)
    float d = 0.0f;
#pragma unroll
    for (int c = 0; c < LB; ++c) {
      const u32x4 u = gr[c], v = zr[c];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (NP == 1) {
          d = fmaf(bf16_to_f32(u[e] & 0xFFFFu), bf16_to_f32(v[e] & 0xFFFFu), d);
          d = fmaf(bf16_to_f32(u[e] >> 16), bf16_to_f32(v[e] >> 16), d);
        } else {
          d = fmaf(__uint_as_float(u[e]), __uint_as_float(v[e]), d);
        }
      }
    }
    d = halves_sum(d);
    load_operand<NP, D>(g.dout.p + b * g.dout.sb + h * g.dout.sh + ic * g.dout.sn, i < a.nq, gf[y]);
    const long long at_row = (long long)bh * a.nq + ic;
    const float L = g.lse[at_row];
    if (part == 0 && lane < 32 && i < a.nq) g.delta[at_row] = d;
    // no key counts: no weight; the same for rows past the last
    const bool none = i >= a.nq || L == -INFINITY;
    nl[y] = none ? -INFINITY : -L * kLog2e;
    delta[y] = none ? 0.0f : d;
  }
  float sum_lo = 0.0f, sum_hi = 0.0f;
  double row_d = 0.0;                              // of this lane's query and keys: D, and P below and above the window
  float row_lo = 0.0f, row_hi = 0.0f;
  float* mine = acc + w * entries;
  float* skew = acc + kExactWaves * entries + w * kSkew;
  double* far_sums = reinterpret_cast<double*>(acc + kExactWaves * (entries + kSkew));
  if constexpr (BIAS) {
    fill_window(a, h, win, tid, kExactThreads);
    for (int x = tid; x < kExactWaves * (entries + kSkew) + (int)(kFarBytes / 4); x += kExactThreads) acc[x] = 0.0f;
  }

  // this wave's sums beyond the window, to their doubles
  auto flush_far = [&]() {
    if constexpr (NP == 1) row_d += (double)sum_lo + (double)sum_hi;
    float* both[2] = {&sum_lo, &sum_hi};
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      double t = (double)*both[x];
#pragma unroll
      for (int y = 1; y < kWave; y *= 2) t += __shfl_xor(t, y);
      if (lane == 0) far_sums[2 * w + x] += t;
      *both[x] = 0.0f;
    }
  };

  // G V^T - delta. The matrix cores' additions fall a little below the exact sum (5e-8 on
  // average where the sum is about 11), and an offset common to a query's keys does not
  // vanish in the bias gradient, where the D of many queries meet, whose sums over all keys
  // are 0. With a bias, float32 takes half of the columns with the opposite sign (gf holds
  // them so) and subtracts; delta is subtracted last, so that both halves start alike. Error of
  // dbias (2-norm), 2 heads x 1503 x 128, buckets (32, 128): 5.7e-6 -> 1.3e-6.
  constexpr bool kTwoSigns = BIAS && NP == 3;
  if constexpr (kTwoSigns) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int c = KC / 2; c < KC; ++c) gf[0][p][c] ^= 0x80008000u;
  }
  auto values_product = [&](int vtile) -> f32x16 {
    if constexpr (kTwoSigns) {
      const f32x16 x = product_part<NP, D, 0, KC / 2>(at, vtile, STEP, gf[0], splat16(0.0f));
      const f32x16 y = product_part<NP, D, KC / 2, KC>(at, vtile, STEP, gf[0], splat16(0.0f));
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = (x[r] - y[r]) - delta[0];
      return z;
    } else {
      return product<NP, D>(at, vtile, STEP, gf[0], splat16(-delta[0]));
    }
  };

  St ks, vs;
  ks.init(a.k.sn, tid);
  vs.init(a.v.sn, tid);
  MaskBytes<KT> bytes;
  RowBits<KT> ok{};
  if (begin < stages) {
    ks.load(kp, a.k.sn, begin * KT, limit);
    vs.load(vp, a.v.sn, begin * KT, limit);
    bytes.load(a, b, begin * KT);
    ok = bytes.bits(begin * KT, limit);
    ks.store(smem, ok, tid);
    vs.store(smem + St::kBytes, ok, tid);
  }
  __syncthreads();
  wait_loads<0>();                                 // the operands too: no wait for them beside the loads in flight below
  constexpr bool kSub = kDqTwo<NP, D> || RT == 2;  // delta subtracted by the vector ALU: 16 registers fewer
  // K's columns read when D has been formed, for registers (32 heads x 2048 x 128 with a bias, training: 408 -> 391 us)
  constexpr bool kLate = kDqTwo<NP, D> && BIAS;
  // stage st in buffer BUF (known at compile time: its part of an LDS address is an
  // offset); PLAIN: every key counts for every query, no bias
  auto stage = [&](int st, auto BUF, auto PLAIN) {
    constexpr int cur = BUF * 2 * St::kBytes;
    const bool more = st + 1 < stages;
    if (more) {
      ks.load(kp, a.k.sn, (st + 1) * KT, limit);
      vs.load(vp, a.v.sn, (st + 1) * KT, limit);
      bytes.load(a, b, (st + 1) * KT);
    }
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
      const uint32_t kb = PLAIN ? ~0u : ok.tile(x);
      const int k0 = st * KT + 32 * x, ktile = cur + x * kTileBytes<D>, vtile = cur + St::kBytes + x * kTileBytes<D>;
      if (!PLAIN && (kb == 0 || (a.causal && k0 > pos0 + 32 * RT - 1))) continue;
      u32x4 kr[KC], vr[KC], kt[2][NT];             // one plane only
      if constexpr (NP == 1) {
        read_rows<D>(at, ktile, kr);
        if constexpr (D < 128) read_rows<D>(at, vtile, vr);
        __builtin_amdgcn_sched_barrier(0);
      }
      Packed<NP> dw[RT];
#pragma unroll
      for (int y = 0; y < RT; ++y) {
        f32x16 s, dp;
        if constexpr (NP == 1) {
          s = splat16(0.0f);
          dp = splat16(kSub ? 0.0f : -delta[y]);
          if constexpr (D < 128) {
#pragma unroll
            for (int c = 0; c < KC; ++c) {
              s = mfma16(kr[c], qf[y][0][c], s);
              dp = mfma16(vr[c], gf[y][0][c], dp);
            }
          } else {                                 // one operand's chunks at a time, for two waves a SIMD
#pragma unroll
            for (int c = 0; c < KC; ++c) s = mfma16(kr[c], qf[y][0][c], s);
            read_rows<D>(at, vtile, vr);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < KC; ++c) dp = mfma16(vr[c], gf[y][0][c], dp);
          }
          if (y == RT - 1 && !kLate) read_trans<D>(at, ktile, kt);
          if (RT == 1) __builtin_amdgcn_sched_barrier(0);
        } else {
          s = product<NP, D>(at, ktile, STEP, qf[0], splat16(0.0f));
          dp = values_product(vtile);
        }
        const int d0 = k0 - pos0 - 32 * y, at_win = d0 + a.far + kWinPad - (lane & 31) + 4 * hf;
        float mul = a.scale_log2, add = nl[y];
        BiasKind kind = kBiasNear;
        if constexpr (BIAS) {
          kind = bias_kind(d0, a.far);
          if (kind == kBiasNear) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale_log2, win[at_win + reg_row(r)]);
            mul = 1.0f;
          } else {
            add += win[kind == kBiasLow ? 0 : entries - 1];
          }
        }
        if (!PLAIN && (kb != ~0u || (a.causal && d0 + 31 > 0)))
          select_rows(s, a.causal ? kb & low_bits((lane & 31) - d0 + 1) : kb, -INFINITY);
        float p[16], ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, add));
          ds[r] = p[r] * (NP == 1 && kSub ? dp[r] - delta[y] : dp[r]);
        }
        if (BIAS && g.diag != nullptr) {
          if (kind == kBiasNear) add_diagonals(skew, ds, mine + (d0 + a.far + kWinPad - 31));
          if (kind != kBiasNear || (NP == 1 && g.row_sums != nullptr)) {
            float t = 0.0f, tp = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) t += ds[r];
            if (kind == kBiasLow) sum_lo += t;
            if (kind == kBiasHigh) sum_hi += t;
            if (NP == 1 && g.row_sums != nullptr) {
              if (kind == kBiasNear) {
                row_d += (double)t;                // of the others: flush_far
              } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) tp += p[r];
                if (kind == kBiasLow) row_lo += tp;
                else row_hi += tp;
              }
            }
          }
        }
        dw[y] = pack_weights<NP>(ds);
      }
      if constexpr (kLate) read_trans<D>(at, ktile, kt);
#pragma unroll
      for (int y = 0; y < RT; ++y) {
        if constexpr (NP == 1) accumulate_chunks<D>(kt, dw[y], dq[y]);
        else accumulate_t<NP, D>(at, ktile, STEP, dw[y], dq[y]);
      }
    }
    if (more) {
      char* nxt = smem + (1 - BUF) * 2 * St::kBytes;
      ok = bytes.bits((st + 1) * KT, limit);
      ks.store(nxt, ok, tid);
      vs.store(nxt + St::kBytes, ok, tid);
    }
    __syncthreads();
  };
  constexpr std::integral_constant<int, 0> b0{};
  constexpr std::integral_constant<int, 1> b1{};
  // the stages whose keys all count for all of the block's queries, in pairs, then the others
  int st = begin;
  if constexpr (!BIAS && NP == 1) {
    const int all = a.causal ? min(limit, start + qb * ROWS + 1) : limit;
    const int plain = a.key_mask != nullptr ? begin : min(max(all, 0) / KT, stages);
    for (; st + 1 < plain; st += 2) {
      stage(st, b0, std::true_type{});
      stage(st + 1, b1, std::true_type{});
    }
  }
  for (; st < stages; st += 2) {
    stage(st, b0, std::false_type{});
    if (st + 1 < stages) stage(st + 1, b1, std::false_type{});
    if constexpr (BIAS) {
      if ((st - begin) % kFarStages == kFarStages - 2) flush_far();
    }
  }
#pragma unroll
  for (int y = 0; y < RT; ++y) {
    const int i = i0 + 32 * y, ic = min(i, a.nq - 1);
    if (parts > 1)
      store_rows<3, D>(dq[y], a.scale,
                       reinterpret_cast<char*>(g.part_q + (((long long)part * a.B * a.H + bh) * a.nq + ic) * D), i < a.nq);
    else
      store_rows<NP, D>(dq[y], a.scale, g.dq.p + b * g.dq.sb + h * g.dq.sh + ic * g.dq.sn, i < a.nq);
  }
  if constexpr (BIAS) {
    if (g.diag == nullptr) return;
    flush_far();
    __syncthreads();
    store_diagonals(g, ((long long)h * a.B + b) * qblocks + qb, part, entries, acc, far_sums);
    if (NP == 1 && g.row_sums != nullptr) {
      const f32x4 t = {(float)(row_d + __shfl_xor(row_d, 32)), halves_sum(row_lo), halves_sum(row_hi), 0.0f};
      if (lane < 32 && i0 < a.nq)
        *reinterpret_cast<f32x4*>(g.row_sums + (((long long)part * a.B * a.H + bh) * a.nq + i0) * 4) = t;
    }
  }
}

// dbias of bfloat16 calls over many keys. Over a query's keys D sums to 0, as P does to 1: delta
// is the mean of G . v_j under P. As formed in the dQ pass, D sums to r = (that mean) - delta: delta is
// G . Z of a Z whose weights and whose result were rounded. In dQ and dK r is one rounding
// among others, but dbias sums D over many keys, which cancel, and P r stays: it grows against
// the result like the root of the keys per distance of the window. So -P r is added to dbias (not to dQ and dK,
// whose bits do not depend on whether dbias is asked for): beyond the window from each query's sums of P, which the
// dQ pass leaves with r, and for the tiles of the window by forming P again, S in one product: few tiles of a long
// row. What is left is the rounding of L, one factor a query. Error of dbias in 2-norm (float32 table): 64 queries x 20000
// keys x 64: 9.7e-3 -> 1.9e-5; 31 x 12000 x 128: 8.8e-4 -> 4.8e-5; 2100 x 2100 x 64 causal 2.9e-3 -> 3.7e-4.
template <int D>
__global__ __launch_bounds__(kExactThreads) void exact_centre_kernel(ExactArgs a, ExactGrads g, int qblocks, int parts) {
  constexpr int KT = kStageRows<1, D>, TILES = KT / 32;
  using St = Stage<1, D, KT, kExactThreads>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int entries = window_entries(a.far);
  float* win = reinterpret_cast<float*>(smem + 2 * St::kBytes);
  float* acc = win + entries;
  const int tid = threadIdx.x, lane = lane_id(), w = wave_uniform(tid / kWave);
  float* mine = acc + w * entries;
  float* skew = acc + kExactWaves * entries + w * kSkew;
  double* far_sums = reinterpret_cast<double*>(acc + kExactWaves * (entries + kSkew));
  const HeadBlock hb = head_block(blockIdx.x, a.B * a.H, qblocks, false);
  const int bh = hb.head, qb = hb.block;
  const int b = bh / a.H, h = bh - b * a.H, hk = h / a.group;
  const int row0 = qb * kDqRows + w * 32, i = row0 + (lane & 31), ic = min(i, a.nq - 1);
  const int limit = key_limit(a, b), start = first_position(a, b), pos0 = start + row0;
  const int kend = a.causal ? min(limit, start + min((qb + 1) * kDqRows, a.nq)) : limit;
  // the stages with tiles in the window of one of the block's waves, whose first queries are 32 apart
  const int p_first = start + qb * kDqRows, p_last = p_first + kDqRows - 32;
  const int begin = max(p_first - a.far - 30, 0) / KT;
  const int stages = min(max(kend, 0), max(p_last + a.far + 31, 0)) > 0
                         ? (min(kend, p_last + a.far + 31) + KT - 1) / KT : 0;
  const char* kp = a.k.p + b * a.k.sb + hk * a.k.sh;

  St ks;
  ks.init(a.k.sn, tid);
  MaskBytes<KT> bytes;
  auto load = [&](int st) {
    ks.load(kp, a.k.sn, st * KT, limit);
    bytes.load(a, b, st * KT);
  };
  if (begin < stages) load(begin);
  TileAddr<D> at;
  at.init(smem);
  u32x4 qf[1][D / 16];
  load_operand<1, D>(a.q.p + b * a.q.sb + h * a.q.sh + ic * a.q.sn, i < a.nq, qf);
  const long long at_row = (long long)bh * a.nq + ic;
  const float L = g.lse[at_row];
  const bool none = i >= a.nq || L == -INFINITY;
  const float nl = none ? -INFINITY : -L * kLog2e;
  f32x4 sums = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = 0; p < parts; ++p) {
    const f32x4 t = *reinterpret_cast<const f32x4*>(g.row_sums + ((long long)p * a.B * a.H * a.nq + at_row) * 4);
#pragma unroll
    for (int e = 0; e < 3; ++e) sums[e] += t[e];
  }
  const float r = none ? 0.0f : sums[0];
  fill_window(a, h, win, tid, kExactThreads);
  for (int x = tid; x < kExactWaves * (entries + kSkew); x += kExactThreads) acc[x] = 0.0f;
  for (int st = begin; st < stages; ++st) {
    const RowBits<KT> ok = bytes.bits(st * KT, limit);
    ks.store(smem + (st & 1) * St::kBytes, ok, tid);   // the other waves are at most a stage behind: in the other buffer
    __syncthreads();
    if (st + 1 < stages) load(st + 1);
#pragma unroll
    for (int x = 0; x < TILES; ++x) {
      const uint32_t kb = ok.tile(x);
      const int k0 = st * KT + 32 * x, d0 = k0 - pos0;
      if (kb == 0 || (a.causal && d0 > 31) || bias_kind(d0, a.far) != kBiasNear) continue;
      f32x16 s = product<1, D>(at, (st & 1) * St::kBytes + x * kTileBytes<D>, 0, qf, splat16(0.0f));
      const float* wp = win + (d0 + a.far + kWinPad - (lane & 31) + 4 * (lane >> 5));
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = fmaf(s[e], a.scale_log2, wp[reg_row(e)]);
      if (kb != ~0u || (a.causal && d0 + 31 > 0))
        select_rows(s, a.causal ? kb & low_bits((lane & 31) - d0 + 1) : kb, -INFINITY);
      float ps[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) ps[e] = -r * __builtin_amdgcn_exp2f(s[e] + nl);
      add_diagonals(skew, ps, mine + (d0 + a.far + kWinPad - 31));
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {                    // below and above the window
    double t = lane < 32 && !none ? -(double)r * (double)sums[1 + x] : 0.0;
#pragma unroll
    for (int y = 1; y < kWave; y *= 2) t += __shfl_xor(t, y);
    if (lane == 0) far_sums[2 * w + x] = t;
  }
  __syncthreads();
  store_diagonals(g, ((long long)h * a.B + b) * qblocks + qb, parts, entries, acc, far_sums);
}

template <int NP, int D, bool BIAS>
// (float32, D = 64: held to the registers of two waves a SIMD: 32 heads x 1500 x 64, training: 562 -> 538 us)
__global__ __launch_bounds__(kExactThreads, NP == 3 && D == 64 ? 2 : 1) void exact_dkv_kernel(ExactArgs a, ExactGrads g, int kblocks) {
  constexpr int QT = kStageRows<NP, D>, TILES = QT / 32, KC = D / 16, NT = D / 32;
  using St = Stage<NP, D, QT, kExactThreads>;
  constexpr int STEP = TILES * kTileBytes<D>;
  constexpr int NUMS = 4 * St::kBytes;             // [2 buffers][-L / scale, -delta][QT] chunks of 16 bytes
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* win = reinterpret_cast<float*>(smem + NUMS + 64 * QT);
  const int tid = threadIdx.x, lane = lane_id(), w = wave_uniform(tid / kWave), hf = lane >> 5;
  const HeadBlock hb = head_block(blockIdx.x, a.B * a.Hkv, kblocks, a.causal);
  const int bk = hb.head, kblk = hb.block;                         // causal: the longest first
  const int part = blockIdx.y, parts = gridDim.y;
  const int b = bk / a.Hkv, hk = bk - b * a.Hkv;
  const int block0 = kblk * kExactWaves * 32, k0 = block0 + w * 32, j = k0 + (lane & 31), jc = min(j, a.nk - 1);
  const int limit = key_limit(a, b), start = first_position(a, b);
  const bool counts = j < limit && (a.key_mask == nullptr || a.key_mask[(long long)b * a.mask_stride + jc] != 0);
  const bool any = __ballot(counts) != 0;          // of the wave's keys

  TileAddr<D> at;
  at.init(smem);
  u32x4 kf[NP][KC], vf[NP][KC];
  load_operand<NP, D>(a.k.p + b * a.k.sb + hk * a.k.sh + jc * a.k.sn, counts, kf);
  load_operand<NP, D>(a.v.p + b * a.v.sb + hk * a.v.sh + jc * a.v.sn, counts, vf);
  f32x16 dk[NT], dv[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) dk[t] = dv[t] = splat16(0.0f);
  // three ones against the first number of a query (half 0's chunk) and its second (half 1's)
  const u32x4 three = {0x3F803F80u, 0x00003F80u, 0u, 0u}, none4 = {0u, 0u, 0u, 0u};
  const u32x4 ones_l = hf == 0 ? three : none4, ones_d = hf == 0 ? none4 : three;
  const uint32_t nums = lds_addr(smem) + NUMS + 16 * (hf * QT + (lane & 31));
  const float inv_scale = 1.0f / a.scale;

  // causal: the first query whose position reaches the block's first key, and the
  // first stage that all of the block's keys are behind
  const int first = a.causal ? min(max(block0 - start, 0), a.nq) / QT * QT : 0;
  const int stages = block0 < limit ? (a.nq - first + QT - 1) / QT : 0;   // per head
  const int border = a.causal ? min(max(block0 + kExactWaves * 32 - 1 - start - first + QT - 1, 0) / QT, stages) : 0;
  // The stages go from the last query down, and with one bias through all heads at each: workgroups
  // that start together then read the same rows, which the XCD's L2 holds, wherever their keys'
  // first query lies (16 heads on 4 x 16384 x 128 causal: 0.9 GB from beyond L2, 5.3 head after
  // head from each block's first query on; training 5.13 -> 5.05 ms in turn on one card, less than cards differ by).
  const int inner = BIAS ? 1 : a.group;
  // this workgroup's part of the stages of all heads
  const long long all = (long long)a.group * stages;
  const long long t0 = parts == 1 ? 0 : all * part / parts, t1 = parts == 1 ? all : all * (part + 1) / parts;
  constexpr bool kPlain = !BIAS && NP == 1;
  const long long turn = (long long)inner * stages;
  for (int hg = stages == 0 ? a.group : (t0 == 0 ? 0 : (int)(t0 / turn) * inner); hg < a.group && (long long)hg * stages < t1; hg += inner) {
    const int begin = (int)max(t0 - (long long)hg * stages, 0ll), end = (int)min(t1 - (long long)hg * stages, turn);
    const int h = hk * a.group + hg;
    const char* qp = a.q.p + b * a.q.sb + h * a.q.sh;
    const char* gp = g.dout.p + b * g.dout.sb + h * g.dout.sh;
    const long long lrow = ((long long)b * a.H + h) * a.nq;
    float lo = 0.0f, hi = 0.0f;
    if constexpr (BIAS) {
      fill_window(a, h, win, tid, kExactThreads);
      lo = bias_value(a, h, 0) * kLog2e;
      hi = bias_value(a, h, 2 * a.far) * kLog2e;
    }
    St qs, gs;
    qs.init(a.q.sn, tid);
    gs.init(g.dout.sn, tid);
    float L = 0.0f, delta = 0.0f;                  // of query tid of the stage
    // the stage at hand and the next: first query, head beyond h
    int q0 = first + (stages - 1 - begin / inner) * QT, hn = begin % inner, qn = q0;
    auto load = [&]() {
      qs.load(qp + hn * a.q.sh, a.q.sn, qn, a.nq);
      gs.load(gp + hn * g.dout.sh, g.dout.sn, qn, a.nq);
      if (tid < QT) {                              // as they are: looked at in store(), when they have arrived
        const long long at_row = lrow + (long long)hn * a.nq + min(qn + tid, a.nq - 1);
        L = g.lse[at_row];
        delta = g.delta[at_row];
      }
    };
    auto store = [&](int buf) {
      const RowBits<QT> ok = row_bits<QT>(qn, a.nq);
      qs.store(smem + buf * 2 * St::kBytes, ok, tid);
      gs.store(smem + buf * 2 * St::kBytes + St::kBytes, ok, tid);
      if (tid < QT) {
        const bool off = qn + tid >= a.nq || L == -INFINITY;   // no weight: finite, as it meets zeros too
        u32x4* to = reinterpret_cast<u32x4*>(smem + NUMS) + 2 * QT * buf + tid;
        to[0] = number_chunk(off ? -3e38f : -L * inv_scale);
        to[QT] = number_chunk(off ? 0.0f : -delta);
      }
    };
    load();
    store(0);
    __syncthreads();
    wait_loads<0>();                               // the operands too: no wait for them beside the loads in flight below
    auto chunk_of = [&](int off) { return *(const __attribute__((address_space(3))) u32x4*)(lds_ptr)(nums + off); };
    // a stage in buffer BUF; PLAIN: every query reaches every key, one bias
    auto stage = [&](int st, auto BUF, auto PLAIN) {
      constexpr int cur = BUF * 2 * St::kBytes;
      const bool more = st + 1 < end;
      if (more) {
        if (++hn == inner) {
          hn = 0;
          qn -= QT;
        }
        load();
      }
#pragma unroll
      for (int x = 0; x < TILES; ++x) {
        const int p0 = start + q0 + 32 * x;        // position of the tile's first query
        // no query reaches a key (PLAIN goes on past the last query, which has no weight)
        if (!PLAIN && (!any || a.nq <= q0 + 32 * x || (a.causal && p0 + 31 < k0))) continue;
        const int qtile = cur + x * kTileBytes<D>, gtile = cur + St::kBytes + x * kTileBytes<D>;
        f32x16 s, dp;
        u32x4 gt[2][NT], qt[2][NT];
        const u32x4 n = chunk_of(32 * QT * BUF + 512 * x);
        if constexpr (NP == 1) {
          u32x4 qr[KC], gr[KC];
          read_rows<D>(at, qtile, qr);
          read_rows<D>(at, gtile, gr);
          __builtin_amdgcn_sched_barrier(0);
          s = dp = splat16(0.0f);
#pragma unroll
          for (int c = 0; c < KC; ++c) {
            s = mfma16(qr[c], kf[0][c], s);
            dp = mfma16(gr[c], vf[0][c], dp);
          }
          s = mfma16(n, ones_l, s);
          dp = mfma16(n, ones_d, dp);
          read_trans<D>(at, gtile, gt);
          if constexpr (D < 128) read_trans<D>(at, qtile, qt);
          __builtin_amdgcn_sched_barrier(0);
        } else {
          s = mfma16(n, ones_l, product<NP, D>(at, qtile, STEP, kf, splat16(0.0f)));
          dp = mfma16(n, ones_d, product<NP, D>(at, gtile, STEP, vf, splat16(0.0f)));
        }
        float mul = a.scale_log2, add = 0.0f;
        if constexpr (!PLAIN) {
          if constexpr (BIAS) {
            const int d0 = k0 - p0;
            const BiasKind kind = bias_kind(d0, a.far);
            if (kind == kBiasNear) {
              const float* wp = win + (d0 + a.far + kWinPad + (lane & 31) - 4 * hf);
#pragma unroll
              for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale_log2, wp[-reg_row(r)]);
              mul = 1.0f;
            } else {
              add = kind == kBiasLow ? lo : hi;
            }
          }
          if (a.causal && p0 < k0 + 31) select_rows(s, ~low_bits(j - p0), -INFINITY);
        }
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(!PLAIN && BIAS ? fmaf(s[r], mul, add) : s[r] * mul);
        const Packed<NP> pw = pack_weights<NP>(p);
        if constexpr (NP == 1) accumulate_chunks<D>(gt, pw, dv);
        else accumulate_t<NP, D>(at, gtile, STEP, pw, dv);
        if constexpr (NP == 1 && D == 128) read_trans<D>(at, qtile, qt);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] *= dp[r];
        const Packed<NP> dw = pack_weights<NP>(p);
        if constexpr (NP == 1) accumulate_chunks<D>(qt, dw, dk);
        else accumulate_t<NP, D>(at, qtile, STEP, dw, dk);
      }
      if (more) store(1 - BUF);
      q0 = qn;
      __syncthreads();
    };
    constexpr std::integral_constant<int, 0> b0{};
    constexpr std::integral_constant<int, 1> b1{};
    // stages whose queries all reach all keys, in pairs, then (with a bias or in float32, all) the others
    int st = begin;
    if constexpr (kPlain) {
      const int plain = begin + (max(min((stages - border) * inner, end) - begin, 0) & ~1);
      // (a second stage is always there; without the question the kernel takes 106 registers more at D = 128:
      // 5.05 -> 5.22 ms)
      for (; st < plain; st += 2) {
        stage(st, b0, std::true_type{});
        if (st + 1 < end) stage(st + 1, b1, std::true_type{});
      }
    }
    for (; st < end; st += 2) {
      stage(st, b0, std::false_type{});
      if (st + 1 < end) stage(st + 1, b1, std::false_type{});
    }
  }
  // a key that does not count has no gradient (its column of P is not one)
  if (!counts) {
#pragma unroll
    for (int t = 0; t < NT; ++t) dk[t] = dv[t] = splat16(0.0f);
  }
  if (parts > 1) {
    const long long row = ((long long)part * a.B * a.Hkv + bk) * a.nk + jc;
    store_rows<3, D>(dk, a.scale, reinterpret_cast<char*>(g.part_k + row * D), j < a.nk);
    store_rows<3, D>(dv, 1.0f, reinterpret_cast<char*>(g.part_v + row * D), j < a.nk);
    return;
  }
  store_rows<NP, D>(dk, a.scale, g.dk.p + b * g.dk.sb + hk * g.dk.sh + jc * g.dk.sn, j < a.nk);
  store_rows<NP, D>(dv, 1.0f, g.dv.p + b * g.dv.sb + hk * g.dv.sh + jc * g.dv.sn, j < a.nk);
}

// Adds the parts of dq, dk and dv (float32 rows, in their order): four columns a thread.
struct PartSums {
  const float* from[3];
  Rows to[3];
  long long rows[3];                               // of one part: batches x heads x n
  int heads[3], n[3], parts[3];
};
template <int NP, int D>
__global__ __launch_bounds__(256) void exact_sum_kernel(PartSums s) {
  constexpr int L = D / 4;
  const int which = blockIdx.y;
  const long long row = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
  if (row >= s.rows[which]) return;
  const int c = threadIdx.x % L, parts = s.parts[which];
  const f32x4* at = reinterpret_cast<const f32x4*>(s.from[which]) + row * L + c;
  f32x4 t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const f32x4 x = at[p * s.rows[which] * L];
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] += x[e];
  }
  const long long bh = row / s.n[which];
  const int i = (int)(row - bh * s.n[which]), b = (int)(bh / s.heads[which]), h = (int)(bh - (long long)b * s.heads[which]);
  const float z[4] = {t[0], t[1], t[2], t[3]};
  const Rows& to = s.to[which];
  store4<NP>(to.p + b * to.sb + h * to.sh + i * to.sn + 4 * c * (NP == 1 ? 2 : 4), z);
}

// dbias: a workgroup per head and bucket. It lists the window's entries that the map
// sends to its bucket, and its threads sum them over the head's blocks in double.
constexpr int kBiasThreads = 256;
constexpr int kMaxEntries = window_entries(MRA_EXACT_MAX_FAR) + 2;
__global__ __launch_bounds__(kBiasThreads) void exact_bias_kernel(ExactArgs a, const float* __restrict__ diag, int parts,
                                                                  void* __restrict__ dbias) {
  __shared__ uint16_t list[kMaxEntries];
  __shared__ int count;
  __shared__ double sums[kBiasThreads];
  const int h = blockIdx.x, c = blockIdx.y, tid = threadIdx.x, entries = window_entries(a.far) + 2;
  const float* src = diag + (long long)h * parts * entries;
  if (tid < kWave) {                               // ascending: one wave, its lanes' hits in order
    int n = 0;
    for (int e0 = 0; e0 < entries; e0 += kWave) {
      const int e = e0 + tid;
      int d = min(max(e - kWinPad, 0), 2 * a.far);
      if (e == entries - 2) d = 0;                 // the tiles below the window, and above it
      if (e == entries - 1) d = 2 * a.far;
      const bool hit = e < entries && a.map[d] == c;
      const uint64_t hits = __ballot(hit);
      if (hit) list[n + bits_below(hits)] = (uint16_t)e;
      n += __popcll(hits);
    }
    if (tid == 0) count = n;
  }
  __syncthreads();
  const int n = count;
  double t = 0.0;
  if (n > 0) {
    // threads side by side take entries side by side of a block, whole blocks where they fit
    const int cols = min(n, kBiasThreads), per = kBiasThreads / cols, col = tid % cols, first = tid / cols;
    if (first < per)
      for (int e = col; e < n; e += cols) {
        const float* at = src + list[e];
#pragma unroll 8
        for (int p = first; p < parts; p += per) t += (double)at[(long long)p * entries];
      }
  }
  sums[tid] = t;
  __syncthreads();
  for (int half = kBiasThreads / 2; half > 0; half /= 2) {
    if (tid < half) sums[tid] += sums[tid + half];
    __syncthreads();
  }
  if (tid == 0) {
    const long long at = (long long)c * a.H + h;
    if (a.bias_bf16) static_cast<uint16_t*>(dbias)[at] = (uint16_t)f32_to_bf16_rne((float)sums[0]);
    else static_cast<float*>(dbias)[at] = (float)sums[0];
  }
}

// Several workgroups share the stages of each block where the blocks would leave half of
// the chip idle, or, in passes that hold one workgroup per CU, part of their last round; each takes
// at least eight stages, and more parts have to save a fifth of the rounds. Their sums are
// float32 rows in the workspace and cost a launch. 8 query heads on 2 key heads x 4 x 1503 x
// 128 float32: dK and dV 968 us in 96 workgroups, 465 + 18 in 480; dQ in 768 instead of 384:
// the training step 1047 -> 1021 us. Where two workgroups fit a CU and fill more than half, the sums
// cost what the parts give (dQ of 96 heads x 333 x 64 on 1501 keys, 288 blocks: 46 us, 39 + 7 in
// four parts).
static int parts_of(long long blocks, long long stages, int per_cu) {
  const long long room = (long long)per_cu * kCus;
  if (blocks == 0 || 2 * blocks > (per_cu == 1 ? 8 : 1) * room) return 1;
  const int most = (int)max(1ll, min(stages / 8, 8ll));
  auto rounds = [&](int p) { return (double)((blocks * p + room - 1) / room) / p; };
  int best = 1;
  for (int p = 2; p <= most; ++p)
    if (rounds(p) <= 0.8 * rounds(best)) best = p;
  return best;
}

BackwardPlan exact_backward_plan(const mra_exact_problem_t& p) {
  BackwardPlan b{};
  const bool f32 = p.dtype == MRA_F32;
  const int rows = !f32 || p.d == 32 ? 64 : 32;
  const long long kheads = (long long)p.B * p.H_kv, heads = (long long)p.B * p.H;
  const long long qstages = (p.n_q + rows - 1) / rows, kstages = (p.n_k + rows - 1) / rows;
  b.dq_parts = parts_of(heads * exact_dq_blocks(p.n_q), kstages, f32 && p.d == 128 ? 1 : 2);
  b.dkv_parts = parts_of(kheads * exact_dq_blocks(p.n_k), qstages * (p.H / p.H_kv), p.d == 128 ? 1 : 2);
  // Below eight keys per distance of the window the 2-norm of dbias's error is a bfloat16 rounding's
  // at most (2.6e-3 at 512 keys and 183 distances, 3.2e-3 at 1503), and the window's tiles are much of a row
  // (training, 8 x 12 heads x 1024 x 32: 133 us, 157 with exact_centre_kernel; where it runs: 32 heads x 2048 x 128
  // causal 390 -> 423, 8 x 8192 x 128 1397 -> 1446).
  b.centre = !f32 && p.bias != nullptr && p.n_k > 8 * (2 * (long long)p.far + 1);
  if (b.dq_parts > 1) b.q_floats = (size_t)b.dq_parts * heads * p.n_q * p.d;
  if (b.dkv_parts > 1) b.k_floats = (size_t)b.dkv_parts * kheads * p.n_k * p.d;
  return b;
}

template <int NP, int D, bool BIAS>
static hipError_t backward_case(const ExactArgs& a, const ExactGrads& g, const BackwardPlan& plan, hipStream_t stream) {
  constexpr size_t dq_stage = 4 * Stage<NP, D, kDqStageRows<NP, D>, kExactThreads>::kBytes;
  constexpr size_t stage = 4 * Stage<NP, D, kStageRows<NP, D>, kExactThreads>::kBytes;
  const size_t entries = BIAS ? window_entries(a.far) : 0;
  const int qblocks = exact_dq_blocks(a.nq), kblocks = exact_dq_blocks(a.nk);
  const long long heads = (long long)a.B * a.H, kheads = (long long)a.B * a.Hkv;
  hipError_t e;
  if (a.nq > 0) {
    const size_t smem = dq_stage + ((1 + kExactWaves) * entries + (BIAS ? kExactWaves * kSkew : 0)) * sizeof(float) + (BIAS ? kFarBytes : 0);
    auto launch = [&](auto kernel, int blocks) {
      const hipError_t lds = allow_lds(kernel, smem);
      if (lds != hipSuccess) return lds;
      kernel<<<dim3((unsigned)(heads * blocks), plan.dq_parts), kExactThreads, smem, stream>>>(a, g, blocks);
      return hipGetLastError();
    };
    if constexpr (NP == 1 && D <= 64 && !BIAS) {
      // (training, 96 heads x 4096 x 64: 1.85 -> 1.82 ms)
      e = wide_rows(heads, a.nq) ? launch(exact_dq_kernel<NP, D, 2, BIAS>, (a.nq + 2 * kDqRows - 1) / (2 * kDqRows))
                                 : launch(exact_dq_kernel<NP, D, 1, BIAS>, qblocks);
    } else {
      e = launch(exact_dq_kernel<NP, D, 1, BIAS>, qblocks);
    }
    if (e != hipSuccess) return e;
    if constexpr (NP == 1 && BIAS) {
      if (g.row_sums != nullptr) {
        const size_t centre = 2 * Stage<1, D, kStageRows<1, D>, kExactThreads>::kBytes +
                              ((1 + kExactWaves) * entries + kExactWaves * kSkew) * sizeof(float) + kFarBytes;
        auto kernel = exact_centre_kernel<D>;
        if ((e = allow_lds(kernel, centre)) != hipSuccess) return e;
        kernel<<<(unsigned)(heads * qblocks), kExactThreads, centre, stream>>>(a, g, qblocks, plan.dq_parts);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
    }
  }
  if (a.nk > 0) {
    const size_t smem = stage + 64 * kStageRows<NP, D> + entries * sizeof(float);
    auto kernel = exact_dkv_kernel<NP, D, BIAS>;
    if ((e = allow_lds(kernel, smem)) != hipSuccess) return e;
    kernel<<<dim3((unsigned)(kheads * kblocks), plan.dkv_parts), kExactThreads, smem, stream>>>(a, g, kblocks);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (plan.q_floats + plan.k_floats > 0) {
    PartSums s{};
    auto add = [&](int i, const float* from, const Rows& to, long long rows, int h, int n, int parts) {
      s.from[i] = from;
      s.to[i] = to;
      s.rows[i] = rows;
      s.heads[i] = h;
      s.n[i] = n;
      s.parts[i] = parts;
    };
    int n = 0;
    if (plan.dq_parts > 1) add(n++, g.part_q, g.dq, heads * a.nq, a.H, a.nq, plan.dq_parts);
    if (plan.dkv_parts > 1) {
      add(n++, g.part_k, g.dk, kheads * a.nk, a.Hkv, a.nk, plan.dkv_parts);
      add(n++, g.part_v, g.dv, kheads * a.nk, a.Hkv, a.nk, plan.dkv_parts);
    }
    long long rows = 0;
    for (int i = 0; i < n; ++i) rows = max(rows, s.rows[i]);
    constexpr int per = 256 / (D / 4);
    exact_sum_kernel<NP, D><<<dim3((unsigned)((rows + per - 1) / per), n), 256, 0, stream>>>(s);
  }
  return hipGetLastError();
}

hipError_t launch_exact_backward(const ExactArgs& a, const ExactGrads& g, const BackwardPlan& plan, int d, int dtype,
                                 hipStream_t stream) {
  auto pick = [&](auto np, auto dd) {
    constexpr int NP = decltype(np)::value, D = decltype(dd)::value;
    return a.bias != nullptr ? backward_case<NP, D, true>(a, g, plan, stream)
                             : backward_case<NP, D, false>(a, g, plan, stream);
  };
  auto width = [&](auto np) {
    if (d == 32) return pick(np, std::integral_constant<int, 32>{});
    if (d == 64) return pick(np, std::integral_constant<int, 64>{});
    return pick(np, std::integral_constant<int, 128>{});
  };
  if (a.B > 0 && a.H > 0) {
    const hipError_t e = dtype == BF16 ? width(std::integral_constant<int, 1>{}) : width(std::integral_constant<int, 3>{});
    if (e != hipSuccess) return e;
  }
  if (g.dbias != nullptr && a.H > 0)
    exact_bias_kernel<<<dim3(a.H, a.buckets), kBiasThreads, 0, stream>>>(a, g.diag, a.B * exact_dq_blocks(a.nq) * g.slots, g.dbias);
  return hipGetLastError();
}

}  // namespace mra
