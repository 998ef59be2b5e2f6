// Exact softmax attention, forward (mra_exact.h): Z = softmax(S) V with
// S = scale Q K^T + position bias over the keys that count, in one pass over the
// keys with a running reference and sum per query.
//
// As in the tile pass of MRA-2 (tile.hip) S is formed transposed, S^T = K Q^T, so
// a lane holds 16 key scores of one query, which are already the B operand of
// O^T += V^T P^T: weights never move between lanes.
//
// exact_fwd_kernel: a workgroup's four waves take 32 QT queries each of one
// head and walk the keys together, a stage of K and V rows in LDS at a time (two
// buffers, one barrier per stage); the next stage's rows are on their way to
// registers meanwhile.
//
// exact_split_kernel: few rows. The workgroup's four waves share 32 rows (the
// queries of all heads of one key head, so a token's heads are one tile) and take
// every fourth tile of 32 keys; several workgroups may share the rows too, each
// with a contiguous part of the keys, and leave partial sums that
// exact_join_kernel adds.
#include "exact_rows.h"

namespace mra {

// The scores of a tile with bias and masks: s, mul and add of add_tile. d0: the
// distance of the tile's first key and this wave's first query; dq: this lane's
// query behind that one; bits: this lane's keys that count; lo, hi: the outer biases.
template <bool BIAS>
__device__ __forceinline__ void finish_scores(f32x16& s, float& mul, float& add, float sl2, bool masked, uint32_t bits, int d0,
                                              int far, const float* win, float lo, float hi) {
  mul = sl2;
  add = 0.0f;
  if constexpr (BIAS) {
    const BiasKind kind = bias_kind(d0, far);      // wave-uniform
    if (kind == kBiasNear) {
      const int lane = lane_id();
      const float* w = win + (d0 + far + kWinPad - (lane & 31) + 4 * (lane >> 5));
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], sl2, w[reg_row(r)]);
      mul = 1.0f;
    } else {
      add = kind == kBiasLow ? lo : hi;
    }
  }
  if (masked) select_rows(s, bits, -INFINITY);
}

// s[x] = K Q_x^T for all rows of a wave (float32: 32), each K chunk read once.
template <int NP, int D, int R>
__device__ __forceinline__ void products(const TileAddr<D>& at, int tile, int step, const FwdRow<NP, D> (&row)[R],
                                         f32x16 (&s)[R]) {
  static_assert(NP == 1 || R == 1, "float32: 32 queries per wave");
  if constexpr (NP == 3 && D == 128) {             // fewer chunks at a time, for registers: 314 -> 296 us, 32 heads x 1503
    s[0] = product<NP, D>(at, tile, step, row[0].qf, splat16(0.0f));
    return;
  }
#pragma unroll
  for (int x = 0; x < R; ++x) s[x] = splat16(0.0f);
#pragma unroll
  for (int p = NP - 1; p >= 0; --p) {
    u32x4 k[D / 16];
#pragma unroll
    for (int c = 0; c < D / 16; ++c) k[c] = at.row(tile + p * step, c);
#pragma unroll
    for (int x = 0; x < R; ++x)
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int q = NP - 1 - p; q >= 0; --q) s[x] = mfma16(k[c], row[x].qf[q][c], s[x]);
  }
}

template <int NP, int D, int QT, bool BIAS>
__global__ __launch_bounds__(kExactThreads) void exact_fwd_kernel(ExactArgs a, float* __restrict__ lse, int qblocks) {
  constexpr int KT = kStageRows<NP, D>, TILES = KT / 32;
  using St = Stage<NP, D, KT, kExactThreads>;
  constexpr int STEP = TILES * kTileBytes<D>;      // bytes from one plane to the next
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* win = reinterpret_cast<float*>(smem + 4 * St::kBytes);
  const int tid = threadIdx.x, lane = lane_id(), w = wave_uniform(tid / kWave);
  const HeadBlock hb = head_block(blockIdx.x, a.B * a.H, qblocks, a.causal);
  // causal rows take the longer the later they are: the last blocks of a head first
  const int bh = hb.head, qb = qblocks - 1 - hb.block;
  const int b = bh / a.H, h = bh - b * a.H, hk = h / a.group;
  const int row0 = (qb * kExactWaves + w) * 32 * QT;
  const int limit = key_limit(a, b), start = first_position(a, b);
  const int last = min((qb + 1) * kExactWaves * 32 * QT, a.nq) - 1;   // the block's last query
  const int kend = a.causal ? min(limit, start + last + 1) : limit;
  const int stages = kend > 0 ? (kend + KT - 1) / KT : 0;
  const char* kp = a.k.p + b * a.k.sb + hk * a.k.sh;
  const char* vp = a.v.p + b * a.v.sb + hk * a.v.sh;

  TileAddr<D> at;
  at.init(smem);
  FwdRow<NP, D> row[QT];
  int pos0[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int i = row0 + 32 * x + (lane & 31);
    load_operand<NP, D>(a.q.p + b * a.q.sb + h * a.q.sh + min(i, a.nq - 1) * a.q.sn, i < a.nq, row[x].qf);
    row[x].init();
    pos0[x] = start + row0 + 32 * x;
  }
  float lo = 0.0f, hi = 0.0f;
  if constexpr (BIAS) {
    fill_window(a, h, win, tid, kExactThreads);
    lo = bias_value(a, h, 0) * kLog2e;
    hi = bias_value(a, h, 2 * a.far) * kLog2e;
  }

  St ks, vs;
  ks.init(a.k.sn, tid);
  vs.init(a.v.sn, tid);
  MaskBytes<KT> bytes;
  RowBits<KT> ok{};
  if (stages > 0) {
    ks.load(kp, a.k.sn, 0, limit);
    vs.load(vp, a.v.sn, 0, limit);
    bytes.load(a, b, 0);
    ok = bytes.bits(0, limit);
    ks.store(smem, ok, tid);
    vs.store(smem + St::kBytes, ok, tid);
  }
  __syncthreads();
  wait_loads<0>();                                 // Q too: no wait for it beside the loads in flight below
  // stage st in buffer BUF (known at compile time: its part of an LDS address is an offset)
  auto stage = [&](int st, auto BUF) {
    constexpr int kbuf = BUF * 2 * St::kBytes, vbuf = kbuf + St::kBytes;
    const bool more = st + 1 < stages;
    if (more) {
      ks.load(kp, a.k.sn, (st + 1) * KT, limit);
      vs.load(vp, a.v.sn, (st + 1) * KT, limit);
      bytes.load(a, b, (st + 1) * KT);
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const uint32_t kb = ok.tile(i);
      const int k0 = st * KT + 32 * i, ktile = kbuf + i * kTileBytes<D>, vtile = vbuf + i * kTileBytes<D>;
      if (kb == 0 || (a.causal && k0 > pos0[QT - 1] + 31)) continue;      // no key counts for the wave
      f32x16 s[QT];
      products<NP, D, QT>(at, ktile, STEP, row, s);
      float mul[QT], add[QT];
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        // keys up to this lane's position
        const uint32_t bits = a.causal ? kb & low_bits(pos0[x] + (lane & 31) - k0 + 1) : kb;
        const bool masked = kb != ~0u || (a.causal && k0 + 31 > pos0[x]);
        finish_scores<BIAS>(s[x], mul[x], add[x], a.scale_log2, masked, bits, k0 - pos0[x], a.far, win, lo, hi);
      }
      Packed<NP> pw[QT];
      if constexpr (NP == 1) {
        u32x4 v[2][D / 32];                        // on their way while the weights are formed
        read_trans<D>(at, vtile, v);
        __builtin_amdgcn_sched_barrier(0);
        tile_weights<NP, D, QT>(row, s, mul, add, pw);
        // ahead of the SIMD's other wave while it forms weights: 8 heads x 12 x 4096 x 64: 432 -> 428 us
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int x = 0; x < QT; ++x) accumulate_chunks<D>(v, pw[x], row[x].o);
        __builtin_amdgcn_s_setprio(0);
      } else {
        tile_weights<NP, D, QT>(row, s, mul, add, pw);
        __builtin_amdgcn_s_setprio(1);
        accumulate_t<NP, D>(at, vtile, STEP, pw[0], row[0].o);
        __builtin_amdgcn_s_setprio(0);
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
  for (int st = 0; st < stages; st += 2) {
    stage(st, std::integral_constant<int, 0>{});
    if (st + 1 < stages) stage(st + 1, std::integral_constant<int, 1>{});
  }
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int i = row0 + 32 * x + (lane & 31);
    const float den = halves_sum(row[x].sum);
    store_rows<NP, D>(row[x].o, den > 0.0f ? 1.0f / den : 0.0f,
                      a.out.p + b * a.out.sb + h * a.out.sh + min(i, a.nq - 1) * a.out.sn, i < a.nq);
    if (lse != nullptr && lane < 32 && i < a.nq)
      lse[(long long)bh * a.nq + i] = den > 0.0f ? (log2f(den) + row[x].ref) * kLn2 : -INFINITY;
  }
}

// Row m of a key head's queries: query m / group of head hk group + m % group.
template <int NP, int D, bool BIAS>
__global__ __launch_bounds__(kExactThreads) void exact_split_kernel(ExactArgs a, float* __restrict__ lse, int mtiles,
                                                                    int splits, float* __restrict__ part_o,
                                                                    float* __restrict__ part_l) {
  using St = Stage<NP, D, 32, kWave>;
  constexpr int NT = D / 32;
  constexpr int SLOT = St::kBytes;                 // a wave's tile: K, then V
  constexpr int MERGE = 32 * D * 4;                // a wave's accumulators
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float refs[kExactWaves][kWave], sums[kExactWaves][kWave];
  const int lane = lane_id(), w = wave_uniform(threadIdx.x / kWave);
  const int g = xcd_remap(blockIdx.x, gridDim.x);
  const int sp = g % splits, mt = g / splits % mtiles, bk = g / splits / mtiles;
  const int b = bk / a.Hkv, hk = bk - b * a.Hkv;
  const int rows = a.nq * a.group;
  const int m = mt * 32 + (lane & 31), mc = min(m, rows - 1);
  const int i = mc / a.group, h = hk * a.group + (mc - i * a.group);
  const int limit = key_limit(a, b), start = first_position(a, b);
  const int pos = start + i, last = start + min(mt * 32 + 31, rows - 1) / a.group;
  const int kend = a.causal ? min(limit, last + 1) : limit;
  const int tiles = kend > 0 ? (kend + 31) / 32 : 0;
  const int t0 = (int)((long long)tiles * sp / splits), t1 = (int)((long long)tiles * (sp + 1) / splits);
  const char* kp = a.k.p + b * a.k.sb + hk * a.k.sh;
  const char* vp = a.v.p + b * a.v.sb + hk * a.v.sh;
  char* slot = smem + w * SLOT;

  TileAddr<D> at;
  at.init(slot);
  FwdRow<NP, D> rows1[1];
  FwdRow<NP, D>& row = rows1[0];
  load_operand<NP, D>(a.q.p + b * a.q.sb + h * a.q.sh + i * a.q.sn, m < rows, row.qf);
  row.init();
  float lo = 0.0f, hi = 0.0f;
  if constexpr (BIAS) {
    lo = bias_value(a, h, 0) * kLog2e;
    hi = bias_value(a, h, 2 * a.far) * kLog2e;
  }
  St ks, vs;
  ks.init(a.k.sn, lane);
  vs.init(a.v.sn, lane);
  MaskBytes<32> bytes;
  int t = t0 + w;
  if (t < t1) {
    ks.load(kp, a.k.sn, t * 32, limit);
    vs.load(vp, a.v.sn, t * 32, limit);
    bytes.load(a, b, t * 32);
  }
  wait_loads<0>();                                 // Q too: no wait for it beside the loads in flight below
  for (; t < t1; t += kExactWaves) {
    const int k0 = t * 32;
    const RowBits<32> ok = bytes.bits(k0, limit);
    ks.store(slot, ok, lane);
    wave_lds_sync();
    const bool more = t + kExactWaves < t1;
    if (more) ks.load(kp, a.k.sn, k0 + 32 * kExactWaves, limit);
    f32x16 s1[1] = {product<NP, D>(at, 0, kTileBytes<D>, row.qf, splat16(0.0f))};
    f32x16& s = s1[0];
    wave_lds_sync();
    vs.store(slot, ok, lane);
    wave_lds_sync();
    if (more) {
      vs.load(vp, a.v.sn, k0 + 32 * kExactWaves, limit);
      bytes.load(a, b, k0 + 32 * kExactWaves);
    }
    const uint32_t kb = ok.tile(0), bits = a.causal ? kb & low_bits(pos - k0 + 1) : kb;
    if (__ballot(bits != 0) != 0) {
      float mul = a.scale_log2, add = 0.0f;
      if constexpr (BIAS) {
        // rows of several heads and queries: every lane has its own distances, d of its first key
        const int d = k0 - pos, r4 = 4 * (lane >> 5);
        const bool below = d + 31 <= -a.far, above = d >= a.far;
        if (__ballot(!(below || above)) == 0) {
          add = below ? lo : hi;
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[r] = fmaf(s[r], a.scale_log2,
                        bias_value(a, h, min(max(d + r4 + reg_row(r), -a.far), a.far) + a.far) * kLog2e);
          mul = 1.0f;
        }
      }
      if (__ballot(bits != ~0u) != 0) select_rows(s, bits, -INFINITY);
      Packed<NP> pw[1];
      tile_weights<NP, D, 1>(rows1, s1, {mul}, {add}, pw);
      accumulate_t<NP, D>(at, 0, kTileBytes<D>, pw[0], row.o);
    }
    wave_lds_sync();
  }
  // the waves' sums relative to the largest reference, added in wave order
  float sum = halves_sum(row.sum);
  refs[w][lane] = row.ref;
  sums[w][lane] = sum;
  __syncthreads();                                 // the slots are idle
  float top = refs[0][lane];
#pragma unroll
  for (int x = 1; x < kExactWaves; ++x) top = fmaxf(top, refs[x][lane]);
  auto factor = [&](float ref) { return ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref - top); };
  const float f = factor(row.ref);
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int r = 0; r < 16; ++r) row.o[x][r] *= f;
  if (w != 0) {
    f32x4* to = reinterpret_cast<f32x4*>(smem + (w - 1) * MERGE) + lane;
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        to[(4 * x + q) * kWave] = f32x4{row.o[x][4 * q], row.o[x][4 * q + 1], row.o[x][4 * q + 2], row.o[x][4 * q + 3]};
  }
  __syncthreads();
  if (w != 0) return;
  sum *= f;
#pragma unroll
  for (int p = 1; p < kExactWaves; ++p) {
    sum += sums[p][lane] * factor(refs[p][lane]);
    const f32x4* from = reinterpret_cast<const f32x4*>(smem + (p - 1) * MERGE) + lane;
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = from[(4 * x + q) * kWave];
#pragma unroll
        for (int e = 0; e < 4; ++e) row.o[x][4 * q + e] += v[e];
      }
  }
  if (splits == 1) {
    store_rows<NP, D>(row.o, sum > 0.0f ? 1.0f / sum : 0.0f, a.out.p + b * a.out.sb + h * a.out.sh + i * a.out.sn,
                      m < rows);
    if (lse != nullptr && lane < 32 && m < rows)
      lse[((long long)b * a.H + h) * a.nq + i] = sum > 0.0f ? (log2f(sum) + top) * kLn2 : -INFINITY;
    return;
  }
  const long long pr = ((long long)sp * a.B * a.Hkv + bk) * rows + mc;   // the partial row
  store_rows<3, D>(row.o, 1.0f, reinterpret_cast<char*>(part_o + pr * D), m < rows);
  if (lane < 32 && m < rows) {
    part_l[2 * pr] = top;
    part_l[2 * pr + 1] = sum;
  }
}

// The split kernel serves calls of fewer 128-row workgroups than CUs, and those whose
// rows would leave at least half of each workgroup idle (up to 64 rows a key head); its
// workgroups are at least two per CU where the keys allow, at most one per 256 keys begun.
// Measured well inside either side (4 and 48 blocks, single tokens; 288 blocks and more), not at the border.
SplitPlan exact_split_plan(const mra_exact_problem_t& p) {
  SplitPlan s{};
  const long long heads = (long long)p.B * p.H, kheads = (long long)p.B * p.H_kv;
  const long long blocks = heads * ((p.n_q + 127) / 128);
  const long long rows = (long long)p.n_q * (p.H / p.H_kv);
  s.mtiles = (int)((rows + 31) / 32);
  s.splits = 1;
  s.use = (blocks < kCus || rows <= 64) && rows < (1 << 20);
  if (s.use) {
    const long long wgs = kheads * s.mtiles, most = (p.n_k + 255) / 256;
    long long want = (2 * kCus + wgs - 1) / wgs;
    if (want > most) want = most;
    if (want > 64) want = 64;
    if (want > 1) s.splits = (int)want;
    if (s.splits > 1) s.bytes = (size_t)s.splits * kheads * rows * (p.d + 2) * sizeof(float);
  }
  return s;
}

template <int NP, int D, int QT, bool BIAS>
static hipError_t launch_rows(const ExactArgs& a, float* lse, hipStream_t stream) {
  const int qblocks = (a.nq + kExactWaves * 32 * QT - 1) / (kExactWaves * 32 * QT);
  const size_t smem = 4 * Stage<NP, D, kStageRows<NP, D>, kExactThreads>::kBytes +
                      (BIAS ? window_entries(a.far) * sizeof(float) : 0);
  auto kernel = exact_fwd_kernel<NP, D, QT, BIAS>;
  const hipError_t e = allow_lds(kernel, smem);
  if (e != hipSuccess) return e;
  kernel<<<(unsigned)((long long)a.B * a.H * qblocks), kExactThreads, smem, stream>>>(a, lse, qblocks);
  return hipGetLastError();
}

template <int NP, int D, bool BIAS>
static hipError_t forward_case(const ExactArgs& a, float* lse, const SplitPlan& plan, void* ws, hipStream_t stream) {
  if (plan.use) {
    using St = Stage<NP, D, 32, kWave>;
    constexpr int slots = kExactWaves * St::kBytes, merge = (kExactWaves - 1) * 32 * D * 4;
    constexpr size_t smem = slots > merge ? slots : merge;
    const long long rows = (long long)a.B * a.Hkv * a.nq * a.group;
    float* part_o = static_cast<float*>(ws);
    float* part_l = part_o + (plan.splits > 1 ? plan.splits * rows * D : 0);
    const unsigned wgs = (unsigned)((long long)a.B * a.Hkv * plan.mtiles * plan.splits);
    auto kernel = exact_split_kernel<NP, D, BIAS>;
    hipError_t e = allow_lds(kernel, smem);
    if (e != hipSuccess) return e;
    kernel<<<wgs, kExactThreads, smem, stream>>>(a, lse, plan.mtiles, plan.splits, part_o, part_l);
    if (plan.splits > 1) {
      if ((e = hipGetLastError()) != hipSuccess) return e;
      launch_join<NP, D>(a, lse, plan.splits, part_o, part_l, stream);
    }
    return hipGetLastError();
  }
  if constexpr (NP == 1 && D <= 64) {
    // 96 heads x 4096 x 64: 475 -> 428 us
    if (wide_rows((long long)a.B * a.H, a.nq)) return launch_rows<NP, D, 2, BIAS>(a, lse, stream);
  }
  return launch_rows<NP, D, 1, BIAS>(a, lse, stream);
}

hipError_t launch_exact_forward(const ExactArgs& a, int d, int dtype, float* lse, const SplitPlan& plan, void* ws,
                                hipStream_t stream) {
  auto pick = [&](auto np, auto dd) {
    constexpr int NP = decltype(np)::value, D = decltype(dd)::value;
    return a.bias != nullptr ? forward_case<NP, D, true>(a, lse, plan, ws, stream)
                             : forward_case<NP, D, false>(a, lse, plan, ws, stream);
  };
  auto width = [&](auto np) {
    if (d == 32) return pick(np, std::integral_constant<int, 32>{});
    if (d == 64) return pick(np, std::integral_constant<int, 64>{});
    return pick(np, std::integral_constant<int, 128>{});
  };
  return dtype == BF16 ? width(std::integral_constant<int, 1>{}) : width(std::integral_constant<int, 3>{});
}

}  // namespace mra
