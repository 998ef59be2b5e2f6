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
    ref[x] = s < splits ? part_l[2 * at] : -INFINITY;
    l[x] = part_l[2 * at + 1];
  }
  float top = ref[0], sum = 0.0f;
#pragma unroll
  for (int x = 1; x < kJoin; ++x) top = fmaxf(top, ref[x]);
  f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [](const f32x4& o, float l, float ref, float top, f32x4& z, float& sum) {
    if (ref == -INFINITY) return;                  // no key
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
    lse[((long long)b * a.H + h) * a.nq + i] = sum > 0.0f ? (log2f(sum) + top) * kLn2 : -INFINITY;
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
      int groups = 1;                              // at most 64 splits: at most eight, of at most 32 threads
      while (groups * kJoin < plan.splits) groups *= 2;
      const int per = 256 / (D / 4 * groups);
      exact_join_kernel<NP, D><<<(unsigned)((rows + per - 1) / per), 256, 0, stream>>>(a, lse, plan.splits, groups,
                                                                                      part_o, part_l);
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
