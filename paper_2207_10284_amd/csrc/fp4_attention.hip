// Attention over the 4-bit cache (mra_layer.h).
//
// As in exact_fwd.hip S is formed transposed, S^T = K Q^T, so that a lane's scores of one
// query are the B operand of O^T += V^T P^T as they are, and the softmax runs against a reference
// that moves only when a tile outgrows it. The rows of a key head, all queries of all its heads,
// are one list: row m is query m / group of head hk group + m % group.
//
// fp4_rows_kernel: a workgroup's waves (eight, or four) take 32 rows each and walk the keys
// together, 64 at a time. Codes come through registers and are converted once per workgroup, to
// bfloat16 rows in LDS in the order and swizzle of the exact kernels, whose transposing reads give the second
// product's operand. What bounds it is a stage's vector work (exponentials, packing, conversion) beside its matrix work, two waves a
// SIMD: 2 x 16 heads on 4, 512 queries on up to 16384 keys x 128 bfloat16, with the join's 8 us, 119 to 146 us by the lengths
// (equal ones 850 to 890 TFLOP/s, 63 to 66% of a large product's rate, unequal ones 710 to 840: each sequence has the same number of
// parts; matrix cores busy 36%, vector ALU 34%, waves waiting 26% of their time); 8 x 12 heads x 2048 x 64, causal, 72 to 77 us
// (matrix cores busy 27%, vector ALU 56%, waves waiting 29%).
//
// fp4_token_kernel: few rows, single tokens above all. A wave takes 16 rows and 32 keys at a time on the
// 16x16x32 matrix instructions. Keys go from memory to registers as the first product takes them; values
// pass through the wave's own part of LDS, which transposes them. A workgroup's waves take every
// kTokenWaves-th tile, and several workgroups may share the rows, each with a part of the keys
// (exact_join_kernel adds them). What bounds it is the cache's bytes and, as much, the chain from tile to tile within a
// wave: one token of 32 x 12 heads on up to 4096 keys x 64, 20 us (80 MB, 4.0 TB/s; loads alone, without any products, take
// 2.5 us less) and the join 4; 4 x 16 heads on 4, up to 32768 x 128, 13 to 15 us (53 MB) and the join 4.
//
// Weights of bfloat16 calls are rounded to bfloat16 for the second product, and their sums are of the rounded ones: a weight is off
// by 2^-9 at most, as much as the result's own rounding, and the 2-norm of a result's error is 2.0 to 2.3e-3 of the result's where
// that rounding alone gives 1.6e-3. As sums of two bfloat16 values they cost single tokens 4 to 6% (32 x 12 heads on up to
// 4096 x 64: 26.7 -> 27.6 us, 4 x 16 heads on 4, up to 32768 x 128: 18.5 -> 19.7) and prompts 24 to 40% (the two calls
// above: 137 -> 171, 86 -> 120). Float32 queries are for the caller who wants more.
#include "exact_rows.h"
#include "fp4_tile.h"

namespace mra {

namespace {

__device__ __forceinline__ int cached_keys(const CacheAttentionArgs& a, int b) {
  return min(max(a.lengths[b], 0), a.c.cap);
}

// Position of query 0 of sequence b.
__device__ __forceinline__ int first_query(const CacheAttentionArgs& a, int b, int keys) {
  constexpr int kFar = 1 << 29;
  return a.q_start == nullptr ? keys - a.nq : min(max(a.q_start[b], -kFar), kFar);
}

// The pages of a wave's tiles of 32 keys, every step-th from `tile` on: a lane holds one entry of the table, loaded
// once for 64 of them, so that no turn of a loop waits for the table.
struct PageList {
  int entry, tile, step, used;
  __device__ __forceinline__ void load(const CacheArgs& c, int b) {
    const int t = tile + lane_id() * step;         // tiles below 2^21, steps below 2^9
    entry = t < c.cap >> 5 ? c.table[(long long)b * c.max_pages + (t >> (c.page_log2 - 5))] : -1;
    used = 0;
    wait_loads<0>();                               // here, not at each use beside the loads in flight
  }
  // Of the next tile; null: no page, or past the table.
  __device__ __forceinline__ const char* next(const CacheArgs& c, int b, int hk) {
    if (used == 64) load(c, b);
    const int page = __builtin_amdgcn_readlane(entry, used++);
    tile += step;
    return (unsigned)page < (unsigned)c.pages ? c.data + ((long long)page * c.Hkv + hk) * c.head_bytes : nullptr;
  }
};

// A stage's 64 keys of one head on their way from the cache to LDS, by T threads.
template <int D, int T>
struct CacheStage {
  using Pg = Fp4Page<D>;
  static constexpr int kKeys = 128 * D;            // bytes of the keys in LDS; the values take as many
  using Unit = Fp4StageUnit<D, T>;
  static constexpr int N = Unit::N;
  u32x4 w[N];
  uint32_t e[N];

  // pg: the pages of the two halves of the stage, null where no key counts
  __device__ __forceinline__ void load(const char* (&pg)[2], int k0, int size, int tid) {
    const int slot0 = k0 & (size - 1), slot1 = (k0 + 32) & (size - 1);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const Unit u(n, tid);
      if (u.x > 1) continue;
      const char* p = u.r < 32 ? pg[0] : pg[1];
      const int slot = (u.r < 32 ? slot0 : slot1) + u.r % 32;
      w[n] = u32x4{0, 0, 0, 0};
      e[n] = 127;
      if (p != nullptr) {
        w[n] = *reinterpret_cast<const u32x4*>(p + Pg::codes(u.x, size) + slot * (D / 2) + u.blk * 16);
        e[n] = (uint8_t)p[Pg::steps(u.x, size) + slot * Pg::NB + u.blk];
      }
    }
  }

  // ok: the keys that count; the steps of others may be anything
  __device__ __forceinline__ void store(char* lds, const RowBits<64>& ok, int tid) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const Unit u(n, tid);
      if (u.x > 1) continue;
      const float step = fp4_step(ok.all() || ok.row(u.r) ? e[n] : 127);
      char* to = lds + u.x * kKeys + (u.r >> 5) * kTileBytes<D>;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<u32x4*>(to + raw_offset<D, exact_swz<D>>(u.r & 31, 32 * u.blk + 8 * j)) = fp4_decode(w[n][j], step);
    }
  }
};

// A lane's part of a query that holds an infinity or a NaN becomes NaN whole, so that every score of the query is (an
// infinity alone may give nothing but scores of -infinity, as float32's planes never do). Sums, and with them Z
// and L, are NaN then; what has no key has sums of 0.
template <int C>
__device__ __forceinline__ void spread_nan(u32x4 (&q)[C]) {
  uint32_t high = 0;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) high |= (q[c][e] & 0x7fff7fffu) + 0x00800080u;   // bit 15 of a half: an exponent of ones
  const bool bad = (high & 0x80008000u) != 0;
  if (__ballot(bad) == 0) return;
#pragma unroll
  for (int c = 0; c < C; ++c) q[c] = bad ? u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u} : q[c];
}

// Weights of the scores s of a stage's two tiles (log2 logits s mul; -inf: does not count) and their sum; a
// reference that they outgrow is moved first (see tile_weights).
template <int D>
__device__ __forceinline__ void stage_weights(FwdRow<1, D>& row, const f32x16 (&s)[2], float mul, Packed<1> (&w)[2]) {
  float t[2];
  bool again = false;
  while (true) {
    const float c = again && row.ref == -INFINITY ? 0.0f : -row.ref;
#pragma unroll
    for (int x = 0; x < 2; ++x) t[x] = row.weights(s[x], mul, c, w[x]);
    if (again || __ballot(!(t[0] <= kCap && t[1] <= kCap)) == 0) break;
#pragma unroll
    for (int x = 0; x < 2; ++x) row.move(s[x], mul, 0.0f);
    again = true;
  }
  row.sum += t[0] + t[1];
}

}  // namespace

template <int NP, int D, int W>
__global__ __launch_bounds__(W * kWave) void fp4_rows_kernel(CacheAttentionArgs a, int mtiles, int splits,
                                                                 float* __restrict__ part_o, float* __restrict__ part_l) {
  using St = CacheStage<D, W * kWave>;
  constexpr int KC = D / 16, NT = D / 32, BUF = 2 * St::kKeys;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int tid = threadIdx.x, lane = lane_id(), w = wave_uniform(tid / kWave);
  // The last rows first, which are the longest of causal calls. Workgroups go round the eight XCDs in turn: a part
  // of a head stays on one XCD, whose L2 its row tiles share; parts that are few are shifted from one level to the next, or an XCD
  // had one or two of them, however short their sequences.
  const int units = a.B * a.c.Hkv * splits, level = blockIdx.x / units, at_level = blockIdx.x - level * units;
  const int mt = mtiles - 1 - level, unit = units < 32 ? (at_level + level) % units : at_level;
  const int bk = unit / splits, sp = unit - bk * splits;
  const int b = bk / a.c.Hkv, hk = bk - b * a.c.Hkv, size = 1 << a.c.page_log2;
  const int rows = a.nq * a.group, row0 = (mt * W + w) * 32;
  const int m = row0 + (lane & 31), mc = min(m, rows - 1), i = mc / a.group, h = hk * a.group + (mc - i * a.group);
  const int limit = cached_keys(a, b), start = first_query(a, b, limit);
  const int pos = start + i;                                  // of this lane's row
  const int pos_first = start + min(row0, rows - 1) / a.group, pos_last = start + min(row0 + 31, rows - 1) / a.group;
  const int kend = a.causal ? min(limit, start + min((mt + 1) * W * 32 - 1, rows - 1) / a.group + 1) : limit;
  const int stages = kend > 0 ? (kend + 63) / 64 : 0;
  const int n0 = (int)((long long)stages * sp / splits), n1 = (int)((long long)stages * (sp + 1) / splits);

  TileAddr<D> at;
  at.init(smem);
  FwdRow<NP, D> row[1];
  load_operand<NP, D>(a.q.p + b * a.q.sb + h * a.q.sh + i * a.q.sn, m < rows, row[0].qf);
  row[0].init();

  auto pages = [&](int k0, const char* (&pg)[2]) {
#pragma unroll
    for (int x = 0; x < 2; ++x) pg[x] = k0 + 32 * x < kend ? fp4_page(a.c, b, hk, k0 + 32 * x) : nullptr;
  };
  // the keys of a stage that count for some row
  auto counted = [&](int k0, const char* const (&pg)[2]) {
    return RowBits<64>{__ballot(k0 + lane < kend && (lane < 32 ? pg[0] : pg[1]) != nullptr)};
  };
  St st;
  RowBits<64> ok{}, ok1{};                         // of this stage and the next
  const char* pg[2] = {nullptr, nullptr};          // of the next stage to load: its loads do not wait for the table
  auto load = [&](int n) {
    st.load(pg, 64 * n, size, tid);
    ok1 = counted(64 * n, pg);
    pages(64 * (n + 1), pg);
  };
  if (n0 < n1) {
    pages(64 * n0, pg);
    load(n0);
    ok = ok1;
    st.store(smem, ok, tid);
    if (n0 + 1 < n1) load(n0 + 1);
  }
  if constexpr (NP == 1) spread_nan(row[0].qf[0]);
  __syncthreads();
  // Of a SIMD's two waves one converts the next stage before its products and the other after them, so that
  // one's vector work runs beside the other's matrix work (16 heads on 4 x 8192 x 128 causal: 196 -> 186 us).
  const bool early = W == 8 && w >= W / 2;
  auto stage = [&](int n, auto B) {
    constexpr int kbuf = B * BUF;
    const bool more = n + 1 < n1;
    const RowBits<64> next = ok1;
    auto refill = [&] {
      st.store(smem + (1 - B) * BUF, next, tid);
      if (n + 2 < n1) load(n + 2);
    };
    if (more && early) refill();
    if constexpr (NP == 1) {
      // both tiles at once: one's products beside the other's exponentials
      const int k0 = 64 * n;
      if (ok.w != 0 && !(a.causal && k0 > pos_last)) {        // some key counts for the wave
        f32x16 s[2] = {splat16(0.0f), splat16(0.0f)};
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
          for (int x = 0; x < 2; ++x) s[x] = mfma16(at.row(kbuf + x * kTileBytes<D>, c), row[0].qf[0][c], s[x]);
        if (!ok.all() || (a.causal && k0 + 63 > pos_first)) {
#pragma unroll
          for (int x = 0; x < 2; ++x)
            select_rows(s[x], a.causal ? ok.tile(x) & low_bits(pos - k0 - 32 * x + 1) : ok.tile(x), -INFINITY);
        }
        Packed<1> pw[2];
        auto value = [&](int x, int u, int t) { return at.trans(kbuf + St::kKeys + x * kTileBytes<D>, u, t); };
        // at d <= 64 the first values are on their way while the weights are formed (16 heads on 4 x 8192 x 64 causal:
        // 131 -> 123 us; at 128, where registers are short, 186 -> 212)
        constexpr bool kAhead = D <= 64;
        u32x4 first[kAhead ? NT : 1];
        if constexpr (kAhead) {
#pragma unroll
          for (int t = 0; t < NT; ++t) first[t] = value(0, 0, t);
          __builtin_amdgcn_sched_barrier(0);
        }
        stage_weights(row[0], s, a.scale_log2, pw);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t)
              row[0].o[t] = mfma16(kAhead && x + u == 0 ? first[kAhead ? t : 0] : value(x, u, t), pw[x].w[0][u], row[0].o[t]);
      }
    } else {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint32_t kb = ok.tile(x);
        const int k0 = 64 * n + 32 * x;
        if (kb == 0 || (a.causal && k0 > pos_last)) continue;   // no key counts for the wave
        f32x16 s[1] = {splat16(0.0f)};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const u32x4 k = at.row(kbuf + x * kTileBytes<D>, c);
#pragma unroll
          for (int q = NP - 1; q >= 0; --q) s[0] = mfma16(k, row[0].qf[q][c], s[0]);
        }
        const uint32_t bits = a.causal ? kb & low_bits(pos - k0 + 1) : kb;
        if (kb != ~0u || (a.causal && k0 + 31 > pos_first)) select_rows(s[0], bits, -INFINITY);
        const float mul[1] = {a.scale_log2}, add[1] = {0.0f};
        Packed<NP> pw[1];
        tile_weights<NP, D, 1>(row, s, mul, add, pw);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const u32x4 v = at.trans(kbuf + St::kKeys + x * kTileBytes<D>, u, t);
#pragma unroll
            for (int q = NP - 1; q >= 0; --q) row[0].o[t] = mfma16(v, pw[0].w[q][u], row[0].o[t]);
          }
      }
    }
    if (more && !early) refill();
    ok = next;
    __syncthreads();
  };
  for (int n = n0; n < n1; n += 2) {
    stage(n, std::integral_constant<int, 0>{});
    if (n + 1 < n1) stage(n + 1, std::integral_constant<int, 1>{});
  }
  const float den = halves_sum(row[0].sum);
  if (splits > 1) {
    const long long pr = ((long long)sp * a.B * a.c.Hkv + bk) * rows + mc;   // the partial row
    store_rows<3, D>(row[0].o, 1.0f, reinterpret_cast<char*>(part_o + pr * D), m < rows);
    if (lane < 32 && m < rows) {
      part_l[2 * pr] = row[0].ref;
      part_l[2 * pr + 1] = den;
    }
    return;
  }
  store_rows<NP, D>(row[0].o, den > 0.0f ? 1.0f / den : 0.0f, a.out.p + b * a.out.sb + h * a.out.sh + i * a.out.sn,
                    m < rows);
  if (a.lse != nullptr && lane < 32 && m < rows)
    a.lse[((long long)b * a.H + h) * a.nq + i] = den == 0.0f ? -INFINITY : (log2f(den) + row[0].ref) * kLn2;
}

// ---- few rows

// Four waves and two workgroups a CU: eight waves and one 31 us, two and four 29, four and one 29, where these take 25.
constexpr int kTokenWaves = 4;
constexpr int kTokenRows = 16;

__device__ __forceinline__ f32x4 mfma4(const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// op over the four lanes of a column (lane, lane ^ 16, lane ^ 32, lane ^ 48).
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// 32 keys of one head as the wave's lanes hold them: lane (g, i) = (lane / 16, lane % 16) has channels
// g D/4 .. of keys 8 (i / 4) + 4 x + i % 4 (x = 0, 1), so that register r of the scores of x is key
// 8 g + 4 x + r of column i; and of the values of keys 16 x + i.
template <int D>
struct CacheTile {
  using Pg = Fp4Page<D>;
  uint32_t w[2][2][D / 32], e[2][2];               // keys and values, x

  static __device__ __forceinline__ int row(int value, int x) { return fp4_tile_row(value, x, lane_id() & 15); }

  // A lane's offsets are the same for every tile: uniform bases, so that a load needs no vector instruction.
  __device__ __forceinline__ void load(const char* page, int slot, int size) {
    const int g = lane_id() >> 4;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const char* codes = page + (Pg::codes(v, size) + slot * (D / 2));
      const char* steps = page + (Pg::steps(v, size) + slot * Pg::NB);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const char* p = codes + (uint32_t)(row(v, x) * (D / 2) + g * (D / 8));
        if constexpr (D == 128) {
          const u32x4 q = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
          for (int n = 0; n < 4; ++n) w[v][x][n] = q[n];
        } else if constexpr (D == 64) {
          const u32x2 q = *reinterpret_cast<const u32x2*>(p);
          w[v][x][0] = q[0];
          w[v][x][1] = q[1];
        } else {
          w[v][x][0] = *reinterpret_cast<const uint32_t*>(p);
        }
        e[v][x] = (uint8_t)steps[(uint32_t)(row(v, x) * Pg::NB + g * Pg::NB / 4)];
      }
    }
  }
};

// A wave's 32 values of D channels in LDS (256-byte aligned), laid out by fp4_value_place.
template <int D>
struct ValueTile {
  uint32_t to, from[2];                            // this lane's first chunk of a row; transposed rows + 0 and + 4

  __device__ __forceinline__ void init(const char* lds) {
    const int lane = lane_id(), g = lane >> 4, i = lane & 15;
    to = lds_addr(lds) + fp4_value_place<D>(i, g * (D / 4));
#pragma unroll
    for (int e = 0; e < 2; ++e) from[e] = lds_addr(lds) + fp4_value_place<D>(8 * g + 4 * e + (i >> 2), 4 * (i & 3));
  }
  // chunk n (8 channels) of this lane's row 16 x + lane % 16
  __device__ __forceinline__ void put(int x, int n, const u32x4& v) const {
    *(__attribute__((address_space(3))) u32x4*)(lds_ptr)((to ^ 16u * n) + x * 16 * 2 * D) = v;
  }
  // the A operand of channels 16 t ..: of channel 16 t + lane % 16, rows 8 (lane / 16) + 0 .. 7
  __device__ __forceinline__ u32x4 get(int t) const {
    u32x2 x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                           (__attribute__((address_space(3))) s16x4*)(lds_ptr)(from[e] ^ 32u * t)));
    return u32x4{x[0][0], x[0][1], x[1][0], x[1][1]};
  }
};

// The running softmax of 16 rows, a column each (as FwdRow).
template <int NP, int D>
struct TokenRows {
  u32x4 qf[NP][D / 32];
  f32x4 o[D / 16];
  float ref, sum;

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int t = 0; t < D / 16; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    ref = -INFINITY;
    sum = 0.0f;
  }

  __device__ __forceinline__ void load_queries(const char* row, bool on) {
    const char* p = row + (lane_id() >> 4) * (D / 4) * (NP == 1 ? 2 : 4);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      if constexpr (NP == 1) {
        qf[0][c] = on ? reinterpret_cast<const u32x4*>(p)[c] : u32x4{0, 0, 0, 0};
      } else {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = on ? reinterpret_cast<const float*>(p)[8 * c + e] : 0.0f;
        u32x4 pl[3];
        split8(f, pl);
#pragma unroll
        for (int q = 0; q < 3; ++q) qf[q][c] = pl[q];
      }
    }
  }

  // weights exp2(s mul - at) of a lane's eight keys as the next operand's planes, and their sum
  __device__ __forceinline__ float weights(const float (&s)[8], float mul, float at, u32x4 (&w)[NP]) const {
    float p[8], t = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, -at));
    if constexpr (NP == 1) {
      const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bf16x2 b;
        b[0] = (__bf16)p[2 * e];
        b[1] = (__bf16)p[2 * e + 1];
        w[0][e] = __builtin_bit_cast(uint32_t, b);
        t = __builtin_amdgcn_fdot2_f32_bf16(b, ones, t, false);
      }
    } else {
      split8(p, w);
#pragma unroll
      for (int r = 0; r < 8; ++r) t += p[r];
    }
    return t;
  }

  // Weights of a tile's scores; a reference that they outgrow is moved first, in all lanes of its column.
  __device__ __forceinline__ void tile(const float (&s)[8], float mul, u32x4 (&w)[NP]) {
    float t = weights(s, mul, ref, w);
    if (__ballot(!(t <= kCap)) != 0) {             // also where ref is -inf
      float mx = s[0];
#pragma unroll
      for (int r = 1; r < 8; ++r) mx = fmaxf(mx, s[r]);
      mx = column_max(mx) * mul;
      const float next = mx > ref ? mx + kMargin : ref;
      const float f = next == ref ? 1.0f : __builtin_amdgcn_exp2f(ref - next);
#pragma unroll
      for (int x = 0; x < D / 16; ++x) o[x] *= f;
      sum *= f;
      ref = next;
      t = weights(s, mul, ref == -INFINITY ? 0.0f : ref, w);    // no key yet: every s is -inf
    }
    sum += t;
  }
};

template <int NP, int D>
__global__ __launch_bounds__(kTokenWaves * kWave) void fp4_token_kernel(CacheAttentionArgs a, int mtiles, int splits,
                                                                        float* __restrict__ part_o,
                                                                        float* __restrict__ part_l) {
  constexpr int W = kTokenWaves, KC = D / 32, NT = D / 16;
  // the waves' values, at the end their sums
  static_assert(64 * D == NT * kWave * 16, "as large");
  __shared__ __attribute__((aligned(256))) char lds[W * 64 * D];
  f32x4(*merged)[NT][kWave] = reinterpret_cast<f32x4(*)[NT][kWave]>(lds);
  __shared__ float refs[W][kWave], sums[W][kWave];
  const int lane = lane_id(), w = wave_uniform(threadIdx.x / kWave), g4 = lane >> 4;
  const int g = blockIdx.x;
  const int sp = g % splits, mt = g / splits % mtiles, bk = g / splits / mtiles;
  const int b = bk / a.c.Hkv, hk = bk - b * a.c.Hkv, size = 1 << a.c.page_log2;
  const int rows = a.nq * a.group, row0 = mt * kTokenRows;
  const int m = row0 + (lane & 15), mc = min(m, rows - 1), i = mc / a.group, h = hk * a.group + (mc - i * a.group);
  // A workgroup takes every splits-th group of W tiles: which ones does not depend on the length, so neither the look
  // into the table nor the first tile waits for that.
  PageList list{0, sp * W + w, splits * W, 0};
  list.load(a.c, b);
  CacheTile<D> next;
  int t = sp * W + w;
  const char* page = list.next(a.c, b, hk);        // of the tile in next
  if (page != nullptr) next.load(page, 32 * t & (size - 1), size);
  TokenRows<NP, D> row;
  row.load_queries(a.q.p + b * a.q.sb + h * a.q.sh + i * a.q.sn, m < rows);
  row.init();
  ValueTile<D> values;
  values.init(lds + w * 64 * D);
  const int limit = cached_keys(a, b), start = first_query(a, b, limit);
  const int pos = start + i, pos_first = start + row0 / a.group;
  const int pos_last = start + min(row0 + kTokenRows - 1, rows - 1) / a.group;
  const int kend = a.causal ? min(limit, pos_last + 1) : limit;
  const int tiles = kend > 0 ? (kend + 31) / 32 : 0;
  if constexpr (NP == 1) spread_nan(row.qf[0]);
  for (; t < tiles; t += splits * W) {
    const CacheTile<D> tile = next;
    const int k0 = 32 * t, end = page != nullptr ? kend : 0;  // no page: no key
    page = t + splits * W < tiles ? list.next(a.c, b, hk) : nullptr;
    if (page != nullptr) next.load(page, 32 * (t + splits * W) & (size - 1), size);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      // the steps of keys that do not count may be anything
      const float step = fp4_step(k0 + CacheTile<D>::row(1, x) < end ? tile.e[1][x] : 127);
#pragma unroll
      for (int n = 0; n < KC; ++n) values.put(x, n, fp4_decode(tile.w[1][x][n], step));
    }
    float s[8];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
      const float step = fp4_step(tile.e[0][x]);
#pragma unroll
      for (int n = 0; n < KC; ++n) {
        const u32x4 k = fp4_decode(tile.w[0][x][n], step);
#pragma unroll
        for (int q = NP - 1; q >= 0; --q) c = mfma4(k, row.qf[q][n], c);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) s[4 * x + r] = c[r];
    }
    if (k0 + 32 > end || (a.causal && k0 + 31 > pos_first)) {
      const uint32_t bits = low_bits((a.causal ? min(end, pos + 1) : end) - k0 - 8 * g4);
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r] = bits >> r & 1 ? s[r] : -INFINITY;
    }
    u32x4 pw[NP];
    row.tile(s, a.scale_log2, pw);
    wave_lds_sync();
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const u32x4 v = values.get(x);
#pragma unroll
      for (int q = NP - 1; q >= 0; --q) row.o[x] = mfma4(v, pw[q], row.o[x]);
    }
    wave_lds_sync();
  }
  // the waves' sums relative to the largest reference, added in wave order, each wave some of the channels
  float sum = column_sum(row.sum);
  refs[w][lane] = row.ref;
  sums[w][lane] = sum;
  __syncthreads();                                 // the values are idle
  float top = refs[0][lane];
#pragma unroll
  for (int x = 1; x < W; ++x) top = fmaxf(top, refs[x][lane]);
  auto factor = [&](float ref) { return ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref - top); };
  const float f = factor(row.ref);
#pragma unroll
  for (int x = 0; x < NT; ++x) merged[w][x][lane] = row.o[x] * f;
  sum = 0.0f;
#pragma unroll
  for (int p = 0; p < W; ++p) sum += sums[p][lane] * factor(refs[p][lane]);
  __syncthreads();
  if (m >= rows) return;
  const float inv = splits > 1 ? 1.0f : sum > 0.0f ? 1.0f / sum : 0.0f;
  const long long pr = ((long long)sp * a.B * a.c.Hkv + bk) * rows + m;   // the partial row
  char* to = splits > 1 ? reinterpret_cast<char*>(part_o + pr * D) : a.out.p + b * a.out.sb + h * a.out.sh + i * a.out.sn;
#pragma unroll
  for (int y = 0; y < (NT + W - 1) / W; ++y) {
    const int x = y * W + w;
    if (x >= NT) break;
    f32x4 o = merged[0][x][lane];
#pragma unroll
    for (int p = 1; p < W; ++p) o += merged[p][x][lane];
    const float z[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    const int c = 16 * x + 4 * g4;
    if (NP == 1 && splits == 1) store4<1>(to + 2 * c, z);
    else store4<3>(to + 4 * c, z);
  }
  if (g4 != 0 || w != 0) return;
  if (splits > 1) {
    part_l[2 * pr] = top;
    part_l[2 * pr + 1] = sum;
  } else if (a.lse != nullptr) {
    a.lse[((long long)b * a.H + h) * a.nq + i] = sum == 0.0f ? -INFINITY : (log2f(sum) + top) * kLn2;
  }
}

// Waves of fp4_rows_kernel: eight where a stage's conversion costs most and registers allow it.
constexpr int row_waves(int np, int d) { return np == 1 && d == 128 ? 8 : 4; }

// The token kernel serves up to 64 rows a key head, and more where its tiles (16 rows x keys) are few: the other's
// stages take 2 to 3 us however little there is to do (bfloat16, d = 64, us; rows kernel, token kernel):
//   64 heads x 4096 keys, 16 rows: 20, 13   64 rows: 23, 21   96 rows: 25, 24   128 rows: 26, 28
//   8 heads x 4096 keys, 128 rows: 17, 12   256 rows: 19, 15   512 rows: 21, 20
//   4 heads x 16384 keys, 128 rows: 19, 16   256 rows: 23, 21   512 rows: 31, 33
// Where the rows' workgroups are fewer than two per CU (one of eight waves) several share the keys of the same
// rows, each at least 256; in the token kernel only beyond 1024 keys, below which adding their parts costs more than it
// saves (bfloat16, d = 64, one token, us, alone and shared: 16 heads x 512 keys 6.5, 10; 256 heads x 1024 keys 8.9, 11.9;
// 16 heads x 1024 keys 8.4, 9.6, at d = 128 10.4, 9.6; 16 heads x 2048 keys 13, 9).
CachePlan cache_plan(int B, int Hkv, long long rows, int cap, int d, int dtype) {
  CachePlan p{};
  const long long heads = (long long)B * Hkv, tiles = heads * ((rows + kTokenRows - 1) / kTokenRows);
  p.few = rows <= 64 || tiles <= (1 << 20) / (cap > 0 ? cap : 1);
  const int waves = p.few ? kTokenWaves : row_waves(dtype == BF16 ? 1 : 3, d);
  p.mtiles = (int)(p.few ? (rows + kTokenRows - 1) / kTokenRows : (rows + 32 * waves - 1) / (32 * waves));
  const long long wgs = heads * p.mtiles, most = p.few && cap <= 1024 ? 1 : (cap + 255) / 256;
  long long want = ((waves == 8 ? 1 : 2) * kCus + wgs - 1) / wgs;
  if (want > most) want = most;
  if (want > 64) want = 64;
  p.splits = want > 1 ? (int)want : 1;
  if (p.splits > 1) p.bytes = (size_t)p.splits * heads * rows * (d + 2) * sizeof(float);
  return p;
}

template <int NP, int D>
static hipError_t attention_case(const CacheAttentionArgs& a, const CachePlan& plan, void* ws, hipStream_t stream) {
  const long long heads = (long long)a.B * a.c.Hkv, rows = (long long)a.nq * a.group;
  const unsigned wgs = (unsigned)(heads * plan.mtiles * plan.splits);
  float* part_o = static_cast<float*>(ws);
  float* part_l = part_o + (plan.splits > 1 ? plan.splits * heads * rows * D : 0);
  if (plan.few) {
    fp4_token_kernel<NP, D><<<wgs, kTokenWaves * kWave, 0, stream>>>(a, plan.mtiles, plan.splits, part_o, part_l);
  } else {
    constexpr int W = row_waves(NP, D);
    constexpr size_t smem = 4 * CacheStage<D, W * kWave>::kKeys;
    auto kernel = fp4_rows_kernel<NP, D, W>;
    const hipError_t e = allow_lds(kernel, smem);
    if (e != hipSuccess) return e;
    kernel<<<wgs, W * kWave, smem, stream>>>(a, plan.mtiles, plan.splits, part_o, part_l);
  }
  if (plan.splits > 1) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ExactArgs x{};
    x.out = a.out;
    x.B = a.B;
    x.H = a.H;
    x.Hkv = a.c.Hkv;
    x.group = a.group;
    x.nq = a.nq;
    launch_join<NP, D>(x, a.lse, plan.splits, part_o, part_l, stream);
  }
  return hipGetLastError();
}

hipError_t launch_cache_attention(const CacheAttentionArgs& a, int d, int dtype, const CachePlan& plan, void* ws,
                                  hipStream_t stream) {
  auto width = [&](auto np) {
    constexpr int NP = decltype(np)::value;
    if (d == 32) return attention_case<NP, 32>(a, plan, ws, stream);
    if (d == 64) return attention_case<NP, 64>(a, plan, ws, stream);
    return attention_case<NP, 128>(a, plan, ws, stream);
  };
  return dtype == BF16 ? width(std::integral_constant<int, 1>{}) : width(std::integral_constant<int, 3>{});
}

}  // namespace mra
