// Device code shared by the exact-attention kernels: staging of 32-row tiles
// in LDS, matrix-core operands and products, masks and the position bias.
//
// Operands are NP bfloat16 planes: one for bfloat16 tensors, three whose sum
// the value is for float32 ones (tile_ops.h). A tile is 32 rows x D of one plane,
// row-major under the swizzle of the gradient passes, which serves row and
// transposed reads without bank conflicts. Rows go from global memory through
// registers, where rows that do not count become zero (what they hold may be
// anything) and float32 values are split, once per workgroup instead of once per
// wave that reads them.
#pragma once

#include "common.h"
#include "exact_kernels.h"
#include "tile_ops.h"

namespace mra {

constexpr int kExactWaves = 4;                     // waves per workgroup
constexpr int kExactThreads = kExactWaves * kWave;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char* lds_ptr;

template <int D>
__host__ __device__ constexpr int exact_swz(int r) {
  return D == 128 ? 4 * (r & 3) + ((r >> 2) & 3) : (D == 64 ? 4 * ((r >> 1) & 1) + ((r >> 2) & 3) : (r >> 2) & 3);
}

template <int D>
constexpr int kTileBytes = 64 * D;                 // 32 rows of one plane

// Rows per stage of the workgroup's shared loops.
template <int NP, int D>
constexpr int kStageRows = NP == 1 || D == 32 ? 64 : 32;

// Which of a stage's R rows count: row r is bit r.
template <int R>
struct RowBits {
  static_assert(R == 32 || R == 64, "one ballot");
  static constexpr uint64_t kAll = R == 64 ? ~uint64_t(0) : (uint64_t(1) << 32) - 1;
  uint64_t w;
  __device__ __forceinline__ uint32_t tile(int i) const { return (uint32_t)(w >> (32 * i)); }
  __device__ __forceinline__ bool all() const { return w == kAll; }
  __device__ __forceinline__ bool row(int r) const { return (w >> r) & 1; }
};

// R rows of D elements moved by T threads from global memory to LDS tiles: plane
// p of rows 32 i .. 32 i + 31 at (p R/32 + i) kTileBytes. Loads go to registers
// (load), so that their latency passes during the previous stage's products;
// store() writes them.
template <int NP, int D, int R, int T>
struct Stage {
  static constexpr int CPR = D / 8;                // units of eight elements per row
  static constexpr int N = R * CPR / T;
  static constexpr int LB = NP == 1 ? 1 : 2;       // 16-byte loads per unit
  static constexpr int kBytes = NP * R * D * 2;
  static_assert(N >= 1 && R * CPR % T == 0, "whole units per thread");
  u32x4 v[N][LB];
  static constexpr int ROWS = T / CPR;             // rows that the threads' units i cover
  static_assert(T % CPR == 0, "whole rows");
  uint32_t off;                                    // of this thread's units from their first row on

  __device__ __forceinline__ void init(long long sn, int tid) {
    off = (uint32_t)(tid / CPR) * (uint32_t)sn + (tid % CPR) * LB * 16;
  }

  // rows row0 .. row0 + R - 1; those at or past limit are zero. One buffer per unit,
  // whose range ends with the last row (row strides are below 2^25 bytes), so a load needs no
  // vector instruction for its address or its bounds.
  __device__ __forceinline__ void load(const char* base, long long sn, int row0, int limit) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row0 + i * ROWS, rows = min(limit - r, ROWS);
      const i32x4 rs = buffer_rsrc(base + (long long)r * sn, rows > 0 ? (unsigned)(rows - 1) * (unsigned)sn + CPR * LB * 16 : 0u);
#pragma unroll
      for (int e = 0; e < LB; ++e) v[i][e] = __builtin_bit_cast(u32x4, mra_raw_buffer_load_f32x4(rs, (int)off + 16 * e, 0, 0));
    }
  }

  // rows that do not count become zero
  __device__ __forceinline__ void store(char* lds, const RowBits<R>& ok, int tid) {
    if (!ok.all()) {                               // wave-uniform
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t keep = ok.row((i * T + tid) / CPR) ? ~0u : 0u;
#pragma unroll
        for (int e = 0; e < LB; ++e)
#pragma unroll
          for (int x = 0; x < 4; ++x) v[i][e][x] &= keep;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * T + tid, r = u / CPR;
      char* dst = lds + (r >> 5) * kTileBytes<D> + raw_offset<D, exact_swz<D>>(r & 31, 8 * (u % CPR));
      if constexpr (NP == 1) {
        *reinterpret_cast<u32x4*>(dst) = v[i][0];
      } else {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(v[i][e / 4][e % 4]);
        u32x4 pl[3];
        split8(f, pl);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4*>(dst + p * (R / 32) * kTileBytes<D>) = pl[p];
      }
    }
  }
};

// Head and block of workgroup p of heads x blocks. Workgroups go round the eight XCDs
// in turn (see xcd_remap): eight heads at a time, an XCD takes one head's blocks in
// their order, so that they share its L2. The last heads % 8 heads are shared by all
// XCDs: causal ones block by block, since a head's blocks then differ in length and a
// range of them per XCD leaves some idle (dK and dV of 4 key heads x 16384 x 128: the
// first half of a head's blocks has three quarters of the work), others in ranges.
struct HeadBlock {
  int head, block;
};
__device__ __forceinline__ HeadBlock head_block(int p, int heads, int blocks, bool causal) {
  const int rest = heads % 8, whole = (heads - rest) * blocks;
  if (p < whole) {
    const int q = p / (8 * blocks), r = p - q * 8 * blocks;
    return {8 * q + r % 8, r / 8};
  }
  const int r = p - whole;
  if (causal) return {heads - rest + r % rest, r / rest};
  const int x = xcd_remap(r, rest * blocks);
  return {heads - rest + x / blocks, x % blocks};
}

// This lane's operand addresses in LDS, of a tile at the start of `base`; a tile
// `off` bytes further on is read with the same addresses and an offset. FEW (D = 128):
// the chunks and column tiles differ from the first by an exclusive or, made at each
// read, where registers decide how many waves a SIMD holds.
template <int D, bool FEW = false>
struct TileAddr {
  static constexpr int KC = D / 16, NT = D / 32;
  static_assert(!FEW || D == 128, "eight chunks and four column tiles within the swizzle's blocks");
  uint32_t rr[FEW ? 1 : KC];                      // row-layout chunk c: row l%32, columns (D/2)(l/32) + 8c ..
  uint32_t tr[FEW ? 1 : NT][2];                   // transposed column tile t, rows + 0 and + 8
  __device__ __forceinline__ void init(const char* base) {
    const int lane = lane_id(), h = lane >> 5, j = lane & 31, i16 = lane & 15;
#pragma unroll
    for (int c = 0; c < (FEW ? 1 : KC); ++c) rr[c] = lds_addr(base) + raw_offset<D, exact_swz<D>>(j, (D / 2) * h + 8 * c);
#pragma unroll
    for (int t = 0; t < (FEW ? 1 : NT); ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        tr[t][e] = lds_addr(base) +
                   raw_offset<D, exact_swz<D>>(4 * h + i16 / 4 + 8 * e, 32 * t + 16 * ((lane >> 4) & 1) + 4 * (i16 & 3));
    // kept as they are, not put together again at each read
#pragma unroll
    for (int c = 0; c < (FEW ? 1 : KC); ++c) asm("" : "+v"(rr[c]));
#pragma unroll
    for (int t = 0; t < (FEW ? 1 : NT); ++t) asm("" : "+v"(tr[t][0]), "+v"(tr[t][1]));
  }
  __device__ __forceinline__ u32x4 row(int off, int c) const {
    return *(const __attribute__((address_space(3))) u32x4*)(lds_ptr)((FEW ? rr[0] ^ 16u * c : rr[FEW ? 0 : c]) + off);
  }
  // transposed chunk (u, t): rows 16u + 8(s/4) + 4(l/32) + s%4 (s = 0..7) of column 32t + l%32
  __device__ __forceinline__ u32x4 trans(int off, int u, int t) const {
    u32x2 x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                           (__attribute__((address_space(3))) s16x4*)(lds_ptr)(
                                               (FEW ? tr[0][e] ^ 64u * t : tr[FEW ? 0 : t][e]) + off + 16 * u * 2 * D)));
    return u32x4{x[0][0], x[0][1], x[1][0], x[1][1]};
  }
};

__device__ __forceinline__ f32x16 mfma16(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ f32x16 splat16(float x) {
  f32x16 s;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = x;
  return s;
}

// A row of D elements as this lane's part of a B operand (row l%32's half l/32),
// in planes; `on` false: zeros.
template <int NP, int D>
__device__ __forceinline__ void load_operand(const char* row, bool on, u32x4 (&f)[NP][D / 16]) {
  constexpr int KC = D / 16;
  const char* p = row + (lane_id() >> 5) * (D / 2) * (NP == 1 ? 2 : 4);
  if constexpr (NP == 1) {
#pragma unroll
    for (int c = 0; c < KC; ++c) f[0][c] = on ? reinterpret_cast<const u32x4*>(p)[c] : u32x4{0, 0, 0, 0};
  } else {
    u32x4 raw[2 * KC];
#pragma unroll
    for (int c = 0; c < 2 * KC; ++c) raw[c] = on ? reinterpret_cast<const u32x4*>(p)[c] : u32x4{0, 0, 0, 0};
    split_chunks(raw, f);
  }
}

// c + A B^T over the column chunks K0 .. K1 - 1 (16 columns each): A the rows of the staged tile (plane 0 at `tile`,
// planes `step` bytes apart), B this lane's operand; the smallest plane products first.
template <int NP, int D, int K0, int K1, class At>
__device__ __forceinline__ f32x16 product_part(const At& a, int tile, int step,
                                               const u32x4 (&b)[NP][D / 16], f32x16 c) {
  constexpr int C = K1 - K0 < 2 ? K1 - K0 : 2;     // chunks read together, ahead of their products
#pragma unroll
  for (int p = NP - 1; p >= 0; --p)
#pragma unroll
    for (int k0 = K0; k0 < K1; k0 += C) {
      u32x4 x[C];
#pragma unroll
      for (int i = 0; i < C; ++i) x[i] = a.row(tile + p * step, k0 + i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < C; ++i)
#pragma unroll
        for (int q = NP - 1 - p; q >= 0; --q) c = mfma16(x[i], b[q][k0 + i], c);
    }
  return c;
}

template <int NP, int D, class At>
__device__ __forceinline__ f32x16 product(const At& at, int tile, int step, const u32x4 (&b)[NP][D / 16],
                                          const f32x16& c) {
  return product_part<NP, D, 0, D / 16>(at, tile, step, b, c);
}

// The 16 weights of a lane as the planes of the next product's B operand.
template <int NP>
struct Packed {
  u32x4 w[NP][2];
};

// All row-layout chunks of a one-plane tile.
template <int D, class At>
__device__ __forceinline__ void read_rows(const At& at, int tile, u32x4 (&f)[D / 16]) {
#pragma unroll
  for (int c = 0; c < D / 16; ++c) f[c] = at.row(tile, c);
}

// All transposed chunks of a one-plane tile.
template <int D, class At>
__device__ __forceinline__ void read_trans(const At& at, int tile, u32x4 (&f)[2][D / 32]) {
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int t = 0; t < D / 32; ++t) f[u][t] = at.trans(tile, u, t);
}

// o += X^T W of a one-plane tile whose transposed chunks are x.
template <int D>
__device__ __forceinline__ void accumulate_chunks(const u32x4 (&x)[2][D / 32], const Packed<1>& w, f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int t = 0; t < D / 32; ++t) o[t] = mfma16(x[u][t], w.w[0][u], o[t]);
}

// A row's number x as an operand chunk: the bfloat16 elements hi, mid, lo of x (each
// the rest rounded, so their sum is x to 2^-24), then zeros. One more step of a
// product, with a chunk of three ones on the other side, adds x to the row's results.
__device__ __forceinline__ u32x4 number_chunk(float x) {
  bf16x2 a, b;
  a[0] = (__bf16)x;
  const float r = x - (float)a[0];
  a[1] = (__bf16)r;
  b[0] = (__bf16)(r - (float)a[1]);
  b[1] = (__bf16)0.0f;
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), 0u, 0u};
}

// The planes of 16 weights.
template <int NP>
__device__ __forceinline__ Packed<NP> pack_weights(const float (&p)[16]) {
  Packed<NP> k;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if constexpr (NP == 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bf16x2 b;
        b[0] = (__bf16)p[8 * u + 2 * e];
        b[1] = (__bf16)p[8 * u + 2 * e + 1];
        k.w[0][u][e] = __builtin_bit_cast(uint32_t, b);
      }
    } else {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = p[8 * u + e];
      u32x4 pl[3];
      split8(v, pl);
#pragma unroll
      for (int q = 0; q < 3; ++q) k.w[q][u] = pl[q];
    }
  }
  return k;
}

// o (D rows x 32 columns) += X^T W: X the staged tile, W packed weights. A plane's chunks
// of all column tiles are read together, and their products are independent.
template <int NP, int D, class At>
__device__ __forceinline__ void accumulate_t(const At& at, int tile, int step, const Packed<NP>& w,
                                             f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int p = NP - 1; p >= 0; --p) {
      u32x4 x[D / 32];
#pragma unroll
      for (int t = 0; t < D / 32; ++t) x[t] = at.trans(tile + p * step, u, t);
#pragma unroll
      for (int q = NP - 1 - p; q >= 0; --q)
#pragma unroll
        for (int t = 0; t < D / 32; ++t) o[t] = mfma16(x[t], w.w[q][u], o[t]);
    }
}

// Register r of a product holds row 8(r/4) + 4(l/32) + r%4 of its 32.
__device__ __forceinline__ constexpr int reg_row(int r) { return 8 * (r >> 2) + (r & 3); }

// s where this lane's bit of the row is set, else x; `bits` by row.
__device__ __forceinline__ void select_rows(f32x16& s, uint32_t bits, float x) {
  const uint32_t m = bits >> (4 * (lane_id() >> 5));
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = (m >> reg_row(r)) & 1 ? s[r] : x;
}

// The lowest n bits (n may be negative or above 32).
__device__ __forceinline__ uint32_t low_bits(int n) {
  return n >= 32 ? ~0u : (n <= 0 ? 0u : (1u << n) - 1);
}

__device__ __forceinline__ int key_limit(const ExactArgs& a, int b) {
  return a.lengths == nullptr ? a.nk : min(max(a.lengths[b], 0), a.nk);
}

// Position of query 0 of batch b.
__device__ __forceinline__ int first_position(const ExactArgs& a, int b) {
  constexpr int kFar = 1 << 29;
  return a.q_start == nullptr ? a.nk - a.nq : min(max(a.q_start[b], -kFar), kFar);
}

// This lane's byte of the mask of the R keys from k0 on (nonzero: counts); a lane past
// the keys repeats the last.
template <int R>
struct MaskBytes {
  uint32_t b;
  __device__ __forceinline__ void load(const ExactArgs& a, int batch, int k0) {
    b = a.key_mask == nullptr ? 1 : a.key_mask[(long long)batch * a.mask_stride + min(k0 + lane_id(), a.nk - 1)];
  }
  // the keys k0 .. k0 + R - 1 that count
  __device__ __forceinline__ RowBits<R> bits(int k0, int limit) const {
    const int r = lane_id();
    return {__ballot(r < R && k0 + r < limit && b != 0)};
  }
};

// The rows row0 .. row0 + R - 1 below limit.
template <int R>
__device__ __forceinline__ RowBits<R> row_bits(int row0, int limit) {
  const int r = lane_id();
  return {__ballot(r < R && row0 + r < limit)};
}

// A bias as every kernel takes it: below -kBiasRange its distances do not count, above kBiasRange it
// is kBiasRange. A log normaliser is one float32, so a probability exp(S - L) is off by about
// |L| 2^-23: at 2^14 by 2^-9, half a bfloat16 rounding. Beyond, the sums of a query whose keys all
// carry such a bias leave 1 (0.93 to 1.07 at 1e6) and at -1e38 are NaN.
constexpr float kBiasRange = 16384.0f;
__device__ __forceinline__ float bias_value(const ExactArgs& a, int h, int entry) {
  const int e = a.map[entry];
  if ((unsigned)e >= (unsigned)a.buckets) return 0.0f;
  const long long at = (long long)e * a.H + h;
  const float x = a.bias_bf16 ? bf16_to_f32(static_cast<const uint16_t*>(a.bias)[at]) : static_cast<const float*>(a.bias)[at];
  return x < -kBiasRange ? -INFINITY : (x > kBiasRange ? kBiasRange : x);
}

// The position bias of a 32 x 32 tile depends on key - position only, 63
// distances. Where all of them are at most -far or at least far it is one
// number (one of the outer entries); the rest read it from a window in LDS: entry
// far + kWinPad + distance, which such a tile never leaves.
constexpr int kWinPad = 64;
__host__ __device__ constexpr int window_entries(int far) { return 2 * far + 2 * kWinPad; }

// Fills the window (log2 units) with T threads; the caller synchronises.
__device__ __forceinline__ void fill_window(const ExactArgs& a, int h, float* win, int tid, int threads) {
  for (int i = tid; i < window_entries(a.far); i += threads)
    win[i] = bias_value(a, h, min(max(i - kWinPad, 0), 2 * a.far)) * kLog2e;
}

enum BiasKind { kBiasNear = 0, kBiasLow = 1, kBiasHigh = 2 };

// d0: the distance of the tile's first key and first query.
__device__ __forceinline__ BiasKind bias_kind(int d0, int far) {
  if (d0 + 31 <= -far) return kBiasLow;
  if (d0 - 31 >= far) return kBiasHigh;
  return kBiasNear;
}

// bfloat16 or float32 elements of four consecutive columns
template <int NP>
__device__ __forceinline__ void store4(char* dst, const float (&z)[4]) {
  if constexpr (NP == 1) {
    bf16x2 lo, hi;
    lo[0] = (__bf16)z[0]; lo[1] = (__bf16)z[1];
    hi[0] = (__bf16)z[2]; hi[1] = (__bf16)z[3];
    *reinterpret_cast<u32x2*>(dst) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  } else {
    *reinterpret_cast<f32x4*>(dst) = f32x4{z[0], z[1], z[2], z[3]};
  }
}

// Stores the transposed accumulators o (column l%32 = a row of the result), times
// f, to the row at `row` if `on` (every lane takes part in the exchange: lanes l
// and l^32 hold four columns of two groups each and store eight of one, 16 bytes).
template <int NP, int D>
__device__ __forceinline__ void store_rows(const f32x16 (&o)[D / 32], float f, char* row, bool on) {
  const int h = lane_id() >> 5;
#pragma unroll
  for (int t = 0; t < D / 32; ++t) {
    if constexpr (NP == 1) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        u32x2 pr[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          bf16x2 lo, hi;
          lo[0] = (__bf16)(o[t][8 * g + 4 * e] * f); lo[1] = (__bf16)(o[t][8 * g + 4 * e + 1] * f);
          hi[0] = (__bf16)(o[t][8 * g + 4 * e + 2] * f); hi[1] = (__bf16)(o[t][8 * g + 4 * e + 3] * f);
          pr[e] = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
        }
        const u32x2 send = h ? pr[0] : pr[1];
        u32x2 recv;
        recv[0] = (uint32_t)__shfl_xor((int)send[0], 32);
        recv[1] = (uint32_t)__shfl_xor((int)send[1], 32);
        const u32x4 st = h ? u32x4{recv[0], recv[1], pr[1][0], pr[1][1]} : u32x4{pr[0][0], pr[0][1], recv[0], recv[1]};
        if (on) *reinterpret_cast<u32x4*>(row + 2 * (32 * t + 16 * g + 8 * h)) = st;
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float z[4] = {o[t][4 * g] * f, o[t][4 * g + 1] * f, o[t][4 * g + 2] * f, o[t][4 * g + 3] * f};
        if (on) store4<3>(row + 4 * (32 * t + 8 * g + 4 * h), z);
      }
    }
  }
}

// Whether a wave takes 64 queries: it then reads K and V from LDS half as often, but needs
// the rows to fill the larger blocks, and blocks to fill the chip more than once
// (forward of 384 heads x 512 x 64, 768 of them: 36 -> 38 us).
inline bool wide_rows(long long heads, int nq) {
  const long long wide = ((long long)nq + 255) / 256, narrow = ((long long)nq + 127) / 128;
  return heads * wide >= 4 * kCus && 20 * wide <= 11 * narrow;
}

// More than 64 KB of dynamic LDS has to be allowed for.
template <class Kernel>
inline hipError_t allow_lds(Kernel kernel, size_t smem) {
  if (smem <= 65536) return hipSuccess;
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
}

}  // namespace mra
