// Writing the 4-bit cache and reading it back (mra_layer.h).
//
// Bound by memory: a value comes in as 2 or 4 bytes and leaves as 17/32 of one. A workgroup
// takes 32 neighbouring tokens (aligned, so of one page) of one head, keys and values. A lane
// has eight channels of a token, four lanes a block and its step. Keys leave from there; values,
// which the cache holds eight tokens of a channel pair together (as the products of attention take them),
// are put in order in LDS first.
#include "fp4_tile.h"

namespace mra {

namespace {

constexpr int kThreads = 256;

// Which tokens of a workgroup's tile a call writes or reads.
struct Span {
  int b, hk, t0;                          // sequence, head, first token of the tile
  int start, lo, hi;                      // the call's first token; the tile's live ones are lo to hi - 1
  char* page;                             // null: none
};

__device__ __forceinline__ Span span_of(const CacheRowsArgs& a, int tiles) {
  Span s;
  const int g = blockIdx.x, bh = g / tiles;
  s.b = bh / a.c.Hkv;
  s.hk = bh - s.b * a.c.Hkv;
  s.start = a.starts == nullptr ? 0 : min(max(a.starts[s.b], 0), a.c.cap);
  const int count = min(a.counts == nullptr ? a.n : min(max(a.counts[s.b], 0), a.n), a.c.cap - s.start);
  s.t0 = (s.start / 32 + g - bh * tiles) * 32;
  s.lo = max(s.t0, s.start);
  s.hi = min(s.t0 + 32, s.start + count);
  s.page = s.lo < s.hi ? fp4_page(a.c, s.b, s.hk, s.t0) : nullptr;
  return s;
}

template <int DT>
__device__ __forceinline__ void load8(const char* p, float (&f)[8]) {
  if constexpr (DT == BF16) {
    const u32x4 r = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(r[e] << 16);
      f[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4 r = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * i + e] = r[e];
    }
  }
}

template <int DT>
__device__ __forceinline__ void store8(char* p, uint32_t w, float step) {
  const u32x4 v = fp4_decode(w, step);
  if constexpr (DT == BF16) {
    *reinterpret_cast<u32x4*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      reinterpret_cast<f32x4*>(p)[i] =
          f32x4{__uint_as_float(v[2 * i] << 16), __uint_as_float(v[2 * i] & 0xffff0000u),
                __uint_as_float(v[2 * i + 1] << 16), __uint_as_float(v[2 * i + 1] & 0xffff0000u)};
  }
}

}  // namespace

template <int DT, int D>
__global__ __launch_bounds__(kThreads) void fp4_write_kernel(CacheRowsArgs a, int tiles) {
  using Pg = Fp4Page<D>;
  constexpr int CPR = D / 8, E = DT == BF16 ? 2 : 4;
  constexpr int N = 2 * 32 * CPR / kThreads;       // units of eight channels per lane
  constexpr int COPY = 16 * D / kThreads;          // bytes of values per lane
  __shared__ __attribute__((aligned(16))) uint8_t vt[16 * D];
  const Span s = span_of(a, tiles);
  if (s.page == nullptr) return;
  const int tid = threadIdx.x, size = 1 << a.c.page_log2, slot = s.t0 & (size - 1);
  float f[N][8];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int unit = u * kThreads + tid, value = unit / (32 * CPR), r = unit / CPR % 32, c = unit % CPR;
    const Rows& x = value ? a.v : a.k;
    const int t = s.t0 + r;
    if (t >= s.lo && t < s.hi) {
      load8<DT>(x.p + s.b * x.sb + s.hk * x.sh + (t - s.start) * x.sn + c * 8 * E, f[u]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[u][e] = 0.0f;
    }
  }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int unit = u * kThreads + tid, value = unit / (32 * CPR), r = unit / CPR % 32, c = unit % CPR;
    const bool on = s.t0 + r >= s.lo && s.t0 + r < s.hi;
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[u][e]));
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    const uint32_t ex = fp4_exponent(top);
    const uint32_t w = fp4_encode(f[u], fp4_step(ex));
    const uint32_t other = (uint32_t)__shfl_xor((int)w, 2);        // the channels 16 further on, or back
    if (c % 4 == 0 && on)
      s.page[(value ? Pg::value_steps(size) : Pg::key_steps(size)) + (slot + r) * Pg::NB + c / 4] = (char)ex;
    if (value == 0) {
      if (on) *reinterpret_cast<uint32_t*>(s.page + (slot + r) * (D / 2) + c * 4) = w;
    } else {
      // entries i = 8 (c % 2) + 0 .. 7: the lane of the lower channels does the even ones, its partner the odd
      const int q = c % 4;
      const uint32_t bytes = q < 2 ? (w & 0x0f0f0f0fu) | (other & 0x0f0f0f0fu) << 4
                                   : (other >> 4 & 0x0f0f0f0fu) | (w & 0xf0f0f0f0u);
      uint8_t* to = vt + r / 8 * Pg::kTile;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        to[Pg::entry(r % 8, c / 4, 8 * (q & 1) + 2 * j + (q >> 1))] = (uint8_t)(bytes >> 8 * j);
    }
  }
  __syncthreads();
  char* to = s.page + Pg::values(size) + slot * (D / 2) + tid * COPY;
  const uint8_t* from = vt + tid * COPY;
  if (s.hi - s.lo == 32) {
    if constexpr (COPY == 8) *reinterpret_cast<u32x2*>(to) = *reinterpret_cast<const u32x2*>(from);
    if constexpr (COPY == 4) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
    if constexpr (COPY == 2) *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(from);
    return;
  }
#pragma unroll
  for (int i = 0; i < COPY; ++i) {
    const int at = tid * COPY + i, t = s.t0 + at / Pg::kTile * 8 + at / Pg::P % 8;
    if (t >= s.lo && t < s.hi) to[i] = (char)from[i];
  }
}

template <int DT, int D>
__global__ __launch_bounds__(kThreads) void fp4_read_kernel(CacheRowsArgs a, int tiles) {
  using Pg = Fp4Page<D>;
  constexpr int CPR = D / 8, E = DT == BF16 ? 2 : 4;
  constexpr int N = 2 * 32 * CPR / kThreads;
  constexpr int COPY = 16 * D / kThreads;
  __shared__ __attribute__((aligned(16))) uint8_t vt[16 * D];
  const Span s = span_of(a, tiles);
  const int tid = threadIdx.x, size = 1 << a.c.page_log2, slot = s.t0 & (size - 1);
  const bool some = s.page != nullptr;             // the same for the whole workgroup
  uint32_t w[N], ex[N];
  if (some) {
    const char* from = s.page + Pg::values(size) + slot * (D / 2) + tid * COPY;
    uint8_t* to = vt + tid * COPY;
    if constexpr (COPY == 8) *reinterpret_cast<u32x2*>(to) = *reinterpret_cast<const u32x2*>(from);
    if constexpr (COPY == 4) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
    if constexpr (COPY == 2) *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(from);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int unit = u * kThreads + tid, value = unit / (32 * CPR), r = unit / CPR % 32, c = unit % CPR;
      ex[u] = (uint8_t)s.page[(value ? Pg::value_steps(size) : Pg::key_steps(size)) + (slot + r) * Pg::NB + c / 4];
      w[u] = value ? 0 : *reinterpret_cast<const uint32_t*>(s.page + (slot + r) * (D / 2) + c * 4);
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int unit = u * kThreads + tid, value = unit / (32 * CPR), r = unit / CPR % 32, c = unit % CPR;
    const int t = s.t0 + r;
    if (t < s.start || t - s.start >= a.n) continue;
    const bool on = some && t < s.hi;
    if (value && on) {
      const uint8_t* from = vt + r / 8 * Pg::kTile;
      const int q = c % 4;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        w[u] |= (uint32_t)(from[Pg::entry(r % 8, c / 4, 8 * (q & 1) + j)] >> 4 * (q >> 1) & 15) << 4 * j;
    }
    const Rows& x = value ? a.v : a.k;
    store8<DT>(x.p + s.b * x.sb + s.hk * x.sh + (long long)(t - s.start) * x.sn + c * 8 * E, on ? w[u] : 0,
               fp4_step(on ? ex[u] : 127));
  }
}

// Tiles of 32 that n tokens can touch.
static unsigned row_groups(const CacheRowsArgs& a, int* tiles) {
  *tiles = (a.n + 30) / 32 + 1;
  return (unsigned)((long long)a.B * a.c.Hkv * *tiles);
}

template <class F>
static hipError_t cache_variant(int d, int dtype, F run) {
  auto width = [&](auto dt) {
    if (d == 32) return run(dt, std::integral_constant<int, 32>{});
    if (d == 64) return run(dt, std::integral_constant<int, 64>{});
    return run(dt, std::integral_constant<int, 128>{});
  };
  return dtype == BF16 ? width(std::integral_constant<int, BF16>{}) : width(std::integral_constant<int, F32>{});
}

hipError_t launch_cache_write(const CacheRowsArgs& a, int d, int dtype, hipStream_t stream) {
  return cache_variant(d, dtype, [&](auto dt, auto dd) {
    int tiles;
    const unsigned groups = row_groups(a, &tiles);
    fp4_write_kernel<dt.value, dd.value><<<groups, kThreads, 0, stream>>>(a, tiles);
    return hipGetLastError();
  });
}

hipError_t launch_cache_read(const CacheRowsArgs& a, int d, int dtype, hipStream_t stream) {
  return cache_variant(d, dtype, [&](auto dt, auto dd) {
    int tiles;
    const unsigned groups = row_groups(a, &tiles);
    fp4_read_kernel<dt.value, dd.value><<<groups, kThreads, 0, stream>>>(a, tiles);
    return hipGetLastError();
  });
}

}  // namespace mra
