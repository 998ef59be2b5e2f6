// Writing the 4-bit cache and reading it back (mra_layer.h).
//
// Bound by memory: a value comes in as 2 or 4 bytes and leaves as 17/32 of one. A workgroup takes 64
// neighbouring tokens (aligned, so of one or two pages) of one head, keys and values. Writing, a lane has sixteen channels of a
// token and two lanes a block and its step; reading back, a lane has eight, so that it stores 16 bytes. Sixteen
// and 64 tokens against eight and 32: 48.7 -> 47.6 us for the first two figures below together.
// Measured (bfloat16): 8 x 12 heads x 4096 x 64 written in 24.5 us (127 MB, 5.2 TB/s), read back in 20.8 (127 MB,
// 6.1 TB/s, from cache in part); 4 x 4 heads x up to 32768 x 128 read back in 62 us (322 MB, 5.2 TB/s, a large copy's rate).
#include "fp4_tile.h"

namespace mra {

namespace {

constexpr int kThreads = 256;

constexpr int kTokens = kFp4RowTokens;

// Which tokens of a workgroup's tile a call writes or reads.
struct Span {
  int b, hk, t0;                          // sequence, head, first token of the tile
  int start, lo, hi;                      // the call's first token; the tile's live ones are lo to hi - 1
  char* page[2];                          // of the tile's halves; null: none

  __device__ __forceinline__ void pages(const CacheRowsArgs& a) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
      page[x] = max(lo, t0 + 32 * x) < min(hi, t0 + 32 * x + 32) ? fp4_page(a.c, b, hk, t0 + 32 * x) : nullptr;
  }
};

__device__ __forceinline__ Span span_of(const CacheRowsArgs& a, int tiles) {
  Span s;
  const int g = blockIdx.x, bh = g / tiles;
  s.b = bh / a.c.Hkv;
  s.hk = bh - s.b * a.c.Hkv;
  s.start = a.starts == nullptr ? 0 : min(max(a.starts[s.b], 0), a.c.cap);
  const int count = min(a.counts == nullptr ? a.n : min(max(a.counts[s.b], 0), a.n), a.c.cap - s.start);
  s.t0 = (s.start / kTokens + g - bh * tiles) * kTokens;
  s.lo = max(s.t0, s.start);
  s.hi = min(s.t0 + kTokens, s.start + count);
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
  using Unit = Fp4RowUnit<D, 16>;
  constexpr int E = DT == BF16 ? 2 : 4, N = Unit::kUnits / kThreads;
  Span s = span_of(a, tiles);
  if (s.lo >= s.hi) return;
  const int tid = threadIdx.x, size = 1 << a.c.page_log2;
  float f[N][2][8];                                // on their way while the table is looked up
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const Unit at(u * kThreads + tid);
    const Rows& x = at.value ? a.v : a.k;
    const int t = min(max(s.t0 + at.r, s.lo), s.hi - 1);
    const char* p = x.p + s.b * x.sb + s.hk * x.sh + (t - s.start) * x.sn + at.c * 16 * E;
    load8<DT>(p, f[u][0]);
    load8<DT>(p + 8 * E, f[u][1]);
  }
  s.pages(a);
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const Unit at(u * kThreads + tid);
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(fabsf(f[u][0][e]), fabsf(f[u][1][e])));
    top = fmaxf(top, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(top), 0xB1, 0xF, 0xF, true)));   // lane ^ 1
    const uint32_t ex = fp4_exponent(top);
    char* page = at.r < 32 ? s.page[0] : s.page[1];
    const int t = s.t0 + at.r, slot = t & (size - 1);
    if (page == nullptr || t < s.lo || t >= s.hi) continue;
    *reinterpret_cast<u32x2*>(page + at.codes_at(slot, size)) =
        u32x2{fp4_encode(f[u][0], fp4_step(ex)), fp4_encode(f[u][1], fp4_step(ex))};
    if (at.c % 2 == 0) page[at.step_at(slot, size)] = (char)ex;
  }
}

template <int DT, int D>
__global__ __launch_bounds__(kThreads) void fp4_read_kernel(CacheRowsArgs a, int tiles) {
  using Unit = Fp4RowUnit<D, 8>;
  constexpr int E = DT == BF16 ? 2 : 4, N = Unit::kUnits / kThreads;
  Span s = span_of(a, tiles);
  s.pages(a);
  const int tid = threadIdx.x, size = 1 << a.c.page_log2;
  uint32_t w[N], ex[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const Unit at(u * kThreads + tid);
    const char* page = at.r < 32 ? s.page[0] : s.page[1];
    const int t = s.t0 + at.r, slot = t & (size - 1);
    w[u] = 0;
    ex[u] = 127;
    if (page != nullptr && t < s.hi) {
      w[u] = *reinterpret_cast<const uint32_t*>(page + at.codes_at(slot, size));
      ex[u] = (uint8_t)page[at.step_at(slot, size)];
    }
  }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const Unit at(u * kThreads + tid);
    const int i = s.t0 + at.r - s.start;
    if (i < 0 || i >= a.n) continue;
    const Rows& x = at.value ? a.v : a.k;
    store8<DT>(x.p + s.b * x.sb + s.hk * x.sh + i * x.sn + at.c * 8 * E, w[u], fp4_step(ex[u]));
  }
}

int cache_row_tiles(int n) { return fp4_row_tiles(n); }

static unsigned row_groups(const CacheRowsArgs& a, int* tiles) {
  *tiles = cache_row_tiles(a.n);
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
