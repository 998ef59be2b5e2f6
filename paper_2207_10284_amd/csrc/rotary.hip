// Rotary positions and head norms, forward and gradients (mra_layer.h).
//
// Bound by memory: an element is read and written once (backward with a norm: two read, one
// written) for some ten operations. What is left to do is to keep the angles
// cheap, some float64 products and a sine and cosine each: a workgroup takes a tile of
// tokens with all their heads, makes the tile's sines and cosines once in LDS, and
// its rows read them there. Measured on data that no cache holds: 8 x 24 heads x 4096 x 64 bfloat16, forward or backward
// 41 us (201 MB, 4.9 TB/s, 97% of a large copy's rate); 20 heads x 32768 x 128 bfloat16 with norms, forward 62 us (336 MB,
// 5.4 TB/s), backward 109 us (503 MB, 4.6 TB/s: three rows in flight take 190 registers, two waves a SIMD) and
// 6 us for the weights' sums; 10 heads x 4 x 2999 x 128 float32, forward 28 us (123 MB, 4.4 TB/s).
//
// A row is shared by D / 16 lanes. A lane holds two chunks of eight elements such that
// the eight pairs within them are its own: chunks i and rot/2 + i (half), or
// two neighbours (interleaved); norms are sums over the row's lanes, and nothing else moves between
// lanes. Where a row's lanes are fewer than a cache line's, rows that lie next to each other
// are taken next to each other (head_fast).
#include "common.h"
#include "layer_kernels.h"
#include "tile_ops.h"

namespace mra {

namespace {

constexpr int kThreads = 256;
// Tokens of a tile (24 heads x 8 x 4096 x 64 bfloat16, training: four 84.5, eight 81.7, sixteen 84.8 us)
constexpr int kMaxTile = 8;

// Eight consecutive elements.
template <int DT>
struct Chunk {
  static constexpr int kBytes = DT == BF16 ? 16 : 32;
  u32x4 raw[DT == BF16 ? 1 : 2];

  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < (DT == BF16 ? 1 : 2); ++i) raw[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (DT == BF16)
        f[e] = e % 2 ? __uint_as_float(raw[0][e / 2] & 0xffff0000u) : __uint_as_float(raw[0][e / 2] << 16);
      else
        f[e] = __uint_as_float(raw[e / 4][e % 4]);
    }
  }
};

template <int DT>
__device__ __forceinline__ void store_chunk(char* p, const float* f) {
  if constexpr (DT == BF16) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bf16x2 b;
      b[0] = (__bf16)f[2 * e];
      b[1] = (__bf16)f[2 * e + 1];
      r[e] = __builtin_bit_cast(uint32_t, b);
    }
    *reinterpret_cast<u32x4*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      reinterpret_cast<f32x4*>(p)[i] = f32x4{f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]};
  }
}

// Sum over the L lanes of a row.
template <int L>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int s = 1; s < L; s *= 2) v += __shfl_xor(v, s);
  return v;
}

// The pair elements of v (16 elements of a lane) turned by (cos, sin), sin's sign times `sign`.
template <bool INTER>
__device__ __forceinline__ void turn(float (&v)[16], const float2 (&cs)[8], float sign) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float &a = INTER ? v[2 * j] : v[j], &b = INTER ? v[2 * j + 1] : v[8 + j];
    const float c = cs[j].x, s = sign * cs[j].y, x = a, y = b;
    a = x * c - y * s;
    b = y * c + x * s;
  }
}

// What the rows of a workgroup's tile share.
template <int D>
struct Tile {
  static constexpr int L = D / 16, ROWS = kThreads / L;
  int c, row;                             // this lane's part of a row, and its row among ROWS
  int pairs;                              // lanes of a row that hold pairs
  int e0, e1;                             // the elements of the lane's two chunks

  __device__ __forceinline__ void init(int rot, bool inter) {
    c = threadIdx.x % L;
    row = threadIdx.x / L;
    pairs = rot / 16;
    e0 = inter || c >= pairs ? 16 * c : 8 * c;
    e1 = inter || c >= pairs ? 16 * c + 8 : rot / 2 + 8 * c;
  }
};

// cos and sin (times the magnitude) of the tile's tokens and frequencies. Tokens are below 2^27. What is
// left of pos freq / (2 pi) without its whole turns is off by some 2^-53 of a turn, not of all turns: the
// frequency in turns is the sum of two float64 values, and whole turns leave the product before it is rounded.
__device__ __forceinline__ void fill_angles(const RotaryArgs& a, int first, int tokens, float2* cs) {
  const int half = a.rot / 2;                      // a multiple of eight, at most 64, not always a power of two
  for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
    const int t = i / half, f = i - t * half;
    const int b = (first + t) / a.n, n = first + t - b * a.n;
    const double pos = a.positions == nullptr ? n : a.positions[b * a.positions_stride + n];
    constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;   // 1 / (2 pi)
    const double freq = a.freqs[f], high = freq * kHigh, low = fma(freq, kHigh, -high) + freq * kLow;
    double turns = fma(pos, low, fma(pos, high, -rint(pos * high)));
    turns -= rint(turns);                          // one more, or those of products past 2^53
    // sine and cosine of the float32 part, turned by the rest of at most 2^-26 turns (without it they are off by up to
    // 1.1e-7, with it 7.8e-8; both make the same time)
    const float near = (float)turns, rest = (float)((turns - near) * 6.283185307179586);
    float s, c;
    sincospif(2.0f * near, &s, &c);
    cs[i] = float2{fmaf(-s, rest, c) * a.magnitude, fmaf(c, rest, s) * a.magnitude};
  }
}

template <int D>
__device__ __forceinline__ void read_angles(const float2* cs, int token, int half, int c, float2 (&out)[8]) {
  const f32x4* p = reinterpret_cast<const f32x4*>(cs + token * half + 8 * c);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x4 v = p[j];
    out[2 * j] = float2{v[0], v[1]};
    out[2 * j + 1] = float2{v[2], v[3]};
  }
}

// Where row r of a side's tile lies: its token in the tile, batch, place in the batch, head.
struct RowAt {
  int token, b, i, h;
  __device__ __forceinline__ RowAt(const RotaryArgs& a, const RotarySide& s, int first, int tokens, int r) {
    if (s.head_fast) {
      token = r / s.heads;
      h = r - token * s.heads;
    } else {
      h = r / tokens;
      token = r - h * tokens;
    }
    b = (first + token) / a.n;
    i = first + token - b * a.n;
  }
  __device__ __forceinline__ long long in(const Rows& x) const { return b * x.sb + h * x.sh + i * x.sn; }
};

// Both sides' weights as float32 in LDS, and a lane's sixteen of one.
template <size_t D>
__device__ __forceinline__ void fill_weights(const RotaryArgs& a, float (&ws)[2][D]) {
  const int x = threadIdx.x / (int)D, e = threadIdx.x % (int)D;
  if (x > 1 || a.side[x].w == nullptr) return;
  ws[x][e] = a.weight_bf16 ? bf16_to_f32(static_cast<const uint16_t*>(a.side[x].w)[e])
                           : static_cast<const float*>(a.side[x].w)[e];
}
template <size_t D>
__device__ __forceinline__ void read_weights(const float (&ws)[D], int e0, int e1, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(&ws[(i < 2 ? e0 : e1) + 4 * (i % 2)]);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[4 * i + j] = v[j];
  }
}

}  // namespace

// U rows of a lane, on their way from memory.
template <int DT, int U>
struct Batch {
  static constexpr int E = DT == BF16 ? 2 : 4;
  Chunk<DT> c[U][2];
  int token[U];
  long long to[U];

  template <int D>
  __device__ __forceinline__ void load(const RotaryArgs& a, const RotarySide& s, const Rows& from, const Tile<D>& t,
                                       int first, int tokens, int r0, int rows) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * Tile<D>::ROWS;
      if (r >= rows) break;                        // the same for all lanes of a row
      const RowAt at(a, s, first, tokens, r);
      const char* p = from.p + at.in(from);
      c[u][0].load(p + t.e0 * E);
      c[u][1].load(p + t.e1 * E);
      token[u] = at.token;
      to[u] = at.in(s.y);
    }
  }
};

template <int DT, int D, bool INTER, bool NORM>
__global__ __launch_bounds__(kThreads) void rotary_forward_kernel(RotaryArgs a, int tile) {
  using T = Tile<D>;
  constexpr int E = DT == BF16 ? 2 : 4;
  // Rows of a lane in flight (8 x 24 heads x 4096 x 64 bfloat16: one 46, four 42 us; float32 4 x 10 x 2999 x 128: 25, 29;
  // with a norm 20 x 32768 x 128 bfloat16: no difference)
  constexpr int U = NORM || DT == F32 ? 1 : 4;
  __shared__ __attribute__((aligned(16))) float2 cs[kMaxTile * (D / 2)];
  __shared__ __attribute__((aligned(16))) float ws[2][NORM ? D : 4];
  T t;
  t.init(a.rot, INTER);
  const int first = blockIdx.x * tile, tokens = min(tile, (int)a.tokens - first), half = a.rot / 2;
  bool filled = false;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const RotarySide& s = a.side[x];
    const int rows = tokens * s.heads;
    if (rows == 0) continue;
    int r0 = t.row;
    Batch<DT, U> in;
    in.load(a, s, s.x, t, first, tokens, r0, rows);
    if (!filled) {                                 // beside the first rows' loads
      fill_angles(a, first, tokens, cs);
      if constexpr (NORM) fill_weights(a, ws);
      __syncthreads();
      filled = true;
    }
    float w[16];
    const bool norm = NORM && s.w != nullptr;
    if (norm) read_weights(ws[x], t.e0, t.e1, w);
    for (; r0 < rows; r0 += U * T::ROWS) {
      if (r0 != t.row) in.load(a, s, s.x, t, first, tokens, r0, rows);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r0 + u * T::ROWS >= rows) break;
        float v[16];
        in.c[u][0].get(v);
        in.c[u][1].get(v + 8);
        if (norm) {
          float sum = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) sum = fmaf(v[i], v[i], sum);
          const float inv = 1.0f / sqrtf(row_sum<T::L>(sum) * (1.0f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = v[i] * inv * w[i];
        }
        if (t.c < t.pairs) {
          float2 c[8];
          read_angles<D>(cs, in.token[u], half, t.c, c);
          turn<INTER>(v, c, 1.0f);
        }
        char* p = s.y.p + in.to[u];
        store_chunk<DT>(p + t.e0 * E, v);
        store_chunk<DT>(p + t.e1 * E, v + 8);
      }
    }
  }
}

// Each workgroup takes every gridDim.x-th tile and leaves one row of sums of g y per side.
template <int DT, int D, bool INTER, bool NORM>
__global__ __launch_bounds__(kThreads) void rotary_backward_kernel(RotaryArgs a, int tile) {
  using T = Tile<D>;
  constexpr int E = DT == BF16 ? 2 : 4;
  // with a norm, 20 heads x 32768 x 128 bfloat16: one row in flight 118, two 112, three 108 us
  constexpr int U = DT == BF16 ? 3 : 2;
  __shared__ __attribute__((aligned(16))) float2 cs[kMaxTile * (D / 2)];
  __shared__ __attribute__((aligned(16))) float ws[2][NORM ? D : 4];
  __shared__ __attribute__((aligned(16))) float sums[NORM ? kThreads * 16 : 4];
  T t;
  t.init(a.rot, INTER);
  const int half = a.rot / 2;
  float dw[2][16];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) dw[x][i] = 0.0f;
  for (int first = blockIdx.x * tile; first < a.tokens; first += gridDim.x * tile) {
    const int tokens = min(tile, (int)a.tokens - first);
    bool filled = false;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const RotarySide& s = a.side[x];
      const int rows = tokens * s.heads;
      if (rows == 0) continue;
      const bool norm = NORM && s.w != nullptr;
      int r0 = t.row;
      Batch<DT, U> gr, in;
      auto load = [&] {
        gr.load(a, s, s.g, t, first, tokens, r0, rows);
        if (norm) in.load(a, s, s.x, t, first, tokens, r0, rows);
      };
      load();
      if (!filled) {                               // beside the first rows' loads
        __syncthreads();                           // the last tile's angles have been read
        fill_angles(a, first, tokens, cs);
        if (NORM && first == (int)blockIdx.x * tile) fill_weights(a, ws);
        __syncthreads();
        filled = true;
      }
      float w[16];
      if (norm) read_weights(ws[x], t.e0, t.e1, w);
      for (; r0 < rows; r0 += U * T::ROWS) {
        if (r0 != t.row) load();
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (r0 + u * T::ROWS >= rows) break;
          float g[16];
          gr.c[u][0].get(g);
          gr.c[u][1].get(g + 8);
          if (t.c < t.pairs) {
            float2 c[8];
            read_angles<D>(cs, gr.token[u], half, t.c, c);
            turn<INTER>(g, c, -1.0f);
          }
          if (norm) {
            float v[16], sum = 0.0f, dot = 0.0f;
            in.c[u][0].get(v);
            in.c[u][1].get(v + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(v[i], v[i], sum);
            const float inv = 1.0f / sqrtf(row_sum<T::L>(sum) * (1.0f / D) + a.eps);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              v[i] *= inv;
              const float gy = g[i] * v[i];
              dw[x][i] += gy;
              dot = fmaf(gy, w[i], dot);
            }
            dot = row_sum<T::L>(dot) * (1.0f / D);
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] = inv * (g[i] * w[i] - v[i] * dot);
          }
          char* p = s.y.p + gr.to[u];
          store_chunk<DT>(p + t.e0 * E, g);
          store_chunk<DT>(p + t.e1 * E, g + 8);
        }
      }
    }
  }
  if (!NORM || a.part == nullptr) return;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (a.side[x].w == nullptr) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[t.row * D + (i < 8 ? t.e0 + i : t.e1 + i - 8)] = dw[x][i];
    __syncthreads();
    if ((int)threadIdx.x < D) {
      float v = 0.0f;
      for (int r = 0; r < T::ROWS; ++r) v += sums[r * D + threadIdx.x];
      a.part[((long long)blockIdx.x * 2 + x) * D + threadIdx.x] = v;
    }
  }
}

// The workgroups' sums in double, 32 threads across columns and 32 across the sums.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void rotary_weight_kernel(const float* __restrict__ part, int groups, int D,
                                                                    void* dq_weight, void* dk_weight, int bf16) {
  __shared__ double sums[32][33];
  const int x = blockIdx.y, i = threadIdx.x % 32, g = threadIdx.x / 32, e = blockIdx.x * 32 + i;
  void* to = x == 0 ? dq_weight : dk_weight;
  if (to == nullptr) return;
  double v = 0.0;
  for (int r0 = g; r0 < groups; r0 += 8 * 32) {    // eight loads under way
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = part[((long long)min(r0 + 32 * i, groups - 1) * 2 + x) * D + e];
#pragma unroll
    for (int i = 0; i < 8; ++i) v += r0 + 32 * i < groups ? f[i] : 0.0f;
  }
  sums[g][i] = v;
  __syncthreads();
  if (g != 0) return;
  for (int r = 1; r < 32; ++r) v += sums[r][i];
  if (bf16) {
    const float f = (float)v;
    // a float32 on the way is at most 2^-24 of the value off, which moves only values that near a tie
    static_cast<__bf16*>(to)[e] = (__bf16)f;
  } else {
    static_cast<float*>(to)[e] = (float)v;
  }
}

// Tokens of a tile: kMaxTile, fewer while that leaves CUs without a workgroup.
static int rotary_tile(long long tokens) {
  int tile = kMaxTile;
  while (tile > 1 && tokens < (long long)tile * 2 * kCus) tile /= 2;
  return tile;
}

int rotary_backward_groups(long long tokens) {
  const long long tiles = (tokens + rotary_tile(tokens) - 1) / rotary_tile(tokens);
  return (int)(tiles < 4 * kCus ? tiles : 4 * kCus);
}

template <class F>
static hipError_t rotary_variant(const RotaryArgs& a, int d, int dtype, int interleaved, F run) {
  auto norm = [&](auto dt, auto dd, auto inter) {
    return a.side[0].w != nullptr || a.side[1].w != nullptr ? run(dt, dd, inter, std::true_type{})
                                                            : run(dt, dd, inter, std::false_type{});
  };
  auto inter = [&](auto dt, auto dd) {
    return interleaved ? norm(dt, dd, std::true_type{}) : norm(dt, dd, std::false_type{});
  };
  auto width = [&](auto dt) {
    if (d == 32) return inter(dt, std::integral_constant<int, 32>{});
    if (d == 64) return inter(dt, std::integral_constant<int, 64>{});
    return inter(dt, std::integral_constant<int, 128>{});
  };
  return dtype == BF16 ? width(std::integral_constant<int, BF16>{}) : width(std::integral_constant<int, F32>{});
}

hipError_t launch_rotary_forward(const RotaryArgs& a, int d, int dtype, int interleaved, hipStream_t stream) {
  const int tile = rotary_tile(a.tokens);
  return rotary_variant(a, d, dtype, interleaved, [&](auto dt, auto dd, auto inter, auto norm) {
    rotary_forward_kernel<dt.value, dd.value, inter.value, norm.value>
        <<<(unsigned)((a.tokens + tile - 1) / tile), kThreads, 0, stream>>>(a, tile);
    return hipGetLastError();
  });
}

hipError_t launch_rotary_backward(const RotaryArgs& a, int d, int dtype, int interleaved, void* dq_weight,
                                  void* dk_weight, hipStream_t stream) {
  const int tile = rotary_tile(a.tokens);
  const bool weights = dq_weight != nullptr || dk_weight != nullptr;
  // without sums to leave, a workgroup per tile
  const unsigned groups = weights ? (unsigned)rotary_backward_groups(a.tokens) : (unsigned)((a.tokens + tile - 1) / tile);
  if (a.tokens > 0) {
    const hipError_t e = rotary_variant(a, d, dtype, interleaved, [&](auto dt, auto dd, auto inter, auto norm) {
      rotary_backward_kernel<dt.value, dd.value, inter.value, norm.value><<<groups, kThreads, 0, stream>>>(a, tile);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (weights) {
    rotary_weight_kernel<<<dim3(d / 32, 2), kSumThreads, 0, stream>>>(a.part, a.tokens > 0 ? (int)groups : 0, d, dq_weight,
                                                                   dk_weight, a.weight_bf16);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace mra
