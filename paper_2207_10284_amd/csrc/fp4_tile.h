// Device code shared by the kernels of the 4-bit cache (mra_layer.h): where its parts lie and
// how codes become values. The conversion instructions of gfx950 take two codes (a byte) and
// a power-of-two step each way; every value is exact in bfloat16.
#pragma once

#include "common.h"
#include "fp4_layout.h"
#include "layer_kernels.h"
#include "tile_ops.h"

namespace mra {

// The page of a head that holds token t of sequence b (t below the table's end), or null.
__device__ __forceinline__ char* fp4_page(const CacheArgs& c, int b, int hk, int t) {
  const int page = c.table[(long long)b * c.max_pages + (t >> c.page_log2)];
  return (unsigned)page < (unsigned)c.pages ? c.data + ((long long)page * c.Hkv + hk) * c.head_bytes : nullptr;
}

__device__ __forceinline__ float fp4_step(uint32_t e) { return __uint_as_float(e << 23); }

// The held exponent of a block whose largest magnitude is `top`: of the smallest power of
// two with top <= 7 of it. 7 is 1.75 times a power of two: a mantissa above that takes the next.
__device__ __forceinline__ uint32_t fp4_exponent(float top) {
  const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 2;
  return (uint32_t)min(max(e, 2), 252);
}

// Eight values as codes, the first lowest.
__device__ __forceinline__ uint32_t fp4_encode(const float (&f)[8], float step) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], step, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], step, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], step, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], step, 3);
}

// Byte SEL of w as two bfloat16 values, the low code's in the low half.
template <int SEL>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float step) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, SEL));
}

// The eight values of w as bfloat16.
__device__ __forceinline__ u32x4 fp4_decode(uint32_t w, float step) {
  return u32x4{fp4_pair<0>(w, step), fp4_pair<1>(w, step), fp4_pair<2>(w, step), fp4_pair<3>(w, step)};
}

}  // namespace mra
