// Device helpers of the 8-bit paged cache: the order of codes in a page and
// the rounding of a block.
#pragma once
#include "tppsd_cache.h"
#include "tppsd_device.h"

namespace tppsd {

// ---- fragment order ---------------------------------------------------------
// A (page, layer, head) tile is the keys' 64 dh codes, then the values'. The
// attention reads both in 16-byte words, word c of lane l = 16 g + m at
// c 1024 + 16 l:
//   keys: fragment (tile t of 16 keys, k step s) holds key 16 t + m, columns
//     32 s + 8 g .. + 7 (d_head 16: columns 4 g .. + 3 of the one step)
//   values: fragment (column tile u, half w) holds column 16 u + m of the keys
//     16 (2 w + (j >> 2)) + 4 g + (j & 3), j = 0..7: the keys whose scores that
//     lane group holds after the S^T products of tiles 2 w and 2 w + 1
// byte i of word c of lane l of the keys: (key, column)
template <int DH> __device__ __forceinline__ void key_at(int c, int lane, int i, int &key, int &col) {
  const int m = lane & 15, g = lane >> 4;
  if (DH == 16) {
    key = 16 * (i >> 2) + m;
    col = 4 * g + (i & 3);
  } else {
    constexpr int NS = DH >= 32 ? DH / 32 : 1;
    const int f = 2 * c + (i >> 3), t = f / NS, s = f - t * NS;
    key = 16 * t + m;
    col = 32 * s + 8 * g + (i & 7);
  }
}
__device__ __forceinline__ void value_at(int c, int lane, int i, int &key, int &col) {
  const int m = lane & 15, g = lane >> 4, w = i >> 3, j = i & 7;
  key = 16 * (2 * w + (j >> 2)) + 4 * g + (j & 3);
  col = 16 * c + m;
}
// where element (key, column) is
template <int DH> __device__ __forceinline__ int key_byte(int key, int col) {
  const int t = key >> 4, m = key & 15;
  if (DH == 16) return (16 * (col >> 2) + m) * 16 + t * 4 + (col & 3);
  constexpr int NS = DH >= 32 ? DH / 32 : 1;
  const int f = t * NS + (col >> 5), g = (col >> 3) & 3;
  return (f >> 1) * 1024 + (16 * g + m) * 16 + (f & 1) * 8 + (col & 7);
}
__device__ __forceinline__ int value_byte(int key, int col) {
  const int t = key >> 4, g = (key >> 2) & 3;
  return (col >> 4) * 1024 + (16 * g + (col & 15)) * 16 + (t >> 1) * 8 + (t & 1) * 4 + (key & 3);
}

// exponent of the scale for block maximum m (>= 0, finite): the least e with m <= 448 2^e
__device__ __forceinline__ int scale_exp(float m) {
  const uint32_t u = __float_as_uint(m);
  if (m == 0.f) return 0;
  // 448 = 1.75 2^8 (subnormal maxima fall under the least exponent anyway)
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, CACHE_E_MIN);
}

// x 2^-e as an e4m3 code; infinities and NaN become NaN
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}

}  // namespace tppsd
