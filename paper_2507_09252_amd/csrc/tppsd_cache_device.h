// Device helpers of the 8-bit paged cache: the order of codes in a page and
// the rounding of a block.
#pragma once
#include "tppsd_cache.h"
#include "tppsd_device.h"

namespace tppsd {

constexpr int PLAN_ID = 3;   // counts: number of the plan

// ---- fragment order ---------------------------------------------------------
// A (page, layer, head) tile is the keys' 64 dh codes, then the values'. The
// attention reads both in 16-byte words, word c of lane l = 16 g + m at
// c 1024 + 16 l:
//   keys: fragment (tile t of 16 keys, k step s) holds key 16 t + m, columns
//     32 s + 8 g .. + 7 (d_head 16: columns 4 g .. + 3 of the one step)
//   values: fragment (column tile u, half w) holds column 16 u + m of the keys
//     16 (2 w + (j >> 2)) + 4 g + (j & 3), j = 0..7: the keys whose scores that
//     lane group holds after the S^T products of tiles 2 w and 2 w + 1
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

__device__ __forceinline__ bool not_finite(float x) { return !(fabsf(x) < INFINITY); }
// running maximum of finite magnitudes
__device__ __forceinline__ void top_up(float &top, float x) {
  const float a = fabsf(x);
  top = a < INFINITY ? fmaxf(top, a) : top;
}

// 8 elements in registers as 16-byte words (two for fp32), and element e of them
template <typename ACT> struct Eight {
  static constexpr int W = sizeof(ACT) * 8 / 16;
  u32x4_t w[W];
  __device__ __forceinline__ void load(const ACT *p) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = ((const u32x4_t *)p)[i];
  }
  __device__ __forceinline__ void store(ACT *p) const {
#pragma unroll
    for (int i = 0; i < W; ++i) ((u32x4_t *)p)[i] = w[i];
  }
  __device__ __forceinline__ ACT at(int e) const {
    if constexpr (W == 1) return (ACT)(w[0][e >> 1] >> (16 * (e & 1)));
    else return __uint_as_float(w[e >> 2][e & 3]);
  }
  // (e even first: a bf16 word is put together from its two elements)
  __device__ __forceinline__ void put(int e, ACT v) {
    if constexpr (W == 1) w[0][e >> 1] = e & 1 ? w[0][e >> 1] | (uint32_t)v << 16 : (uint32_t)v;
    else w[e >> 2][e & 3] = __float_as_uint(v);
  }
};

// A whole block's page tile from its rows in LDS (keys row per position, values
// row per column), under the maxima that the NW waves found (top[side][wave]):
// each thread rounds 16-byte words of codes, whose elements are runs of 8 (4 for
// d_head 16) columns of a key or 4 keys of a column. LDK and LDV: row strides.
template <typename ACT, int DH, int NW, int LDK, int LDV>
__device__ __forceinline__ void seal_page(const ACT (*k)[LDK], const ACT (*v)[LDV], const float (*top)[NW], uint8_t *page,
                                          float *scales) {
  constexpr int NS = DH >= 32 ? DH / 32 : 1;
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  float inv[2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    float mx = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) mx = fmaxf(mx, top[side][w]);
    const int e = scale_exp(mx);
    inv[side] = __uint_as_float((uint32_t)(127 - e) << 23);
    if (threadIdx.x == 0) scales[side] = __uint_as_float((uint32_t)(127 + e) << 23);
  }
  auto four = [&](const ACT *p, float i) { return codes4(ld(p, 0), ld(p, 1), ld(p, 2), ld(p, 3), i); };
  for (int x = threadIdx.x; x < CACHE_BLOCK * DH / 8; x += 64 * NW) {
    const bool val = x >= CACHE_BLOCK * DH / 16;
    const int c = (val ? x - CACHE_BLOCK * DH / 16 : x) >> 6;
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const ACT *p;
      if (val) {
        p = &v[16 * c + m][16 * q + 4 * g];   // half q >> 1, its keys' tile 2 (q >> 1) + (q & 1)
      } else if (DH == 16) {
        p = &k[16 * q + m][4 * g];
      } else {
        const int f = 2 * c + (q >> 1), t = f / NS;
        p = &k[16 * t + m][32 * (f - t * NS) + 8 * g + 4 * (q & 1)];
      }
      w[q] = four(p, inv[val]);
    }
    ((uint4 *)page)[x] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// The reverse for one word x of a page tile (words of the keys, then of the
// values): its 16 elements go to put(key, column, value).
template <int DH, typename PUT>
__device__ __forceinline__ void open_word(int x, u32x4_t w, float scale_k, float scale_v, PUT put) {
  constexpr int NS = DH >= 32 ? DH / 32 : 1;
  const int lane = x & 63, m = lane & 15, g = lane >> 4;
  const bool val = x >= CACHE_BLOCK * DH / 16;
  const int c = (val ? x - CACHE_BLOCK * DH / 16 : x) >> 6;
  const float sc = val ? scale_v : scale_k;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float e[4] = {__builtin_amdgcn_cvt_f32_fp8(w[q], 0) * sc, __builtin_amdgcn_cvt_f32_fp8(w[q], 1) * sc,
                        __builtin_amdgcn_cvt_f32_fp8(w[q], 2) * sc, __builtin_amdgcn_cvt_f32_fp8(w[q], 3) * sc};
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      if (val) {
        put(true, 16 * q + 4 * g + z, 16 * c + m, e[z]);
      } else if (DH == 16) {
        put(false, 16 * q + m, 4 * g + z, e[z]);
      } else {
        const int f = 2 * c + (q >> 1), t = f / NS;
        put(false, 16 * t + m, 32 * (f - t * NS) + 8 * g + 4 * (q & 1) + z, e[z]);
      }
    }
  }
}

}  // namespace tppsd
