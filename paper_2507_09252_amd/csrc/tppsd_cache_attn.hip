// Causal attention over the 8-bit paged cache.
//
// Position i sees the blocks of 64 positions before its own through their
// codes and its own block as its rows came:
//   o_i = sum_j p_ij V_ij / (sum_j p_ij [+ the extra key of score 0]),
//   p_ij = exp(scale q_i . K_ij - m_i)
// with the running maximum and sum of an online softmax, so that one pass over
// the pages serves all new positions of a sequence.
//
// As in the 16-bit kernels S^T = K Q^T and O^T = V^T P^T run on 16x16 MFMA
// tiles, a query per column: lane 16 g + m holds the scores of query m for the
// keys 16 t + 4 g + i of key tile t, and pages store values so that the A
// operand of O^T takes those very keys. Scores never move between lanes. Codes
// become bf16 in the conversion that applies the page's scale (a power of
// two: exact), so an fp32 query needs no fp32 page: it is taken in three bf16
// parts whose products with an exact bf16 key are exact.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "tppsd_cache.h"
#include "tppsd_device.h"

namespace tppsd {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// 8 values as bf16 operands: one part for bf16 sources; for fp32 three parts
// that add up to the value (each the bf16 rounding of what the ones before
// leave)
template <int NP> struct Parts {
  bf16x8_t p[NP];
};
template <int NP> struct Parts4 {
  short4_t p[NP];
};
// nearest bf16 pairs of 8 values, and what they leave (kept in x)
__device__ __forceinline__ uint4 take8(float (&x)[8], bool rest) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = pk2bf(x[2 * i], x[2 * i + 1]);
    if (rest) {
      x[2 * i] -= __uint_as_float(w[i] << 16);
      x[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int NP> __device__ __forceinline__ void split8(float (&x)[8], bf16x8_t (&p)[NP]) {
#pragma unroll
  for (int n = 0; n < NP; ++n) p[n] = __builtin_bit_cast(bf16x8_t, take8(x, n + 1 < NP));
}

// dequantised operand of 8 (4) codes under scale s
__device__ __forceinline__ uint32_t dec2(uint32_t w, float s, bool hi) {
  return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true))
            : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
}
__device__ __forceinline__ bf16x8_t dec8(uint32_t a, uint32_t b, float s) {
  return __builtin_bit_cast(bf16x8_t, make_uint4(dec2(a, s, false), dec2(a, s, true), dec2(b, s, false), dec2(b, s, true)));
}
__device__ __forceinline__ short4_t dec4(uint32_t a, float s) {
  return __builtin_bit_cast(short4_t, make_uint2(dec2(a, s, false), dec2(a, s, true)));
}

__device__ __forceinline__ f32x4_t mma(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma(short4_t a, short4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0);
}

// NP: bf16 parts of a query or probability (1 for bf16 models, 3 for fp32);
// MT: query tiles of 16 per wave; WK: 4 = the workgroup's waves share the
// queries and split the keys, 1 = each wave has its own queries
template <typename ACT, int DH, int MT, int WK> struct Attend {
  static constexpr int NP = sizeof(ACT) == 2 ? 1 : 3;
  static constexpr int NS = DH >= 32 ? DH / 32 : 1;   // k steps of a score
  static constexpr int NU = DH / 16;                  // column tiles; also 16-byte words of a lane per side
  typedef typename std::conditional<DH >= 32, bf16x8_t, short4_t>::type kfrag;

  kfrag q[MT][NP][NS];
  f32x4_t o[MT][NU];
  f32x4_t l1[MT];     // bf16: sums of the rounded probabilities (rows of ones through the matrix unit)
  float l[MT], m[MT];
  int pos[MT];        // position of this lane's query
  float scale2;
  int rr, g;

  // One tile of 64 keys: kf(t, s, part) and vf(u, w, part) give the operands,
  // seen(t, key) whether this lane's query of tile t sees key; KP: parts of a key
  // or value (1: page codes or bf16 rows)
  template <int KP, bool MASK, typename KF, typename VF, typename SEEN>
  __device__ __forceinline__ void tile(KF kf, VF vf, SEEN seen, bool poison) {
    f32x4_t s[MT][4];
#pragma unroll
    for (int t4 = 0; t4 < 4; ++t4) {
#pragma unroll
      for (int t = 0; t < MT; ++t) s[t][t4] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < NS; ++ks) {
#pragma unroll
        for (int a = 0; a < KP; ++a) {
          const kfrag k = kf(t4, ks, a);
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int b = 0; b < NP; ++b)
              if (a + b <= 2) s[t][t4] = mma(k, q[t][b][ks], s[t][t4]);
        }
      }
    }
    bf16x8_t p[MT][NP][2], vis[MT][2];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      float mx = -INFINITY;
#pragma unroll
      for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (MASK && !seen(t, 16 * t4 + 4 * g + i)) s[t][t4][i] = -INFINITY;
          mx = fmaxf(mx, s[t][t4][i]);
        }
      if (MASK && poison)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint32_t x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int key = 16 * (2 * w + (j >> 1)) + 4 * g + 2 * (j & 1);
            x[j] = (seen(t, key) ? 0x3F80u : 0u) | (seen(t, key + 1) ? 0x3F800000u : 0u);
          }
          vis[t][w] = __builtin_bit_cast(bf16x8_t, make_uint4(x[0], x[1], x[2], x[3]));
        }
      const float m_new = fmaxf(m[t], xor32_max(xor16_max(mx)) * scale2);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m[t] - ref);
      m[t] = m_new;
      if (__ballot(alpha != 1.f) != 0ull) {
        l[t] *= alpha;
        l1[t] *= alpha;
#pragma unroll
        for (int u = 0; u < NU; ++u) o[t][u] *= alpha;
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = __builtin_amdgcn_exp2f(fmaf(s[t][2 * w + (j >> 2)][j & 3], scale2, -ref));
          if (NP > 1) l[t] += x[j];
        }
        bf16x8_t part[NP];
        split8<NP>(x, part);
#pragma unroll
        for (int b = 0; b < NP; ++b) p[t][b][w] = part[b];
      }
    }
    if (NP == 1) {
      const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int w = 0; w < 2; ++w) l1[t] = mma(ones, p[t][0][w], l1[t]);
    }
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int a = 0; a < KP; ++a) {
          const bf16x8_t v = vf(u, w, a);
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int b = 0; b < NP; ++b)
              if (a + b <= 2) o[t][u] = mma(v, p[t][b][w], o[t][u]);
        }
    if (MASK && poison) {
      // Some value of the tile is not finite (the operands above hold 0 there):
      // it reaches the queries that see its key, and no other
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          f32x4_t bad = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < 2; ++w) bad = mma(vf(u, w, -1), vis[t][w], bad);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][u][i] = bad[i] > 0.f ? NAN : o[t][u][i];
        }
    }
  }
};

// code bytes that are NaN (0x7F, 0xFF), as 0x80 in their place; and codes without them
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t drop_codes(uint32_t w) {
  const uint32_t n = nan_codes(w);
  return w & ~((n >> 7) * 0xFFu);
}

template <typename ACT, int DH, int MT, int WK>
__global__ __launch_bounds__(256) void k_cache_attend(CacheDev c, CacheAttend a) {
  typedef Attend<ACT, DH, MT, WK> A;
  constexpr int NP = A::NP, NS = A::NS, NU = A::NU;
  typedef typename A::kfrag kfrag;
  __shared__ f32x4_t fold_o[WK == 4 ? 2 : 1][WK == 4 ? MT * NU : 1][64];
  __shared__ float fold_m[2][MT][64], fold_l[2][MT][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int h = blockIdx.y, G = c.H / c.KV;
  int i, page0 = 0, page1 = INT32_MAX, item = 0;
  bool tail = true, only = true;   // takes the exact blocks; is its row's one item
  if (WK == 4) {
    item = blockIdx.x;
    if (item >= c.counts[0]) return;
    const int4 w = c.items[item];
    i = w.x;
    page0 = w.y;
    page1 = w.z;
    tail = w.w != 0;
    only = c.p_item[i + 1] - c.p_item[i] == 1;
  } else {
    i = blockIdx.x;
  }
  const int zb = gridDim.z - 1 - blockIdx.z;   // the groups with the most keys first
  const int cnt = c.p_count[i], start = c.p_start[i], seq = c.p_seq[i];
  const int r0 = (WK == 4 ? zb : zb * 4 + wave) * 16 * MT;
  const size_t head0 = (size_t)h * G * DH;
  ACT *const O = (ACT *)a.o;
  if (cnt <= 0) {
    if (a.zero)
      for (int x = lane; x < 16 * MT * DH; x += 64) {
        const int r = r0 + x / DH;
        if (r < a.P * G && (WK == 1 || wave == 0))
          O[((size_t)i * a.P + r / G) * a.ldo + head0 + (r % G) * DH + x % DH] = 0;
      }
    return;
  }
  const int R = cnt * G;
  if (r0 >= R) return;   // (no barrier ahead that other waves would wait at: WK == 4 leaves as a whole)
  A s;
  s.rr = lane & 15;
  s.g = lane >> 4;
  s.scale2 = a.scale * LOG2E;
  const int g = s.g, rr = s.rr;
  const int bb = (start + (min(r0 + 16 * MT, R) - 1) / G) / CACHE_BLOCK;   // block of the last query
  const int ba = (start + r0 / G) / CACHE_BLOCK;                           // and of the first
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = min(r0 + 16 * t + rr, R - 1);   // (rows past the last repeat it and are not stored)
    s.pos[t] = start + r / G;
    const ACT *qp = (const ACT *)a.q + ((size_t)i * a.P + r / G) * a.ldq + head0 + (r % G) * DH;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
      if constexpr (DH >= 32) {
        if constexpr (NP == 1) {
          s.q[t][0][ks] = *(const bf16x8_t *)(qp + 32 * ks + 8 * g);
        } else {
          float x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = qp[32 * ks + 8 * g + j];
          bf16x8_t part[NP];
          split8<NP>(x, part);
#pragma unroll
          for (int b = 0; b < NP; ++b) s.q[t][b][ks] = part[b];
        }
      } else if constexpr (NP == 1) {
        s.q[t][0][ks] = *(const short4_t *)(qp + 4 * g);
      } else {
        float x[8] = {qp[4 * g], qp[4 * g + 1], qp[4 * g + 2], qp[4 * g + 3], 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < NP; ++b) {
          const uint4 w = take8(x, true);
          s.q[t][b][ks] = __builtin_bit_cast(short4_t, make_uint2(w.x, w.y));
        }
      }
    }
    s.m[t] = -INFINITY;
    s.l[t] = 0.f;
    s.l1[t] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NU; ++u) s.o[t][u] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  }

  // ---- pages: blocks before the last query's -----------------------------
  const int32_t *table = c.table + (size_t)seq * c.NP;
  const size_t layer0 = (size_t)a.layer * c.n_pages;
  const int j_end = min(page1, bb);
  for (int j = page0 + (WK == 4 ? wave : 0); j < j_end; j += WK) {
    const size_t tile = (layer0 + table[j]) * c.KV + h;
    const uint4 *kp = (const uint4 *)(c.pages + tile * (2 * CACHE_BLOCK * DH)) + lane;
    uint32_t kw[NU][4], vw[NU][4];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const uint4 x = kp[64 * u], y = kp[64 * (NU + u)];
      kw[u][0] = x.x, kw[u][1] = x.y, kw[u][2] = x.z, kw[u][3] = x.w;
      vw[u][0] = y.x, vw[u][1] = y.y, vw[u][2] = y.z, vw[u][3] = y.w;
    }
    const float ks = c.scales[tile * 2], vs = c.scales[tile * 2 + 1];
    auto kf = [&](int t4, int s2, int) -> kfrag {
      if constexpr (DH >= 32) {
        const int f = t4 * NS + s2;
        return dec8(kw[f >> 1][2 * (f & 1)], kw[f >> 1][2 * (f & 1) + 1], ks);
      } else {
        return dec4(kw[0][t4], ks);
      }
    };
    if (j < ba) {   // every query sees it
      auto vf = [&](int u, int w, int) { return dec8(vw[u][2 * w], vw[u][2 * w + 1], vs); };
      s.template tile<1, false>(kf, vf, [](int, int) { return true; }, false);
    } else {
      uint32_t any = 0;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int x = 0; x < 4; ++x) any |= nan_codes(vw[u][x]);
      auto vf = [&](int u, int w, int part) {
        const uint32_t x = vw[u][2 * w], y = vw[u][2 * w + 1];
        if (part >= 0) return dec8(drop_codes(x), drop_codes(y), vs);
        // 1.0 (code 0x38) where a code is NaN
        return dec8((nan_codes(x) >> 7) * 0x38u, (nan_codes(y) >> 7) * 0x38u, 1.f);
      };
      s.template tile<1, true>(kf, vf, [&](int t, int) { return s.pos[t] / CACHE_BLOCK > j; }, __ballot(any != 0) != 0ull);
    }
  }

  // ---- the queries' own blocks, as their rows came -----------------------
  if (tail) {
    const bool ring_all = a.P <= CACHE_BLOCK;   // the append has put every row of the call into the ring
    const int end = start + cnt;
    const ACT *ring = (const ACT *)c.tails + (((size_t)a.layer * c.S + seq) * c.KV + h) * 2 * CACHE_RING * DH;
    const ACT *stash = (const ACT *)c.stash + ((size_t)i * c.KV + h) * 2 * CACHE_BLOCK * DH;
    const CacheRows &R2 = a.kv;
    auto k_row = [&](int p) -> const ACT * {
      if (ring_all) return ring + (p % CACHE_RING) * DH;
      if (p < start) return stash + (p % CACHE_BLOCK) * DH;
      return (const ACT *)R2.k + i * R2.k_sb + (size_t)(p - start) * R2.k_sp + h * R2.k_sh;
    };
    auto v_el = [&](int p, int j) -> ACT {
      if (ring_all) return ring[(CACHE_RING + p % CACHE_RING) * DH + j];
      if (p < start) return stash[(CACHE_BLOCK + p % CACHE_BLOCK) * DH + j];
      const ACT *V = (const ACT *)R2.v;
      const int pn = p - start;
      return R2.v_blocked ? V[i * R2.v_sb + h * R2.v_sh + (size_t)(pn >> 3) * 8 * DH + j * 8 + (pn & 7)]
                          : V[i * R2.v_sb + (size_t)pn * R2.v_sp + h * R2.v_sh + j];
    };
    for (int b = ba; b <= bb; ++b) {
      if (WK == 4 && ((b - ba + j_end) & 3) != wave) continue;
      const int base = b * CACHE_BLOCK;
      kfrag kr[4][NP][NS];
#pragma unroll
      for (int t4 = 0; t4 < 4; ++t4) {
        const ACT *kp = k_row(min(base + 16 * t4 + rr, end - 1));
#pragma unroll
        for (int k2 = 0; k2 < NS; ++k2) {
          if constexpr (DH >= 32) {
            if constexpr (NP == 1) {
              kr[t4][0][k2] = *(const bf16x8_t *)(kp + 32 * k2 + 8 * g);
            } else {
              float x[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) x[j] = kp[32 * k2 + 8 * g + j];
              bf16x8_t part[NP];
              split8<NP>(x, part);
#pragma unroll
              for (int n = 0; n < NP; ++n) kr[t4][n][k2] = part[n];
            }
          } else if constexpr (NP == 1) {
            kr[t4][0][k2] = *(const short4_t *)(kp + 4 * g);
          } else {
            float x[8] = {kp[4 * g], kp[4 * g + 1], kp[4 * g + 2], kp[4 * g + 3], 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NP; ++n) {
              const uint4 w = take8(x, true);
              kr[t4][n][k2] = __builtin_bit_cast(short4_t, make_uint2(w.x, w.y));
            }
          }
        }
      }
      bf16x8_t vr[NU][2][NP], vbad[NU][2];
      bool any = false;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float x[8];
          uint32_t bad[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int p = base + 16 * (2 * w + (j >> 2)) + 4 * g + (j & 3);
            const ACT e = v_el(min(p, end - 1), 16 * u + rr);
            x[j] = p < end ? ld(&e, 0) : 0.f;
            const bool nf = !(fabsf(x[j]) < INFINITY);
            any |= nf;
            bad[j] = nf ? 0x3F80u : 0u;
            x[j] = nf ? 0.f : x[j];
          }
          split8<NP>(x, vr[u][w]);
          vbad[u][w] = __builtin_bit_cast(bf16x8_t, make_uint4(bad[0] | bad[1] << 16, bad[2] | bad[3] << 16,
                                                               bad[4] | bad[5] << 16, bad[6] | bad[7] << 16));
        }
      s.template tile<NP, true>(
          [&](int t4, int k2, int part) { return kr[t4][part][k2]; },
          [&](int u, int w, int part) { return part < 0 ? vbad[u][w] : vr[u][w][part < 0 ? 0 : part]; },
          [&](int t, int key) { return s.pos[t] / CACHE_BLOCK == b && base + key <= s.pos[t]; }, __ballot(any) != 0ull);
    }
  }

  // ---- sums over the lane groups, then over the waves ---------------------
#pragma unroll
  for (int t = 0; t < MT; ++t) s.l[t] = NP == 1 ? s.l1[t][0] : xor32_sum(xor16_sum(s.l[t]));
  if constexpr (WK == 4) {
#pragma unroll
    for (int half = 2; half > 0; half >>= 1) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          fold_m[wave - half][t][lane] = s.m[t];
          fold_l[wave - half][t][lane] = s.l[t];
#pragma unroll
          for (int u = 0; u < NU; ++u) fold_o[wave - half][t * NU + u][lane] = s.o[t][u];
        }
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const float mo = fold_m[wave][t][lane], mn = fmaxf(s.m[t], mo), ref = mn == -INFINITY ? 0.f : mn;
          const float fa = __builtin_amdgcn_exp2f(s.m[t] - ref), fb = __builtin_amdgcn_exp2f(mo - ref);
          s.m[t] = mn;
          s.l[t] = s.l[t] * fa + fold_l[wave][t][lane] * fb;
#pragma unroll
          for (int u = 0; u < NU; ++u) {
            const f32x4_t x = fold_o[wave][t * NU + u][lane];
#pragma unroll
            for (int i2 = 0; i2 < 4; ++i2) s.o[t][u][i2] = s.o[t][u][i2] * fa + x[i2] * fb;
          }
        }
      }
      __syncthreads();
    }
    if (wave != 0) return;
    if (!only) {
      // [item][head][group][m, l, o][64]: what k_cache_join reads lane by lane
      constexpr int N = 2 * MT + 4 * MT * NU;
      float *pp = c.part + (((size_t)item * c.KV + h) * gridDim.z + zb) * N * 64 + lane;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        pp[64 * t] = s.m[t];
        pp[64 * (MT + t)] = s.l[t];
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2) pp[64 * (2 * MT + 4 * (t * NU + u) + i2)] = s.o[t][u][i2];
      }
      return;
    }
  }
  // ---- normalise and store: lane (rr, g) holds columns 16 u + 4 g .. + 3 of query rr ----
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = r0 + 16 * t + rr;
    float f = 1.f, L = s.l[t];
    if (a.sink) {   // one more key of score 0 and value 0
      const float ms = fmaxf(s.m[t], 0.f);
      f = __builtin_amdgcn_exp2f(s.m[t] - ms);
      L = L * f + __builtin_amdgcn_exp2f(-ms);
    }
    f = f / L;
    if (r >= R) continue;
    ACT *op = O + ((size_t)i * a.P + r / G) * a.ldo + head0 + (r % G) * DH + 4 * g;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if constexpr (NP == 1)
        *(uint2 *)(op + 16 * u) = make_uint2(pk2bf(s.o[t][u][0] * f, s.o[t][u][1] * f), pk2bf(s.o[t][u][2] * f, s.o[t][u][3] * f));
      else
        *(f32x4_t *)(op + 16 * u) = s.o[t][u] * f;
    }
  }
}

// joins the splits of a (row, head, group of query rows): one wave each
template <typename ACT, int DH, int MT>
__global__ __launch_bounds__(64) void k_cache_join(CacheDev c, CacheAttend a) {
  constexpr int NU = DH / 16, N = 2 * MT + 4 * MT * NU;
  const int i = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, rr = lane & 15, g = lane >> 4, G = c.H / c.KV;
  const int it0 = c.p_item[i], it1 = c.p_item[i + 1], R = c.p_count[i] * G, r0 = blockIdx.z * 16 * MT;
  if (it1 - it0 <= 1 || r0 >= R) return;
  const size_t step = (size_t)c.KV * gridDim.z * N * 64;
  const float *p0 = c.part + (((size_t)it0 * c.KV + h) * gridDim.z + blockIdx.z) * N * 64 + lane;
  for (int t = 0; t < MT; ++t) {
    float m = -INFINITY, l = 0.f;
    for (int x = it0; x < it1; ++x) m = fmaxf(m, p0[(x - it0) * step + 64 * t]);
    if (a.sink) m = fmaxf(m, 0.f);
    f32x4_t o[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) o[u] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    for (int x = it0; x < it1; ++x) {
      const float *pp = p0 + (x - it0) * step;
      const float f = __builtin_amdgcn_exp2f(pp[64 * t] - m);
      l += pp[64 * (MT + t)] * f;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[u][e] += pp[64 * (2 * MT + 4 * (t * NU + u) + e)] * f;
    }
    if (a.sink) l += __builtin_amdgcn_exp2f(-m);
    const int r = r0 + 16 * t + rr;
    if (r >= R) continue;
    const float f = 1.f / l;
    ACT *op = (ACT *)a.o + ((size_t)i * a.P + r / G) * a.ldo + (size_t)(h * G + r % G) * DH + 4 * g;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if constexpr (sizeof(ACT) == 2)
        *(uint2 *)(op + 16 * u) = make_uint2(pk2bf(o[u][0] * f, o[u][1] * f), pk2bf(o[u][2] * f, o[u][3] * f));
      else
        *(f32x4_t *)(op + 16 * u) = o[u] * f;
    }
  }
}

// query tiles of a wave for R rows
int tiles_of(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : 4; }

}  // namespace

// Rows of queries enough to fill the chip with four waves of their own each
// take the key range whole; otherwise the waves of a workgroup, and workgroups,
// split the keys.
static bool by_rows(const CacheDev &c, int B, int P) {
  const long R = (long)P * (c.H / c.KV);
  return R > 64 && (long)B * c.KV * ((R + 127) / 128) >= 256;
}

int cache_split_target(const CacheDev &c, int B, int P) {
  if (by_rows(c, B, P)) return 0;
  const long R = (long)P * (c.H / c.KV), groups = (R + 63) / 64;
  const long per = c.KV * groups;
  if (B * per >= CACHE_SPLIT_WGS) return 0;
  return (int)((CACHE_SPLIT_WGS + per - 1) / per);
}

// items of a call: at most one per row and split_target more
int cache_max_items(int S, int KV) { return S + CACHE_SPLIT_WGS / KV + 2; }

// Partials of a split call: items x heads x groups of query rows slots, fewer
// than 3 CACHE_SPLIT_WGS (both the rows' own and split_target's are at most
// that many, and a group more), and no more than the items that pages of
// splits of four give. A slot holds maximum, sum and output of up to four tiles
// of 16 queries, lane by lane.
size_t cache_part_floats(const CacheDev &c) {
  const size_t groups = ((size_t)c.max_events * (c.H / c.KV) + 63) / 64;
  const size_t most = (size_t)c.KV * groups * ((size_t)c.S + (size_t)c.S * c.NP / 4 + 1);
  return std::min<size_t>(3 * CACHE_SPLIT_WGS, most) * (2 * 4 + 4 * 4 * (c.dh / 16)) * 64;
}

void launch_cache_attend(const CacheDev &c, const CacheAttend &a, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const int G = c.H / c.KV;
  const long R = (long)a.P * G;
  auto go = [&](auto act, auto width) {
    typedef decltype(act) ACT;
    constexpr int DH = decltype(width)::value;
    if (by_rows(c, a.B, a.P)) {
      constexpr int MT = 2;
      hipExtLaunchKernelGGL((k_cache_attend<ACT, DH, MT, 1>), dim3(a.B, c.KV, (unsigned)((R + 64 * MT - 1) / (64 * MT))),
                            dim3(256), 0, st, ev0, ev1, 0, c, a);
      return;
    }
    const int target = cache_split_target(c, a.B, a.P), items = a.B + target;
    auto split = [&](auto mt) {
      constexpr int MT = decltype(mt)::value;
      const unsigned groups = (unsigned)((R + 16 * MT - 1) / (16 * MT));
      hipExtLaunchKernelGGL((k_cache_attend<ACT, DH, MT, 4>), dim3(items, c.KV, groups), dim3(256), 0, st, ev0, ev1, 0,
                            c, a);
      if (target) k_cache_join<ACT, DH, MT><<<dim3(a.B, c.KV, groups), 64, 0, st>>>(c, a);
    };
    const int mt = tiles_of((int)std::min<long>(R, 64));
    if (mt == 1) split(std::integral_constant<int, 1>{});
    else if (mt == 2) split(std::integral_constant<int, 2>{});
    else split(std::integral_constant<int, 4>{});
  };
  auto widths = [&](auto act) {
    if (c.dh == 16) go(act, std::integral_constant<int, 16>{});
    else if (c.dh == 32) go(act, std::integral_constant<int, 32>{});
    else if (c.dh == 64) go(act, std::integral_constant<int, 64>{});
    else go(act, std::integral_constant<int, 128>{});
  };
  if (c.bf16) widths(bf16_t{});
  else widths(float{});
}

}  // namespace tppsd
