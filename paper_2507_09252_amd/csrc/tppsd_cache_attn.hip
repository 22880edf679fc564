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

#include "tppsd_cache_device.h"

namespace tppsd {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int EIGHT_PAGES = 32;   // pages of a sequence at its longest from which eight waves share it

// 8 values as bf16 operands: one part for bf16 sources; for fp32 three parts
// that add up to the value (each the bf16 rounding of what the ones before
// leave)
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

// the operand of a query or key row at p (8 elements, 4 for d_head 16), part by part into to(part)
template <typename ACT, int DH, typename TO> __device__ __forceinline__ void load_k(const ACT *p, TO to) {
  if constexpr (sizeof(ACT) == 2) {
    to(0) = *(const std::remove_reference_t<decltype(to(0))> *)p;
  } else {
    float x[8] = {};
    const f32x4_t a = *(const f32x4_t *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i];
    if constexpr (DH >= 32) {
      const f32x4_t b = *(const f32x4_t *)(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 + i] = b[i];
    }
#pragma unroll
    for (int n = 0; n < 3; ++n) {
      const uint4 w = take8(x, n < 2);
      if constexpr (DH >= 32) to(n) = __builtin_bit_cast(bf16x8_t, w);
      else to(n) = __builtin_bit_cast(short4_t, make_uint2(w.x, w.y));
    }
  }
}

// bits 15 and 31: the halves of w that are not finite bf16 (an exponent of ones carries into the sign's place)
__device__ __forceinline__ uint32_t bf_odd(uint32_t w) { return (w & 0x7FFF7FFFu) + 0x00800080u; }
// halves of w that are not finite bf16, as 0xFFFF
__device__ __forceinline__ uint32_t bf_bad(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}

// 8 elements of a key with its infinities as NaN: a product of infinity with an
// element of the other sign would be a score of -inf, a weight of 0, and the key
// as good as masked. (fp32 keys have it from their parts: inf - inf.)
__device__ __forceinline__ Eight<bf16_t> nan_keys(Eight<bf16_t> k) {
#pragma unroll
  for (int i = 0; i < 4; ++i) k.w[0][i] |= bf_odd(k.w[0][i]) >> 9 & 0x00400040u;
  return k;
}
__device__ __forceinline__ Eight<float> nan_keys(const Eight<float> &k) { return k; }
// whether any of 8 elements is not finite
__device__ __forceinline__ bool any_odd(const Eight<bf16_t> &v) {
  uint32_t x = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) x |= bf_odd(v.w[0][i]);
  return (x & 0x80008000u) != 0u;
}
__device__ __forceinline__ bool any_odd(const Eight<float> &v) {
  bool x = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) x |= not_finite(v.at(e));
  return x;
}

// The operand of 8 values of a column, four at p and four at p + 16, in parts;
// clean: those that are not finite as 0, or (bad) 1 in their place and 0 elsewhere.
template <int NP> __device__ __forceinline__ void value8(const bf16_t *p, bool clean, bf16x8_t (&v)[NP]) {
  const uint2 a = *(const uint2 *)p, b = *(const uint2 *)(p + 16);
  uint4 w = make_uint4(a.x, a.y, b.x, b.y);
  if (clean) w = make_uint4(w.x & ~bf_bad(w.x), w.y & ~bf_bad(w.y), w.z & ~bf_bad(w.z), w.w & ~bf_bad(w.w));
  v[0] = __builtin_bit_cast(bf16x8_t, w);
}
template <int NP> __device__ __forceinline__ void value8(const float *p, bool clean, bf16x8_t (&v)[NP]) {
  const f32x4_t a = *(const f32x4_t *)p, b = *(const f32x4_t *)(p + 16);
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  if (clean)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = not_finite(x[i]) ? 0.f : x[i];
  split8<NP>(x, v);
}
__device__ __forceinline__ bf16x8_t bad8(const bf16_t *p) {
  const uint2 a = *(const uint2 *)p, b = *(const uint2 *)(p + 16);
  const uint32_t one = 0x3F803F80u;
  return __builtin_bit_cast(bf16x8_t, make_uint4(bf_bad(a.x) & one, bf_bad(a.y) & one, bf_bad(b.x) & one, bf_bad(b.y) & one));
}
__device__ __forceinline__ bf16x8_t bad8(const float *p) {
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float *q = p + (i >> 1) * 16 + (i & 1) * 2;
    y[i] = (not_finite(q[0]) ? 0x3F80u : 0u) | (not_finite(q[1]) ? 0x3F800000u : 0u);
  }
  return __builtin_bit_cast(bf16x8_t, make_uint4(y[0], y[1], y[2], y[3]));
}

// What a wave holds of its query rows: operands, running maxima, sums and
// outputs. NP: bf16 parts of a query or probability (1 for bf16 models, 3 for
// fp32); MT: tiles of 16 query rows.
template <typename ACT, int DH, int MT> struct Rows {
  static constexpr int NP = sizeof(ACT) == 2 ? 1 : 3;
  static constexpr int NS = DH >= 32 ? DH / 32 : 1;   // k steps of a score
  static constexpr int NU = DH / 16;                  // column tiles; also 16-byte words of a lane per side
  typedef typename std::conditional<DH >= 32, bf16x8_t, short4_t>::type kfrag;

  kfrag q[MT][NP][NS];
  f32x4_t o[MT][NU];
  f32x4_t l1[MT];     // bf16: sums of the rounded probabilities (rows of ones through the matrix unit)
  float l[MT], m[MT]; // fp32: this lane's keys' sum; running maximum, in base-2 units
  int pos[MT];        // position of this lane's query
  float scale2;       // scale log2 e: exponentials are one exp2 each
  int g;

  // A block's 64 keys are taken at once, or, where four tiles' scores fill the
  // registers, in two halves
  static constexpr int STEPS = MT == 4 || DH == 128 ? 2 : 1, TILES = 4 / STEPS, HALVES = 2 / STEPS;

  // Scores and probabilities of step w: kf(tile, k step, part) gives the key
  // operand of KP parts, seen(t, key) whether this lane's query of tile t sees it.
  template <int KP, bool MASK, typename KF, typename SEEN>
  __device__ __forceinline__ void scores(int w, KF kf, SEEN seen, bf16x8_t (&p)[MT][NP][HALVES]) {
    f32x4_t s[MT][TILES];
#pragma unroll
    for (int k4 = 0; k4 < TILES; ++k4) {
#pragma unroll
      for (int t = 0; t < MT; ++t) s[t][k4] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < NS; ++ks)
#pragma unroll
        for (int a = 0; a < KP; ++a) {
          const kfrag k = kf(TILES * w + k4, ks, a);
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int b = 0; b < NP; ++b)
              if (a + b <= 2) s[t][k4] = mma(k, q[t][b][ks], s[t][k4]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      float mx = -INFINITY;
#pragma unroll
      for (int k4 = 0; k4 < TILES; ++k4)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (MASK && !seen(t, 16 * (TILES * w + k4) + 4 * g + i)) s[t][k4][i] = -INFINITY;
          mx = fmaxf(mx, s[t][k4][i]);
        }
      mx *= scale2;
      // The running maximum moves only when a score passes it by 2^8: until then
      // probabilities stay below 2^8, which fp32 sums and bf16 operands carry
      // as well, and a step costs no exchange between lanes and no rescaling.
      if (__ballot(mx > m[t] + 8.f) != 0ull) {
        const float m_new = fmaxf(m[t], xor32_max(xor16_max(mx)));
        const float alpha = __builtin_amdgcn_exp2f(m[t] - (m_new == -INFINITY ? 0.f : m_new));
        m[t] = m_new;
        l[t] *= alpha;
        l1[t] *= alpha;
#pragma unroll
        for (int u = 0; u < NU; ++u) o[t][u] *= alpha;
      }
      const float ref = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
      for (int hf = 0; hf < HALVES; ++hf) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = __builtin_amdgcn_exp2f(fmaf(s[t][2 * hf + (j >> 2)][j & 3], scale2, -ref));
          if (NP > 1) l[t] += x[j];
        }
        bf16x8_t part[NP];
        split8<NP>(x, part);
#pragma unroll
        for (int b = 0; b < NP; ++b) p[t][b][hf] = part[b];
      }
    }
    if (NP == 1) {
      const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int hf = 0; hf < HALVES; ++hf) l1[t] = mma(ones, p[t][0][hf], l1[t]);
    }
  }
  // a block: o += P V, vf(column tile, half of the keys, part)
  template <int KP, bool MASK, typename KF, typename VF, typename SEEN>
  __device__ __forceinline__ void block(KF kf, VF vf, SEEN seen) {
#pragma unroll
    for (int w = 0; w < STEPS; ++w) {
      bf16x8_t p[MT][NP][HALVES];
      scores<KP, MASK>(w, kf, seen, p);
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
          for (int a = 0; a < KP; ++a) {
            const bf16x8_t v = vf(u, HALVES * w + hf, a);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
              for (int b = 0; b < NP; ++b)
                if (a + b <= 2) o[t][u] = mma(v, p[t][b][hf], o[t][u]);
          }
    }
  }
  // Where values of a tile are not finite the operands hold 0 in their place;
  // bad(u, w) holds 1 there: NaN for the queries that see such a key, nothing for the others.
  template <typename BAD, typename SEEN> __device__ __forceinline__ void poison(BAD bad, SEEN seen) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      bf16x8_t vis[2];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint32_t x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = 16 * (2 * w + (j >> 1)) + 4 * g + 2 * (j & 1);
          x[j] = (seen(t, key) ? 0x3F80u : 0u) | (seen(t, key + 1) ? 0x3F800000u : 0u);
        }
        vis[w] = __builtin_bit_cast(bf16x8_t, make_uint4(x[0], x[1], x[2], x[3]));
      }
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        f32x4_t b = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 2; ++w) b = mma(bad(u, w), vis[w], b);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][u][i] = b[i] > 0.f ? NAN : o[t][u][i];
      }
    }
  }
  // folds another wave's (or split's) state of the same rows into this one
  template <typename M, typename L, typename O> __device__ __forceinline__ void fold(M om, L ol, O oo) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const float mo = om(t), mn = fmaxf(m[t], mo), ref = mn == -INFINITY ? 0.f : mn;
      const float fa = __builtin_amdgcn_exp2f(m[t] - ref), fb = __builtin_amdgcn_exp2f(mo - ref);
      m[t] = mn;
      l[t] = l[t] * fa + ol(t) * fb;
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const f32x4_t x = oo(t, u);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][u][i] = o[t][u][i] * fa + x[i] * fb;
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

// Query rows of a workgroup: a chunk of the query heads that share the
// key/value head, of consecutive positions. ONE: a call's positions all at once
// (they reach at most two blocks, as they are at most 64). Otherwise groups
// that stay inside a block of 64 positions, so that a group has one block to see as
// its rows came and none to see in part.
struct Group {
  int hc, gh, ppg, gpb;   // heads of a chunk, chunks, positions of a group, groups of a block
};
__host__ __device__ inline Group group_of(int G, int rows) {
  Group x;
  x.hc = G < rows ? G : rows;
  x.gh = (G + x.hc - 1) / x.hc;
  x.ppg = rows / x.hc;
  if (x.ppg > CACHE_BLOCK) x.ppg = CACHE_BLOCK;
  x.gpb = (CACHE_BLOCK + x.ppg - 1) / x.ppg;
  return x;
}
inline int groups_of(int G, int rows, int P, bool one) {
  const Group x = group_of(G, rows);
  // (an int: at most 2^24 + 1 blocks of 64 groups, saturated)
  const long n = ((long)P + 2 * CACHE_BLOCK - 2) / CACHE_BLOCK * x.gpb * x.gh;
  return one ? 1 : (int)std::min<long>(n, INT32_MAX);
}

// Waves per SIMD that the registers are held to: a workgroup's first and last
// steps are latency, which others hide (a chunk of 16 x 1001 rows with one wave
// per SIMD 120 us, with two 71); fp32 rows of 128 columns need them all.
constexpr int min_waves(int dh, int mt, bool bf16) { return !bf16 ? (dh == 128 ? 1 : 2) : dh * mt <= 64 && mt < 4 ? 4 : 2; }

// Attention of a work item (a row of the batch and a range of its pages) for
// one key/value head and one group of query rows. The NW waves share the
// queries and take the pages round robin, each with its own running softmax,
// folded at the end; the splits of a row are joined by the workgroup that
// finishes last. HINT: rows of at least nt_pages read them with the non-temporal
// hint (an instance of its own: a second page loop costs short rows a few
// per cent in instruction fetches). The item with the row's last pages also takes the blocks that
// the queries see as their rows came, from LDS. ONE: that item appends the
// call's rows to the cache as well (ring, and pages of blocks that became
// whole), so that a decoding step is one launch.
//
// Bound by memory for long rows (32 x 4600 positions, 8 heads of 64, 17 new: 32
// us a layer, 4.8 TB/s; 32 x 16000 89 us, 5.9 TB/s), by one chain of dependent
// loads and steps for short ones (fp32, heads of 16: 5 us for one sequence of
// 220, 10 for 64 of 550). Chunks (16 rows of up to 1001 new positions after up to
// 2000: 73 us, 270 TFLOP/s) use nothing up: SIMDs issue VALU instructions in 34 %
// of the launch's cycles and MFMA is busy in 13 %, waves wait 42 % of theirs, and
// compute units have work in two thirds of them. A wave has about three pages,
// and around them come the queries' load, the window's staging, one wave's step
// on the own block while three wait, and the fold.
template <typename ACT, int DH, int MT, int NW, bool ONE, bool HINT>
__global__ __launch_bounds__(64 * NW, min_waves(DH, MT, sizeof(ACT) == 2)) void k_cache_attend(CacheDev c, CacheAttend a) {
  typedef Rows<ACT, DH, MT> R;
  constexpr int NP = R::NP, NS = R::NS, NU = R::NU, NT = 64 * NW;
  constexpr int WIN = ONE ? 2 * CACHE_BLOCK : CACHE_BLOCK;   // rows as they came that a group may see
  constexpr int LDK = DH + 16 / sizeof(ACT), LDV = WIN + 4;
  typedef typename R::kfrag kfrag;
  constexpr int FOLD = NW / 2;
  struct Win {
    ACT k[WIN][LDK];      // keys, row per position
    ACT v[DH][LDV];       // values, row per column
  };
  struct Fold {
    f32x4_t o[FOLD][MT * NU][64];
    float m[FOLD][MT][64], l[FOLD][MT][64];
  };
  union Shared {
    Win win;
    Fold fold;
  };
  __shared__ __align__(16) char shared[sizeof(Shared)];
  __shared__ float top[2][NW];
  __shared__ int last_of_row;
  Win &win = *(Win *)shared;
  Fold &fold = *(Fold *)shared;

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, rr = lane & 15, g = lane >> 4;
  const int h = blockIdx.y, G = c.H / c.KV, item = blockIdx.x;
  const int plan = ONE ? c.counts[PLAN_ID] : 0;
  CacheItem it;
  if (a.whole) {   // rows are not split: the plan's rows say it all
    it.row = item;
    it.seq = c.p_seq[item], it.start = c.p_start[item], it.count = c.p_count[item];
    it.lo = it.piece = it.slot0 = 0;
    it.hi = it.count > 0 ? (it.start + it.count - 1) / CACHE_BLOCK : 0;
    it.pieces = 1;
  } else {
    if (item >= c.counts[0]) return;
    it = c.items[item];
  }
  const int i = it.row, cnt = it.count, start = it.start, seq = it.seq;
  const size_t head0 = (size_t)h * G * DH;
  ACT *const O = (ACT *)a.o;
  // this group: query heads hd0 .. + hn - 1 of positions p0 .. + pn - 1
  const Group grp = group_of(G, 16 * MT);
  int hd0 = 0, hn = G, p0 = start, pn = cnt, z = 0;
  if (!ONE) {
    z = gridDim.z - 1 - blockIdx.z;   // the groups with the most keys first
    const int gh = z % grp.gh, sub = z / grp.gh % grp.gpb, blk = z / grp.gh / grp.gpb;
    hd0 = gh * grp.hc;
    hn = min(grp.hc, G - hd0);
    const int b0 = (start / CACHE_BLOCK + blk) * CACHE_BLOCK, lo = b0 + sub * grp.ppg;
    p0 = max(start, lo);
    pn = min(start + cnt, min(lo + grp.ppg, b0 + CACHE_BLOCK)) - p0;
  }
  if (cnt <= 0) {
    if (a.zero && (ONE || z == 0))
      for (int x = tid; x < a.P * G * DH; x += NT)
        O[((size_t)i * a.P + x / (G * DH)) * a.ldo + head0 + x % (G * DH)] = 0;
    return;
  }
  if (pn <= 0) return;   // (the group's position range of this row is empty: for all its splits)
  const int end = start + cnt;
  const int ba = p0 / CACHE_BLOCK, bb = (p0 + pn - 1) / CACHE_BLOCK;
  const bool tail = it.piece + 1 == it.pieces;
  // the split that takes the group's own block: the one whose pages it is among,
  // or would follow
  const bool mine = ONE ? tail : (it.lo <= ba && ba < it.hi) || (tail && ba >= it.hi);
  R s;
  s.g = g;
  s.scale2 = a.scale * LOG2E;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = min(16 * t + rr, pn * hn - 1);   // (rows past the last repeat it and are not stored)
    const int p = r / hn, hd = hd0 + r - p * hn;
    s.pos[t] = p0 + p;
    const ACT *qp = (const ACT *)a.q + ((size_t)i * a.P + (p0 - start + p)) * a.ldq + head0 + hd * DH;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) load_k<ACT, DH>(qp + (DH >= 32 ? 32 * ks + 8 * g : 4 * g), [&](int b) -> kfrag & { return s.q[t][b][ks]; });
    s.m[t] = -INFINITY;
    s.l[t] = 0.f;
    s.l1[t] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NU; ++u) s.o[t][u] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  }

  // ---- rows of the queries' own blocks, into LDS (and the cache) ------------
  const size_t layer0 = (size_t)a.layer * c.n_pages;
  const int32_t *table = c.table + (size_t)seq * c.NP;
  const int j0 = it.lo, j1 = min(it.hi, ba);
  auto tile_of = [&](int page) { return (layer0 + page) * c.KV + h; };
  // (nt: pages that the next pass will not find in a cache pass the caches by)
  auto load_side = [&](uint4 (&w)[NU], size_t tile, int side, auto nt) {
    const u32x4_t *p = (const u32x4_t *)(c.pages + tile * (2 * CACHE_BLOCK * DH)) + side * (64 * NU) + lane;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if constexpr (decltype(nt)::value) w[u] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(p + 64 * u));
      else w[u] = ((const uint4 *)p)[64 * u];
    }
  };
  auto word = [](const uint4 &x, int n) { return n == 0 ? x.x : n == 1 ? x.y : n == 2 ? x.z : x.w; };
  auto k_codes = [&](const uint4 (&w)[NU], float sc, int t4, int ks) -> kfrag {
    if constexpr (DH >= 32) {
      const int f = t4 * NS + ks;
      return dec8(word(w[f >> 1], 2 * (f & 1)), word(w[f >> 1], 2 * (f & 1) + 1), sc);
    } else {
      return dec4(word(w[0], t4), sc);
    }
  };
  // page ids and scales of the wave's next 64 pages, one per lane, and its first
  // page's keys: on their way while the rows below are
  int jc = j0 + wave, id = 0;
  float2 sc = {0.f, 0.f};
  uint4 kw[NU];
  auto fetch = [&] {
    id = table[min(jc + lane * NW, j1 - 1)];
    sc = *(const float2 *)(c.scales + tile_of(id) * 2);
    load_side(kw, tile_of(__builtin_amdgcn_readlane(id, 0)), 0, std::false_type{});
  };
  if (jc < j1) fetch();
  int any_bad = 0;
  if (mine) {
    const int base = ba * CACHE_BLOCK, n = min(end - base, WIN);
    const ACT *ring = (const ACT *)c.tails + (((size_t)a.layer * c.S + seq) * c.KV + h) * 2 * CACHE_RING * DH;
    const ACT *stash = (const ACT *)c.stash + ((size_t)i * c.KV + h) * 2 * CACHE_BLOCK * DH;
    const bool in_ring = a.P <= CACHE_BLOCK;   // rows from before the call (longer ones have moved them to the stash)
    constexpr int C8 = DH / 8;                 // pieces of 8 elements of a row
    const CacheRows &src = a.kv;
    int bad = 0;
    float top_k = 0.f, top_v = 0.f;   // largest finite elements of the first block
    for (int x = tid; x < WIN * C8; x += NT) {
      const int row = x / C8, j = (x - row * C8) * 8, pos = base + row;
      const ACT *kp, *vp;
      bool blocked = false;
      if (pos < start) {
        const ACT *from = in_ring ? ring + (pos % CACHE_RING) * DH : stash + row * DH;
        kp = from + j;
        vp = from + (in_ring ? CACHE_RING : CACHE_BLOCK) * DH + j;
      } else {
        const int pr = min(pos, end - 1) - start;
        kp = (const ACT *)src.k + i * src.k_sb + (size_t)pr * src.k_sp + h * src.k_sh + j;
        blocked = src.v_blocked != 0;
        vp = (const ACT *)src.v + i * src.v_sb + h * src.v_sh +
             (blocked ? (size_t)(pr >> 3) * 8 * DH + j * 8 + (pr & 7) : (size_t)pr * src.v_sp + j);
      }
      Eight<ACT> kk, vv;
      const bool in = row < n;
      kk.load(kp);
      if (blocked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) vv.put(e, vp[8 * e]);
      } else {
        vv.load(vp);
      }
      nan_keys(kk).store(&win.k[row][j]);
      bad |= in && any_odd(vv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const ACT v = in ? vv.at(e) : (ACT)0, k = kk.at(e);
        win.v[j + e][row] = v;
        if (ONE && n >= CACHE_BLOCK && row < CACHE_BLOCK) top_up(top_k, ld(&k, 0)), top_up(top_v, ld(&v, 0));
      }
      if (ONE && in && pos >= start) {
        ACT *to = (ACT *)ring + (pos % CACHE_RING) * DH + j;
        kk.store(to);
        vv.store(to + CACHE_RING * DH);
      }
    }
    if (ONE && h == 0 && tid == 0) c.came[(size_t)a.layer * c.S + seq] = plan;
    any_bad = __syncthreads_or(bad);
    if constexpr (ONE) {
      if (n >= CACHE_BLOCK) {   // the first block is whole: its page
        top_k = lanes_max(top_k);
        top_v = lanes_max(top_v);
        if (lane == 0) top[0][wave] = top_k, top[1][wave] = top_v;
        __syncthreads();
        const size_t tile = tile_of(table[ba]);
        seal_page<ACT, DH, NW>(win.k, win.v, top, c.pages + tile * (2 * CACHE_BLOCK * DH), c.scales + tile * 2);
        __syncthreads();   // (the page is read below, by waves of this workgroup)
      }
    }
  }

  // ---- the pages that every query sees ------------------------------------
  if constexpr (HINT) {
    if ((end - 1) / CACHE_BLOCK >= a.nt_pages)   // (uniform)
      while (jc < j1) {
        const int n = min(64, (j1 - jc + NW - 1) / NW);
        uint4 vw[NU], kn[NU];
        for (int x = 0; x < n; ++x) {
          const float ks = lane_val(sc.x, x), vs = lane_val(sc.y, x);
          load_side(vw, tile_of(__builtin_amdgcn_readlane(id, x)), 1, std::true_type{});
          load_side(kn, tile_of(__builtin_amdgcn_readlane(id, min(x + 1, n - 1))), 0, std::true_type{});
          s.template block<1, false>([&](int t4, int k2, int) { return k_codes(kw, ks, t4, k2); },
                                     [&](int u, int w, int) { return dec8(word(vw[u], 2 * w), word(vw[u], 2 * w + 1), vs); },
                                     [](int, int) { return true; });
#pragma unroll
          for (int u = 0; u < NU; ++u) kw[u] = kn[u];
        }
        jc += 64 * NW;
        if (jc < j1) fetch();
      }
  }
  // (a loop of its own: choosing the hint page by page keeps the loads from
  // running ahead, 32 rows of 16000 positions 89 -> 100 us)
  while (jc < j1) {
    const int n = min(64, (j1 - jc + NW - 1) / NW);
    uint4 vw[NU], kn[NU];
    for (int x = 0; x < n; ++x) {
      const size_t tile = tile_of(__builtin_amdgcn_readlane(id, x));
      const float ks = lane_val(sc.x, x), vs = lane_val(sc.y, x);
      load_side(vw, tile, 1, std::false_type{});
      load_side(kn, tile_of(__builtin_amdgcn_readlane(id, min(x + 1, n - 1))), 0, std::false_type{});
      s.template block<1, false>([&](int t4, int k2, int) { return k_codes(kw, ks, t4, k2); },
                                 [&](int u, int w, int) { return dec8(word(vw[u], 2 * w), word(vw[u], 2 * w + 1), vs); },
                                 [](int, int) { return true; });
#pragma unroll
      for (int u = 0; u < NU; ++u) kw[u] = kn[u];
    }
    jc += 64 * NW;
    if (jc < j1) fetch();
  }

  // ---- the queries' own blocks, as their rows came -------------------------
  // step 0: block ba as it came; ONE, past its border: 1: block bb as it came, 2: block ba's page
  const int steps = ONE && bb > ba ? 3 : 1;
  if (mine) {
    for (int st = (wave + NW - (max(j1 - j0, 0)) % NW) % NW; st < steps; st += NW) {
      if (ONE && st == 2) {
        const size_t tile = tile_of(table[ba]);
        uint4 kw[NU], vw[NU];
        load_side(kw, tile, 0, std::false_type{});
        load_side(vw, tile, 1, std::false_type{});
        const float ks = c.scales[tile * 2], vs = c.scales[tile * 2 + 1];
        auto seen = [&](int t, int) { return s.pos[t] / CACHE_BLOCK > ba; };
        s.template block<1, true>([&](int t4, int k2, int) { return k_codes(kw, ks, t4, k2); },
                                  [&](int u, int w, int) {
                                    return dec8(drop_codes(word(vw[u], 2 * w)), drop_codes(word(vw[u], 2 * w + 1)), vs);
                                  }, seen);
        if (any_bad)   // 1.0 (code 0x38) where a code is NaN
          s.poison([&](int u, int w) {
            return dec8((nan_codes(word(vw[u], 2 * w)) >> 7) * 0x38u, (nan_codes(word(vw[u], 2 * w + 1)) >> 7) * 0x38u, 1.f); }, seen);
        continue;
      }
      const int b = ba + st, w0 = st * CACHE_BLOCK;
      auto seen = [&](int t, int key) { return s.pos[t] / CACHE_BLOCK == b && b * CACHE_BLOCK + key <= s.pos[t]; };
      kfrag kr[NP][NS];
      bf16x8_t vr[NP];
      s.template block<NP, true>(
          [&](int t4, int k2, int part) {
            if (part == 0)
              load_k<ACT, DH>(&win.k[w0 + 16 * t4 + rr][DH >= 32 ? 32 * k2 + 8 * g : 4 * g], [&](int x) -> kfrag & { return kr[x][k2]; });
            return kr[part][k2];
          },
          [&](int u, int w, int part) {
            if (part == 0) value8<NP>(&win.v[16 * u + rr][w0 + 32 * w + 4 * g], any_bad != 0, vr);
            return vr[part];
          },
          seen);
      if (any_bad)
        s.poison([&](int u, int w) { return bad8(&win.v[16 * u + rr][w0 + 32 * w + 4 * g]); }, seen);
    }
    __syncthreads();   // (the window's memory is the folding's next)
  }

  // ---- sums over the lane groups, then over the waves ----------------------
#pragma unroll
  for (int t = 0; t < MT; ++t) s.l[t] = NP == 1 ? s.l1[t][0] : xor32_sum(xor16_sum(s.l[t]));
  // wave 0 gets the state of the first `busy` waves (the others have none)
  auto fold_waves = [&](int busy) {
#pragma unroll
    for (int half = NW / 2; half > 0; half >>= 1) {
      if (busy <= half) continue;
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          fold.m[wave - half][t][lane] = s.m[t];
          fold.l[wave - half][t][lane] = s.l[t];
#pragma unroll
          for (int u = 0; u < NU; ++u) fold.o[wave - half][t * NU + u][lane] = s.o[t][u];
        }
      }
      __syncthreads();
      if (wave < half)
        s.fold([&](int t) { return fold.m[wave][t][lane]; }, [&](int t) { return fold.l[wave][t][lane]; },
               [&](int t, int u) { return fold.o[wave][t * NU + u][lane]; });
      if (half > 1) __syncthreads();
    }
  };
  fold_waves(max(j1 - j0, 0) + (mine ? steps : 0));
  if (it.pieces > 1) {
    // [slot][head][group][o, m, l][64]: lane by lane. The state goes out and comes
    // in by accesses that are coherent over the whole GPU (its dies have an L2
    // each), so that no cache has to be written back (with fences at that scope
    // instead, 48 ragged rows took 153 us, not 83): the wait puts the stores ahead
    // of the arrival.
    constexpr int N = 4 * MT * NU + 2 * MT;
    const int Z = gridDim.z;
    auto part = [&](int piece) { return c.part + (((size_t)(it.slot0 + piece) * c.KV + h) * Z + z) * N * 64 + lane; };
    int *arrived = c.joins + ((size_t)i * c.KV + h) * Z + z;
    if (wave == 0) {
      float *pp = part(it.piece);
      auto put = [&](int at, float v) { __hip_atomic_store(pp + 64 * at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) put(4 * (t * NU + u) + e, s.o[t][u][e]);
        put(4 * MT * NU + t, s.m[t]);
        put(4 * MT * NU + MT + t, s.l[t]);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (lane == 0) {
        const int before = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last_of_row = before == it.pieces - 1;
        if (before == it.pieces - 1) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    __syncthreads();
    if (!last_of_row) return;
    asm volatile("" ::: "memory");
    // the pieces, dealt to the waves in order whoever comes last
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      s.m[t] = -INFINITY;
      s.l[t] = 0.f;
#pragma unroll
      for (int u = 0; u < NU; ++u) s.o[t][u] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
    for (int x = wave; x < it.pieces; x += NW) {
      const float *pq = part(x);
      auto get = [&](int at) { return __hip_atomic_load(pq + 64 * at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
      s.fold([&](int t) { return get(4 * MT * NU + t); }, [&](int t) { return get(4 * MT * NU + MT + t); },
             [&](int t, int u) {
               const int at = 4 * (t * NU + u);
               return (f32x4_t){get(at), get(at + 1), get(at + 2), get(at + 3)};
             });
    }
    fold_waves(it.pieces);
  }
  if (wave != 0) return;
  // ---- normalise and store: lane (rr, g) holds columns 16 u + 4 g .. + 3 of query rr ----
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = 16 * t + rr;
    float f = 1.f, L = s.l[t];
    if (a.sink) {   // one more key of score 0 and value 0
      const float ms = fmaxf(s.m[t], 0.f);
      f = __builtin_amdgcn_exp2f(s.m[t] - ms);
      L = L * f + __builtin_amdgcn_exp2f(-ms);
    }
    f = f / L;
    if (r >= pn * hn) continue;
    const int p = r / hn, hd = hd0 + r - p * hn;
    ACT *op = O + ((size_t)i * a.P + (p0 - start + p)) * a.ldo + head0 + hd * DH + 4 * g;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if constexpr (NP == 1)
        *(uint2 *)(op + 16 * u) = make_uint2(pk2bf(s.o[t][u][0] * f, s.o[t][u][1] * f), pk2bf(s.o[t][u][2] * f, s.o[t][u][3] * f));
      else
        *(f32x4_t *)(op + 16 * u) = s.o[t][u] * f;
    }
  }
}

// Tiles of 16 query rows of a workgroup for R rows in all: up to four, two
// where four do not fit the registers (outputs of d_head 128; fp32's three
// parts of queries and probabilities).
constexpr int max_tiles(int dh, bool bf16) { return dh <= (bf16 ? 64 : 32) ? 4 : 2; }
int tiles_of(const CacheDev &c, long R) { return std::min(R <= 16 ? 1 : R <= 32 ? 2 : 4, max_tiles(c.dh, c.bf16)); }

// all of a call's query rows in one group
bool one_group(const CacheDev &c, int P) {
  return P <= CACHE_BLOCK && (long)P * (c.H / c.KV) <= 16 * max_tiles(c.dh, c.bf16);
}

int call_groups(const CacheDev &c, int P) {
  const int G = c.H / c.KV;
  const bool one = one_group(c, P);
  return groups_of(G, 16 * (one ? tiles_of(c, (long)P * G) : max_tiles(c.dh, c.bf16)), P, one);
}

// Waves of a workgroup: eight where their registers and LDS leave room and
// either sequences may be long or there are no more workgroups than compute
// units; four otherwise. Eight and four, bf16 heads of 64, workgroups x positions:
// 64 x 500 7.9 and 8.6 us, 256 x 500 9.9 and 10.2, 512 x 500 13.2 and 16.7, 2048 x
// 500 42 and 34, 256 x 1500 14.8 and 16.6, 512 x 4000 42.6 and 49.8, 2048 x 4000
// equal (186).
constexpr bool eight_fit(int dh, bool bf16, int mt, bool one) { return one && dh <= (bf16 ? 64 : 32) && mt < 4; }
int waves_of(const CacheDev &c, int B, int P) {
  const bool one = one_group(c, P);
  if (!eight_fit(c.dh, c.bf16, tiles_of(c, (long)P * (c.H / c.KV)), one)) return 4;
  return c.NP >= EIGHT_PAGES || (long)B * c.KV <= 256 ? 8 : 4;
}

}  // namespace

// Pages of a sequence from which they are read with the non-temporal hint: where
// those of all layers and rows are 384 MiB, which the 256 MB last-level cache
// does not keep for the next pass. Four layers of 32 x 4600 positions (620 MB)
// 150 -> 137 us; a layer of them alone (155 MB), again and again, 32.3 -> 34.4.
static int nt_pages(const CacheDev &c, int B) {
  const size_t page = (size_t)c.L * B * c.KV * 2 * CACHE_BLOCK * c.dh;
  return (int)std::min<size_t>((((size_t)384 << 20) + page - 1) / page, INT32_MAX);
}

int cache_split_target(const CacheDev &c, int B, int P) {
  const long per = (long)c.KV * call_groups(c, P), full = CACHE_SPLIT_WAVES / waves_of(c, B, P);
  return per > full || B * per > CACHE_JOINS ? 0 : (int)(full / per);
}

int cache_groups(const CacheDev &c, int P) { return call_groups(c, P); }

// items of a batch: one per row, and for a split one about three times the target more
int cache_max_items(int S, int KV) { return S + 3 * (CACHE_SPLIT_WAVES / 4 / KV + 1) + 2; }

// Partial states: a row of t pages in pieces of C >= pages / (3 target) takes
// ceil(t / C) < 2 t / C slots, so all rows at most 6 target, each of heads x
// groups states; target x heads x groups <= CACHE_SPLIT_WAVES / 4. A state is
// output, maximum and sum of up to four tiles of 16 query rows, lane by lane.
size_t cache_part_floats(const CacheDev &c) {
  const size_t most = 6 * CACHE_SPLIT_WAVES / 4;
  const size_t groups = std::min(most, c.KV * (size_t)call_groups(c, c.max_events));   // (their product with the rows fits)
  const size_t few = groups * ((size_t)c.S + (size_t)c.S * c.NP / CACHE_MIN_PIECE);
  return std::min(most, few) * (2 * 4 + 4 * 4 * (c.dh / 16)) * 64;
}

void launch_cache_attend(const CacheDev &c, const CacheAttend &call, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  CacheAttend a = call;
  const long R = (long)a.P * (c.H / c.KV);
  const bool one = one_group(c, a.P);
  const int waves = waves_of(c, a.B, a.P);
  const int target = cache_split_target(c, a.B, a.P), items = a.B + (target ? 3 * target + 1 : 0);
  a.whole = target == 0;
  a.nt_pages = nt_pages(c, a.B);
  if (!one) launch_cache_append(c, a.layer, a.B, a.P, a.kv, st);
  auto go = [&](auto act, auto width) {
    typedef decltype(act) ACT;
    constexpr int DH = decltype(width)::value;
    auto launch = [&](auto mt, auto is_one) {
      constexpr int MT = decltype(mt)::value;
      constexpr bool ONE = decltype(is_one)::value;
      const dim3 grid(items, c.KV, call_groups(c, a.P));
      auto with = [&](auto nt) {
        constexpr bool HINT = decltype(nt)::value;
        if constexpr (eight_fit(DH, sizeof(ACT) == 2, MT, ONE)) {
          if (waves == 8) {
            hipExtLaunchKernelGGL((k_cache_attend<ACT, DH, MT, 8, ONE, HINT>), grid, dim3(512), 0, st, ev0, ev1, 0, c, a);
            return;
          }
        }
        hipExtLaunchKernelGGL((k_cache_attend<ACT, DH, MT, 4, ONE, HINT>), grid, dim3(256), 0, st, ev0, ev1, 0, c, a);
      };
      if constexpr (ONE && sizeof(ACT) == 2) {   // (groups of a row share its pages; fp32 rows are bound by other things)
        if (c.NP > a.nt_pages) {
          with(std::true_type{});
          return;
        }
      }
      with(std::false_type{});
    };
    constexpr int MOST = max_tiles(DH, sizeof(ACT) == 2);
    const int mt = tiles_of(c, R);
    if (!one) launch(std::integral_constant<int, MOST>{}, std::false_type{});
    else if (mt == 1) launch(std::integral_constant<int, 1>{}, std::true_type{});
    else if (mt == 2) launch(std::integral_constant<int, 2>{}, std::true_type{});
    else launch(std::integral_constant<int, MOST>{}, std::true_type{});
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
