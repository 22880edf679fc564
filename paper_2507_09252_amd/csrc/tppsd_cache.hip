// 8-bit paged cache: page bookkeeping, appending (quantisation), reading back,
// forks and copies. Page ids are given out lowest first and freed into a
// bitmap, so that tables depend on the calls alone, never on the order in
// which atomics arrive.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/tppsd.h"
#include "tppsd_cache_device.h"

namespace tppsd {

namespace {

constexpr int PLAN_NT = 1024;   // the bookkeeping scans run in one workgroup

__device__ __forceinline__ int ld_agent(const int32_t *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t ld_agent(const uint32_t *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// a barrier behind which the workgroup's accesses to the L2 (atomics, and the loads and stores here) are done
__device__ __forceinline__ void sync_agent() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}
__device__ __forceinline__ void st_agent(int32_t *p, int v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// running sum over the wave's lanes, this one included (row shifts, then row and half-wave broadcasts)
__device__ __forceinline__ int wave_scan(int v) {
  auto add = [&](auto ctrl, auto rows) {
    v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
  };
  add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});   // row_shr:1, 2, 4, 8
  add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
  add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
  add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});   // row_bcast:15
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});   // row_bcast:31
  return v;
}

struct Sums {
  int a, b, top;   // two exclusive sums and a maximum (of numbers below 2^24, exact as floats)
};
// over the workgroup's threads in order: *before the sums ahead of this thread,
// returned the whole (and the largest top). `sums`: a slot per wave.
__device__ Sums block_sums(Sums v, Sums *before, Sums *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const Sums x = {wave_scan(v.a), wave_scan(v.b), (int)lanes_max((float)v.top)};
  if (waves == 1) {
    before->a = x.a - v.a;
    before->b = x.b - v.b;
    return {__builtin_amdgcn_readlane(x.a, 63), __builtin_amdgcn_readlane(x.b, 63), x.top};
  }
  __syncthreads();   // (the last call's sums have been read)
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  // lane w has the sums of wave w
  const Sums mine = lane < waves ? sums[lane] : Sums{0, 0, 0};
  const int ra = wave_scan(mine.a), rb = wave_scan(mine.b);
  const int last = waves - 1, prev = max(wave - 1, 0);
  const int ua = __builtin_amdgcn_readfirstlane(__shfl(ra, prev, 64)), ub = __builtin_amdgcn_readfirstlane(__shfl(rb, prev, 64));
  before->a = (wave ? ua : 0) + x.a - v.a;
  before->b = (wave ? ub : 0) + x.b - v.b;
  return {__shfl(ra, last, 64), __shfl(rb, last, 64), (int)lanes_max((float)mine.top)};
}

// The set bits of bits[0 .. nbits) in ascending order into list, from word w0 on, until at least
// `want` are found; returns how many (at most want).
__device__ int list_bits(const uint32_t *bits, int nbits, int w0, int want, int32_t *list, Sums *sums) {
  const int words = (nbits + 31) / 32;
  int found = 0;
  for (; w0 < words && found < want; w0 += blockDim.x) {
    const int w = w0 + threadIdx.x;
    uint32_t m = w < words ? ld_agent(bits + w) : 0u;
    Sums before;
    const Sums all = block_sums(Sums{(int)__popc(m), 0, 0}, &before, sums);
    int k = found + before.a;
    while (m && k < want) {
      const int bit = __ffs(m) - 1;
      m &= m - 1;
      list[k++] = w * 32 + bit;
    }
    found += all.a;
  }
  __syncthreads();   // the list is complete (one workgroup: its global writes are visible past the barrier)
  return min(found, want);
}

// gives pages [j0, j1) of a sequence's table back, a workgroup's threads
// together: the last holder sets a page's bit. counts[2], where the search for
// free pages begins, is one address for the whole chip: it is read first, and
// as it only falls here, hardly any thread has to write it.
__device__ __forceinline__ void pages_drop(const CacheDev &c, int s, int j0, int j1) {
  const int seen = c.counts[2];
  int low = INT32_MAX;
  for (int j = j0 + threadIdx.x; j < j1; j += blockDim.x) {
    int32_t *e = &c.table[(size_t)s * c.NP + j];
    const int page = *e;
    *e = -1;
    if (atomicSub(&c.refs[page], 1) == 1) {
      atomicOr(&c.freeb[page >> 5], 1u << (page & 31));
      low = min(low, page >> 5);
    }
  }
  if (low < seen) atomicMin(&c.counts[2], low);
}

// Whether a sequence of n positions has an open block that the ring (from block
// `low` on) no longer holds: a call of more than two blocks that was dropped has
// taken its place. Until the sequence ends at a block's border again `low` only
// rises, so that nothing takes the slots' rows for that block's.
__device__ __forceinline__ bool open_lost(int n, int low) { return n % CACHE_BLOCK != 0 && n / CACHE_BLOCK < low; }

// Positions of a sequence that another can take over: without the open block
// where that is lost.
__device__ __forceinline__ int sound_len(const CacheDev &c, int s) {
  const int n = c.lens[s], low = c.low[s];
  return open_lost(n, low) ? n / CACHE_BLOCK * CACHE_BLOCK : n;
}

// whole pages that a sequence of n positions has to share or copy: never more than it holds
// (entries of the table behind those are -1)
__device__ __forceinline__ int pages_of(const CacheDev &c, int s, int n) { return min(n / CACHE_BLOCK, c.held[s]); }

__global__ void k_cache_reset(CacheDev c) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x, n = (size_t)gridDim.x * blockDim.x;
  for (size_t j = i; j < (size_t)c.S * c.NP; j += n) c.table[j] = -1;
  for (size_t j = i; j < (size_t)c.S; j += n)
    c.lens[j] = c.held[j] = c.low[j] = c.pend[j] = c.planned[j] = 0;
  for (size_t j = i; j < (size_t)c.L * c.S; j += n) c.came[j] = 0;
  for (size_t j = i; j < (size_t)c.n_pages; j += n) c.refs[j] = 0;
  for (size_t j = i; j < (size_t)(c.n_pages + 31) / 32; j += n) {
    const int left = c.n_pages - (int)j * 32;
    c.freeb[j] = left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u;
    c.mark[j] = 0u;
  }
  for (size_t j = i; j < (size_t)CACHE_JOINS; j += n) c.joins[j] = 0;
  if (i == 0) {
    *c.status = 0u;
    c.counts[2] = 0;
    c.counts[PLAN_ID] = 0;
  }
}

__device__ __forceinline__ int next_plan(int plan) { return (plan + 1) & 0x3FFFFFFF; }   // (stored doubled as well)
// a plan in progress is dropped: what it brought is nobody's
__device__ __forceinline__ void drop_plan(const CacheDev &c) { c.counts[PLAN_ID] = next_plan(c.counts[PLAN_ID]); }

// Plans a call: which sequence each row of the batch names, its first new
// position and how many it brings; pages for the blocks that become whole; and
// the attention's work items. One workgroup, as many threads as rows (PER rows
// a thread past 1024, held in registers; 0: any number, in memory): the batch's
// bookkeeping is a few integers a row, and two sums over the rows are all that
// threads exchange. Plans that take next to no pages: 64 rows 2.9 us, 4096 rows
// 13 us. Pages are given out by each row's thread one after another, some 0.35 us
// each: one row of 500 pages 183 us, 48 rows of 40 17, 48 of 500 180, 4096 of one 63.
template <int PER> __global__ __launch_bounds__(PLAN_NT) void k_cache_begin(CacheDev c, CacheBegin b) {
  __shared__ Sums sums[PLAN_NT / 64];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int per = PER ? PER : (b.B + nt - 1) / nt, i0 = min(b.B, tid * per), n = min(b.B, i0 + per) - i0;
  struct Row {
    int seq, start, cnt, held;
  };
  Row mem[PER ? PER : 1];
  // f(i, row of the batch, its plan): the plan stays between passes
  auto each = [&](bool first, auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int k = 0; k < PER; ++k)
        if (k < n) f(i0 + k, mem[k]);
    } else {
      for (int k = 0; k < n; ++k) {
        const int i = i0 + k;
        Row r;
        if (!first) {
          r.seq = c.p_seq[i], r.start = c.p_start[i], r.cnt = c.p_count[i];
          r.held = r.seq >= 0 ? c.held[r.seq] : 0;
        }
        f(i, r);
        c.p_seq[i] = r.seq, c.p_start[i] = r.start, c.p_count[i] = r.cnt;
      }
    }
  };
  if (b.seqs) {
    // a sequence that is named twice belongs to the first row that names it
    for (int k = 0; k < n; ++k) {
      const int s = b.seqs[i0 + k];
      if (s >= 0 && s < c.S) st_agent(&c.owner[s], INT32_MAX);
    }
    sync_agent();
    for (int k = 0; k < n; ++k) {
      const int s = b.seqs[i0 + k];
      if (s >= 0 && s < c.S) atomicMin(&c.owner[s], i0 + k);
    }
    sync_agent();
  }
  auto top_of = [&](const Row &r) { return r.cnt > 0 ? (r.start + r.cnt - 1) / CACHE_BLOCK : 0; };
  auto need_of = [&](const Row &r) { return r.cnt > 0 ? max(0, (r.start + r.cnt) / CACHE_BLOCK - r.held) : 0; };
  const int hint = c.counts[2], plan = next_plan(c.counts[PLAN_ID]);
  Sums mine = {0, 0, 0}, before;
  each(true, [&](int i, Row &r) {
    const int s = b.seqs ? b.seqs[i] : i;
    bool ok = s >= 0 && s < c.S;
    if (ok && b.seqs) ok = ld_agent(&c.owner[s]) == i;
    r = {ok ? s : -1, 0, 0, 0};
    if (ok) {
      const int want = b.counts ? b.counts[i] : b.P, done = b.done ? b.done[i] : 0;
      r.held = c.held[s];
      r.start = b.start_in ? b.start_in[i] + b.start_off : c.lens[s];
      r.cnt = done ? 0 : min(max(want, 0), b.P);
      if (b.start_in && !done) c.lens[s] = r.start;
      if (r.start < 0 || r.cnt > c.max_events - r.start) {
        if (r.cnt > 0) atomicOr(c.status, TPPSD_STATUS_CAPACITY);
        r.cnt = 0;
      }
    } else {
      atomicOr(c.status, TPPSD_STATUS_SEQUENCE);
    }
    mine.a += need_of(r);
    mine.b += top_of(r);
    mine.top = max(mine.top, top_of(r));
  });
  Sums all = block_sums(mine, &before, sums);
  const int avail = all.a > 0 ? list_bits(c.freeb, c.n_pages, hint, all.a, c.list, sums) : 0;
  int off = before.a;
  mine.b = mine.top = 0;
  each(false, [&](int i, Row &r) {
    if (r.seq >= 0) {
      const int need = need_of(r);
      if (need > 0) {
        if (off + need <= avail) {
          for (int j = 0; j < need; ++j) {
            const int page = c.list[off + j];
            c.table[(size_t)r.seq * c.NP + r.held + j] = page;
            c.refs[page] = 1;
            atomicAnd(&c.freeb[page >> 5], ~(1u << (page & 31)));
          }
          c.held[r.seq] = r.held + need;
          if (off + need == avail) c.counts[2] = c.list[avail - 1] >> 5;   // (no free page before the last one taken)
        } else {   // the rows before took the pages that were left
          atomicOr(c.status, TPPSD_STATUS_PAGES);
          r.cnt = 0;
        }
        off += need;
      }
      c.pend[r.seq] = r.cnt;
      if (r.cnt > 0) {
        const int low = c.low[r.seq];
        const bool lost = open_lost(r.start, low);
        if (lost) atomicOr(c.status, TPPSD_STATUS_OPEN);
        c.planned[r.seq] = plan << 1 | (lost ? 1 : 0);
        c.low[r.seq] = max(top_of(r) - 1, lost ? low : min(low, r.start / CACHE_BLOCK));
      }
    }
    if (PER > 0) c.p_seq[i] = r.seq, c.p_start[i] = r.start, c.p_count[i] = r.cnt;
    mine.b += top_of(r);
    mine.top = max(mine.top, top_of(r));
  });
  if (tid == 0) c.counts[PLAN_ID] = plan;
  if (avail < all.a && b.split_target > 0) all = block_sums(mine, &before, sums);   // (rows were left out)
  // Work items. Rows of about equal length that fill the chip are taken whole.
  // Otherwise pages are dealt out in pieces of a workgroup's share, or, where
  // many rows leave many remainders, of a third of it (ragged rows of 8 heads of
  // 64, a share and a third: 4 rows of up to 32000 14.2 and 19.4 us, 16 19.6 and
  // 21.0, 64 of up to 16000 31.8 and 30.2). Pieces of a row have adjoining slots
  // for their partial states.
  if (b.split_target <= 0) return;   // (the attention reads the rows)
  int chunk = INT32_MAX;
  const int share = (all.b + b.split_target - 1) / b.split_target, parts = b.B * 4 <= b.split_target ? 1 : 3;
  if (all.top > share + share / 4)
    chunk = max(CACHE_MIN_PIECE, (all.b + parts * b.split_target - 1) / (parts * b.split_target));
  auto pieces = [&](int top) { return top <= chunk ? 1 : (top + chunk - 1) / chunk; };
  mine = {0, 0, 0};
  each(false, [&](int, Row &r) {
    const int k = pieces(top_of(r));
    mine.a += k;
    mine.b += k > 1 ? k : 0;
  });
  all = block_sums(mine, &before, sums);
  each(false, [&](int i, Row &r) {
    CacheItem it;
    it.row = i;
    it.seq = r.seq;
    it.start = r.start;
    it.count = r.cnt;
    const int top = top_of(r);
    it.pieces = pieces(top);
    it.slot0 = before.b;
    it.lo = 0;
    for (it.piece = 0; it.piece < it.pieces; ++it.piece) {
      it.hi = it.piece + 1 == it.pieces ? top : it.lo + chunk;
      c.items[before.a++] = it;
      it.lo = it.hi;
    }
    if (it.pieces > 1) before.b += it.pieces;
  });
  if (tid == 0) c.counts[0] = all.a;
}

__global__ void k_cache_commit(CacheDev c, int B, const int32_t *accept) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= B) return;
  const int s = c.p_seq[i], cnt = c.p_count[i];
  if (s < 0 || cnt <= 0) return;
  int n = c.p_start[i] + (accept ? min(max(accept[i], 0), cnt) : cnt);
  const int planned = c.planned[s];
  if (planned & 1) n = c.p_start[i];   // (rows behind a lost block are no good either)
  if (open_lost(n, c.low[s])) {
    atomicOr(c.status, TPPSD_STATUS_OPEN);
    n = n / CACHE_BLOCK * CACHE_BLOCK;
  }
  c.lens[s] = n;
  c.pend[s] = 0;
  c.planned[s] = planned & ~1;
}

__global__ void k_cache_truncate(CacheDev c, const int32_t *seqs, const int32_t *lens) {
  __shared__ int range[2];
  const int s = seqs[blockIdx.x];
  if (blockIdx.x == 0 && threadIdx.x == 0) drop_plan(c);
  if (threadIdx.x == 0) {
    range[0] = range[1] = 0;
    int n = lens ? lens[blockIdx.x] : 0;
    if (s < 0 || s >= c.S || n < 0) {
      atomicOr(c.status, TPPSD_STATUS_SEQUENCE);
    } else {
      const int len = ld_agent(&c.lens[s]);
      if (n >= len) {
        n = len;
      } else if (open_lost(n, c.low[s])) {
        atomicOr(c.status, TPPSD_STATUS_OPEN);
        n = n / CACHE_BLOCK * CACHE_BLOCK;
      }
      // minima: a sequence that is named twice keeps the shorter length, and
      // each of its pages is let go by one of the two
      atomicMin(&c.lens[s], n);
      range[0] = n / CACHE_BLOCK;
      range[1] = atomicMin(&c.held[s], range[0]);
      c.pend[s] = 0;
    }
  }
  __syncthreads();
  pages_drop(c, s, range[0], range[1]);
}

// Whether pair i of a fork or copy is carried out: both sequences exist, no pair
// before it names its destination and, within one cache, none as its source. A
// pair of two negative numbers is none. Every workgroup looks through the whole
// list for the pair it is about (few pairs; their verdicts depend on the list alone).
__device__ bool pair_stands(const CacheDev &to, const CacheDev &from, int n, const int32_t *src, const int32_t *dst,
                            int i, bool same) {
  const int s = src[i], d = dst[i];
  bool bad = s < 0 || s >= from.S || d < 0 || d >= to.S;
  const bool none = s < 0 && d < 0;
  if (!bad) {
    for (int j = threadIdx.x; j < n; j += blockDim.x) {
      const int sj = src[j], dj = dst[j];
      if (sj < 0 || sj >= from.S || dj < 0 || dj >= to.S) continue;
      bad |= (dj == d && j < i) || (same && sj == d);
    }
    bad = __syncthreads_or(bad);
  }
  if (bad && !none && threadIdx.x == 0) atomicOr(to.status, TPPSD_STATUS_SEQUENCE);
  return !bad;
}
// The same for long lists, once for all pairs, into to.p_seq: the first pair of
// each destination and the sources are marked in LDS, or for more sequences
// than that holds in memory. Lists of 256 pairs and fewer are looked through by
// the working kernel (forks in four layers, so and with this launch in front:
// 256 pairs 11.7 and 10.9 + 2.1 us, 512 20.5 and 19.1 + 3.9, 2048 98 and 87 + 5).
constexpr int FEW_PAIRS = 256, LDS_SEQS = 12288;
template <bool LDS>
__global__ __launch_bounds__(PLAN_NT) void k_cache_pairs(CacheDev to, CacheDev from, int n, const int32_t *src,
                                                         const int32_t *dst, int same) {
  __shared__ int32_t marks[LDS ? LDS_SEQS : 1];
  __shared__ uint32_t sources[LDS ? LDS_SEQS / 32 : 1];
  auto ok = [&](int s, int d) { return s >= 0 && s < from.S && d >= 0 && d < to.S; };
  if (LDS) {
    for (int i = threadIdx.x; i < to.S; i += PLAN_NT) marks[i] = INT32_MAX;
    for (int i = threadIdx.x; i < (to.S + 31) / 32; i += PLAN_NT) sources[i] = 0u;
    __syncthreads();
  } else {
    for (int i = threadIdx.x; i < n; i += PLAN_NT)
      if (ok(src[i], dst[i])) {
        st_agent(&to.owner[dst[i]], INT32_MAX);
        st_agent(&to.role[dst[i]], 0);
        if (same) st_agent(&to.role[src[i]], 0);
      }
    sync_agent();
  }
  for (int i = threadIdx.x; i < n; i += PLAN_NT) {
    const int s = src[i], d = dst[i];
    if (!ok(s, d)) continue;
    if (LDS) {
      atomicMin(&marks[d], i);
      if (same) atomicOr(&sources[s >> 5], 1u << (s & 31));
    } else {
      atomicMin(&to.owner[d], i);
      if (same) atomicOr(&to.role[s], 1);
    }
  }
  if (LDS) __syncthreads();
  else sync_agent();
  for (int i = threadIdx.x; i < n; i += PLAN_NT) {
    const int s = src[i], d = dst[i];
    bool good = ok(s, d);
    if (good) {
      const int first = LDS ? marks[d] : ld_agent(&to.owner[d]);
      const bool source = LDS ? (sources[d >> 5] >> (d & 31) & 1u) != 0 : ld_agent(&to.role[d]) != 0;
      good = first == i && !(same && source);
    }
    if (!good && (s >= 0 || d >= 0)) atomicOr(to.status, TPPSD_STATUS_SEQUENCE);
    to.p_seq[i] = good ? 1 : 0;
  }
}
__device__ __forceinline__ bool pair_goes(const CacheDev &to, const CacheDev &from, int n, const int32_t *src,
                                          const int32_t *dst, int i, bool same) {
  return n <= FEW_PAIRS ? pair_stands(to, from, n, src, dst, i, same) : to.p_seq[i] != 0;
}

// open rows of a source sequence (len mod 64 of them) into the destination's
// ring, of layers l0, l0 + step, ..: 16 bytes a thread, the rows of all heads and
// sides one after the other
__device__ void copy_tail(const CacheDev &to, const CacheDev &from, int l0, int step, int s, int d, int len) {
  const int open = len % CACHE_BLOCK, slot0 = len / CACHE_BLOCK * CACHE_BLOCK % CACHE_RING;
  if (open == 0) return;
  const int row16 = to.dh * (to.bf16 ? 2 : 4) / 16, side16 = CACHE_RING * row16, sides = to.KV * 2;   // 16-byte words
  const int sh = __builtin_ctz(row16), word = threadIdx.x & (row16 - 1), rows = blockDim.x >> sh;
  const int r0 = threadIdx.x >> sh, q = rows / open, rem = rows - q * open;
  for (int layer = l0; layer < to.L; layer += step) {
    const uint4 *a = (const uint4 *)from.tails + (((size_t)layer * from.S + s) * sides) * side16 + slot0 * row16 + word;
    uint4 *b = (uint4 *)to.tails + (((size_t)layer * to.S + d) * sides) * side16 + slot0 * row16 + word;
    int side = r0 / open, r = r0 - side * open;
    while (side < sides) {
      const size_t at = (size_t)side * side16 + r * row16;
      b[at] = a[at];
      r += rem;
      side += q;
      if (r >= open) r -= open, ++side;
    }
  }
}

// Grid (pairs, 1 + groups of layers): the table and counters, then the layers'
// open rows. Latency for few pairs (7: 4 us), memory for many (1792 x 6 layers,
// 142 MB: 36 us).
__global__ __launch_bounds__(256) void k_cache_fork(CacheDev c, int n, const int32_t *src, const int32_t *dst) {
  const int i = blockIdx.x;
  if (i == 0 && blockIdx.y == 0 && threadIdx.x == 0) drop_plan(c);
  if (!pair_goes(c, c, n, src, dst, i, true)) return;
  const int s = src[i], d = dst[i];
  if (blockIdx.y > 0) {   // (the slots of a lost block go along, for nothing: the destination ends before them)
    copy_tail(c, c, blockIdx.y - 1, gridDim.y - 1, s, d, c.lens[s]);
    return;
  }
  const int len = sound_len(c, s), np = pages_of(c, s, len);
  pages_drop(c, d, 0, c.held[d]);
  __syncthreads();
  for (int j = threadIdx.x; j < np; j += blockDim.x) {
    const int page = c.table[(size_t)s * c.NP + j];
    atomicAdd(&c.refs[page], 1);
    c.table[(size_t)d * c.NP + j] = page;
  }
  if (threadIdx.x == 0) {
    if (len < c.lens[s]) atomicOr(c.status, TPPSD_STATUS_OPEN);
    c.lens[d] = len;
    c.held[d] = np;
    c.low[d] = np;
    c.pend[d] = 0;
  }
}

// the source's pages that move (its bitmap `mark` is zero between calls); verdicts into to.p_seq
__global__ __launch_bounds__(256) void k_copy_mark(CacheDev to, CacheDev from, int n, const int32_t *src,
                                                   const int32_t *dst) {
  const int i = blockIdx.x, s = src[i], d = dst[i];
  bool go = pair_goes(to, from, n, src, dst, i, false);
  if (go && sound_len(from, s) > to.max_events) {
    if (threadIdx.x == 0) atomicOr(to.status, TPPSD_STATUS_CAPACITY);
    go = false;
  }
  if (threadIdx.x == 0) to.p_seq[i] = go ? 1 : 0;
  if (!go) return;
  const int np = pages_of(from, s, sound_len(from, s));
  for (int j = threadIdx.x; j < np; j += blockDim.x) {
    const int page = from.table[(size_t)s * from.NP + j];
    atomicOr(&from.mark[page >> 5], 1u << (page & 31));
  }
  pages_drop(to, d, 0, to.held[d]);
  __syncthreads();
  if (threadIdx.x == 0) to.lens[d] = to.held[d] = to.low[d] = to.pend[d] = 0;
}

// the marked pages in ascending order get the destination's lowest free pages
__global__ __launch_bounds__(PLAN_NT) void k_copy_plan(CacheDev to, CacheDev from) {
  __shared__ Sums sums[PLAN_NT / 64];
  const int n = list_bits(from.mark, from.n_pages, 0, from.n_pages, from.list, sums);
  const int avail = n > 0 ? list_bits(to.freeb, to.n_pages, to.counts[2], n, to.list, sums) : 0;
  const bool fits = avail == n;
  for (int k = threadIdx.x; k < n && fits; k += PLAN_NT) {
    const int page = to.list[k];
    from.map[from.list[k]] = page;
    to.refs[page] = 0;
    atomicAnd(&to.freeb[page >> 5], ~(1u << (page & 31)));
  }
  for (int w = threadIdx.x; w < (from.n_pages + 31) / 32; w += PLAN_NT) from.mark[w] = 0u;
  if (threadIdx.x == 0) {
    drop_plan(to);
    to.counts[1] = fits ? n : -1;
    if (fits && n > 0) to.counts[2] = to.list[n - 1] >> 5;
    if (!fits) atomicOr(to.status, TPPSD_STATUS_PAGES);
  }
}

// Bound by memory: 310 MB of pages in 128 us, 4.8 TB/s read and written.
// grid.x = n Y workgroups for the sequences (table and counters, Y - 1 groups of layers), the rest for the pages
__global__ __launch_bounds__(256) void k_copy_data(CacheDev to, CacheDev from, int n, int Y, const int32_t *src,
                                                   const int32_t *dst) {
  const int pages = to.counts[1];
  if (pages < 0) return;
  const int seq_wgs = n * Y;
  if ((int)blockIdx.x < seq_wgs) {
    const int i = blockIdx.x % n, y = (int)blockIdx.x / n;
    if (!to.p_seq[i]) return;
    const int s = src[i], d = dst[i];
    if (y > 0) {   // (as in k_cache_fork)
      copy_tail(to, from, y - 1, Y - 1, s, d, from.lens[s]);
    } else {
      const int len = sound_len(from, s), np = pages_of(from, s, len);
      for (int j = threadIdx.x; j < np; j += blockDim.x) {
        const int page = from.map[from.table[(size_t)s * from.NP + j]];
        to.table[(size_t)d * to.NP + j] = page;
        atomicAdd(&to.refs[page], 1);
      }
      if (threadIdx.x == 0) {
        if (len < from.lens[s]) atomicOr(to.status, TPPSD_STATUS_OPEN);
        to.lens[d] = len;
        to.held[d] = to.low[d] = np;
      }
    }
    return;
  }
  const size_t words = to.KV * page_tile(to) / 16;   // 16-byte words of a page's layer
  const size_t wgs = gridDim.x - seq_wgs;
  for (size_t w = blockIdx.x - seq_wgs; w < (size_t)pages * to.L; w += wgs) {
    const int layer = (int)(w / pages), k = (int)(w - (size_t)layer * pages);
    const size_t a = (size_t)layer * from.n_pages + from.list[k], b = (size_t)layer * to.n_pages + to.list[k];
    const uint4 *x = (const uint4 *)from.pages + a * words;
    uint4 *y = (uint4 *)to.pages + b * words;
    for (size_t j = threadIdx.x; j < words; j += blockDim.x) y[j] = x[j];
    for (int j = threadIdx.x; j < 2 * to.KV; j += blockDim.x)
      to.scales[b * 2 * to.KV + j] = from.scales[a * 2 * to.KV + j];
  }
}

// Appends to one layer. Grid (row, key/value head, block of positions that the
// rows reach): the block's rows go through LDS; its new rows into the ring
// where the ring keeps them (the last two blocks), and a block that becomes
// whole is rounded to 8 bits and written as a page tile. Reads each new row
// once and writes one byte per element of a whole block: bound by memory (32
// histories of 2560 positions, 8 heads of 64: 252 MB in 64 us, 3.9 TB/s; a few
// rows 3.7 us, one chain of loads).
template <typename ACT, int DH>
__global__ __launch_bounds__(256) void k_cache_append(CacheDev c, int layer, int P, CacheRows r) {
  constexpr int LDK = DH + 16 / sizeof(ACT), LDV = CACHE_BLOCK + 4, C8 = DH / 8;
  __shared__ __align__(16) ACT ks[CACHE_BLOCK][LDK];   // keys, row per position
  __shared__ __align__(16) ACT vs[DH][LDV];            // values, row per column
  __shared__ float top[2][4];
  const int i = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int s = c.p_seq[i], cnt = c.p_count[i], start = c.p_start[i], plan = c.counts[PLAN_ID];
  if (s < 0 || cnt <= 0) return;
  const int end = start + cnt, first = start / CACHE_BLOCK, last = (end - 1) / CACHE_BLOCK;
  const int blk = first + blockIdx.z;
  if (blk > last) return;
  const int base = blk * CACHE_BLOCK, n = min(CACHE_BLOCK, end - base);
  const bool whole = n == CACHE_BLOCK, long_call = P > CACHE_BLOCK;
  ACT *const ring = (ACT *)c.tails + (((size_t)layer * c.S + s) * c.KV + h) * 2 * CACHE_RING * DH;
  // The first block's slots may be those of a block that the ring keeps: that
  // block's rows go in with the first block, behind the reads of the old ones.
  const int later = (last - first) % 2 == 0 ? last : last - 1;
  const bool shares = later > first && start % CACHE_BLOCK != 0;
  const bool keep = blk >= last - 1 && !(shares && blk == later);
  // 8 elements of new row p from column j on, of the keys and of the values
  auto fetch = [&](int p, int j, Eight<ACT> &k, Eight<ACT> &v) {
    k.load((const ACT *)r.k + i * r.k_sb + (size_t)p * r.k_sp + h * r.k_sh + j);
    const ACT *vp = (const ACT *)r.v + i * r.v_sb + h * r.v_sh;
    if (r.v_blocked) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v.put(e, vp[(size_t)(p >> 3) * 8 * DH + (j + e) * 8 + (p & 7)]);
    } else {
      v.load(vp + (size_t)p * r.v_sp + j);
    }
  };
  float top_k = 0.f, top_v = 0.f;
  constexpr int IT = (CACHE_BLOCK * C8 + 255) / 256;
  Eight<ACT> k[IT], v[IT];
#pragma unroll
  for (int x = 0; x < IT; ++x) {
    const int at = min(tid + 256 * x, CACHE_BLOCK * C8 - 1), row = min(at / C8, n - 1), j = at % C8 * 8, pos = base + row;
    if (pos >= start) {
      fetch(pos - start, j, k[x], v[x]);
    } else {
      k[x].load(ring + pos % CACHE_RING * DH + j);
      v[x].load(ring + (CACHE_RING + pos % CACHE_RING) * DH + j);
    }
  }
  if (shares && blk == first) __syncthreads();   // (every wave has its old rows)
#pragma unroll
  for (int x = 0; x < IT; ++x) {
    const int at = tid + 256 * x, row = at / C8, j = at % C8 * 8, pos = base + row;
    if (at >= CACHE_BLOCK * C8 || row >= n) continue;
    if (pos < start) {
      if (long_call) {   // the attention of this call still needs the old rows
        ACT *st = (ACT *)c.stash + (((size_t)i * c.KV + h) * 2 * CACHE_BLOCK + row) * DH + j;
        k[x].store(st);
        v[x].store(st + CACHE_BLOCK * DH);
      }
    } else if (keep) {
      k[x].store(ring + pos % CACHE_RING * DH + j);
      v[x].store(ring + (CACHE_RING + pos % CACHE_RING) * DH + j);
    }
    if (whole) {
      k[x].store(&ks[row][j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const ACT kv = k[x].at(e), vv = v[x].at(e);
        vs[j + e][row] = vv;
        top_up(top_k, ld(&kv, 0));
        top_up(top_v, ld(&vv, 0));
      }
    }
  }
  if (shares && blk == first) {
    const int n2 = min(CACHE_BLOCK, end - later * CACHE_BLOCK);
    for (int at = tid; at < n2 * C8; at += 256) {
      const int j = at % C8 * 8, pos = later * CACHE_BLOCK + at / C8;
      Eight<ACT> k2, v2;
      fetch(pos - start, j, k2, v2);
      k2.store(ring + pos % CACHE_RING * DH + j);
      v2.store(ring + (CACHE_RING + pos % CACHE_RING) * DH + j);
    }
  }
  if (blk == first && h == 0 && tid == 0) c.came[(size_t)layer * c.S + s] = plan;
  if (!whole) return;
  top_k = lanes_max(top_k);
  top_v = lanes_max(top_v);
  if (lane == 0) top[0][wave] = top_k, top[1][wave] = top_v;
  __syncthreads();
  const size_t tile = ((size_t)layer * c.n_pages + c.table[(size_t)s * c.NP + blk]) * c.KV + h;
  seal_page<ACT, DH, 4>(ks, vs, top, c.pages + tile * (2 * CACHE_BLOCK * DH), c.scales + tile * 2);
}

// Rows first[i] .. first[i] + count - 1 of sequences, as the cache holds them:
// whole blocks from their codes, through LDS, the open block from the ring;
// positions past the sequence are left as they were. A plan's positions are the
// sequence's once the layer has them and while the plan stands; a lost open
// block is not (but for the plan that follows it). Grid (row, head, block).
// Bound by memory (the histories above in 48 us).
template <typename ACT, int DH>
__global__ __launch_bounds__(256) void k_cache_read(CacheDev c, int layer, const int32_t *seqs, const int32_t *first,
                                                    int count, ACT *k, ACT *v) {
  constexpr int LD = DH + 16 / sizeof(ACT), C8 = DH / 8;
  __shared__ __align__(16) ACT rows[2][CACHE_BLOCK][LD];
  const int i = blockIdx.x, h = blockIdx.y, s = seqs ? seqs[i] : i, tid = threadIdx.x;
  const int f = first ? first[i] : 0;
  if (s < 0 || s >= c.S || f < 0) {
    if (tid == 0) atomicOr(c.status, TPPSD_STATUS_SEQUENCE);
    return;
  }
  const int blk = f / CACHE_BLOCK + blockIdx.z, base = blk * CACHE_BLOCK;
  const int page_id = c.table[(size_t)s * c.NP + min(blk, c.NP - 1)];   // (with the loads below)
  const int len = c.lens[s], pend = c.pend[s], plan = c.counts[PLAN_ID];
  const bool has = c.came[(size_t)layer * c.S + s] == plan;
  int end = has ? len + pend : len;
  const int planned = c.planned[s];
  if (!has && (planned >> 1 == plan ? (planned & 1) != 0 : open_lost(len, c.low[s]))) {
    if (tid == 0) atomicOr(c.status, TPPSD_STATUS_OPEN);
    end = len / CACHE_BLOCK * CACHE_BLOCK;
  }
  const int lo = max(f, base), hi = min(base + CACHE_BLOCK, f > end ? f : min(end, count > end - f ? end : f + count));
  if (lo >= hi) return;
  const bool whole = base + CACHE_BLOCK <= end;
  if (whole) {
    const size_t tile = ((size_t)layer * c.n_pages + page_id) * c.KV + h;
    const u32x4_t *page = (const u32x4_t *)(c.pages + tile * (2 * CACHE_BLOCK * DH));
    const float sk = c.scales[tile * 2], sv = c.scales[tile * 2 + 1];
    for (int x = tid; x < CACHE_BLOCK * DH / 8; x += 256)
      open_word<DH>(x, page[x], sk, sv, [&](bool val, int key, int col, float e) { st(&rows[val][key][col], 0, e); });
    __syncthreads();
  }
  const ACT *ring = (const ACT *)c.tails + (((size_t)layer * c.S + s) * c.KV + h) * 2 * CACHE_RING * DH;
  for (int x = tid; x < 2 * (hi - lo) * C8; x += 256) {
    const int sd = x >= (hi - lo) * C8, y = sd ? x - (hi - lo) * C8 : x, pos = lo + y / C8, j = y % C8 * 8;
    Eight<ACT> w;
    w.load(whole ? &rows[sd][pos - base][j] : ring + (sd * CACHE_RING + pos % CACHE_RING) * DH + j);
    w.store((sd ? v : k) + (((size_t)i * count + (pos - f)) * c.KV + h) * DH + j);
  }
}

template <typename F> void by_width(const CacheDev &c, F f) {
  auto widths = [&](auto act) {
    if (c.dh == 16) f(act, std::integral_constant<int, 16>{});
    else if (c.dh == 32) f(act, std::integral_constant<int, 32>{});
    else if (c.dh == 64) f(act, std::integral_constant<int, 64>{});
    else f(act, std::integral_constant<int, 128>{});
  };
  if (c.bf16) widths(bf16_t{});
  else widths(float{});
}

}  // namespace

void launch_cache_reset(const CacheDev &c, hipStream_t st) {
  const size_t n = std::max((size_t)c.S * c.NP, (size_t)c.n_pages);
  k_cache_reset<<<(unsigned)std::min<size_t>((n + 255) / 256, 1024), 256, 0, st>>>(c);
}

void launch_cache_begin(const CacheDev &c, const CacheBegin &b, hipStream_t st) {
  const int nt = std::min(PLAN_NT, (b.B + 63) / 64 * 64);
  if (b.B <= PLAN_NT) k_cache_begin<1><<<1, nt, 0, st>>>(c, b);
  else if (b.B <= 4 * PLAN_NT) k_cache_begin<4><<<1, nt, 0, st>>>(c, b);
  else k_cache_begin<0><<<1, nt, 0, st>>>(c, b);
}

void launch_cache_append(const CacheDev &c, int layer, int B, int P, const CacheRows &r, hipStream_t st) {
  const dim3 grid(B, c.KV, (CACHE_BLOCK - 1 + P + CACHE_BLOCK - 1) / CACHE_BLOCK);
  by_width(c, [&](auto act, auto w) {
    k_cache_append<decltype(act), decltype(w)::value><<<grid, 256, 0, st>>>(c, layer, P, r);
  });
}

void launch_cache_commit(const CacheDev &c, int B, const int32_t *accept, hipStream_t st) {
  k_cache_commit<<<(B + 255) / 256, 256, 0, st>>>(c, B, accept);
}

void launch_cache_truncate(const CacheDev &c, int n, const int32_t *seqs, const int32_t *lens, hipStream_t st) {
  k_cache_truncate<<<n, 256, 0, st>>>(c, seqs, lens);
}

static void judge_pairs(const CacheDev &to, const CacheDev &from, int n, const int32_t *src, const int32_t *dst,
                        int same, hipStream_t st) {
  if (n <= FEW_PAIRS) return;   // (the working kernels do)
  if (to.S <= LDS_SEQS) k_cache_pairs<true><<<1, PLAN_NT, 0, st>>>(to, from, n, src, dst, same);
  else k_cache_pairs<false><<<1, PLAN_NT, 0, st>>>(to, from, n, src, dst, same);
}

// workgroups that share a sequence's layers (a layer each while that makes some ten thousand)
static int layer_groups(int L, int n) { return std::max(1, std::min(L, 32768 / n)); }

void launch_cache_fork(const CacheDev &c, int n, const int32_t *src, const int32_t *dst, hipStream_t st) {
  judge_pairs(c, c, n, src, dst, 1, st);
  k_cache_fork<<<dim3(n, 1 + layer_groups(c.L, n)), 256, 0, st>>>(c, n, src, dst);
}

void launch_cache_copy(const CacheDev &to, const CacheDev &from, int n, const int32_t *src, const int32_t *dst,
                       hipStream_t st) {
  judge_pairs(to, from, n, src, dst, 0, st);
  k_copy_mark<<<n, 256, 0, st>>>(to, from, n, src, dst);
  k_copy_plan<<<1, PLAN_NT, 0, st>>>(to, from);
  const int Y = 1 + layer_groups(to.L, n);
  k_copy_data<<<n * Y + 2048, 256, 0, st>>>(to, from, n, Y, src, dst);
}

void launch_cache_read(const CacheDev &c, int layer, int n, const int32_t *seqs, const int32_t *first, int count,
                       void *k, void *v, hipStream_t st) {
  const dim3 grid(n, c.KV, (count + 2 * CACHE_BLOCK - 2) / CACHE_BLOCK);   // (blocks that count positions may reach)
  by_width(c, [&](auto act, auto w) {
    typedef decltype(act) ACT;
    k_cache_read<ACT, decltype(w)::value><<<grid, 256, 0, st>>>(c, layer, seqs, first, count, (ACT *)k, (ACT *)v);
  });
}

}  // namespace tppsd
