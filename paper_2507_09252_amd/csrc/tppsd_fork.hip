// Continuing sequences of a sampler state in another state, or others of the
// same one: events, counters and contiguous caches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tppsd.h"
#include "tppsd_internal.h"

namespace tppsd {

namespace {

__global__ void k_fork_clear(uint32_t *status) { *status = 0u; }

__global__ void k_fork_pairs(ForkSide to, ForkSide from, const int32_t *parent, int same, int32_t *src, int32_t *dst) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= to.B) return;
  const int p = parent[b];
  bool ok = p >= 0 && p < from.B;
  // within one state a source stays where it is: it is nobody's destination
  if (ok && same && p != b) ok = parent[p] == p;
  if (ok && from.n[p] > to.cap) ok = false;
  if (!ok) atomicOr(to.status, TPPSD_STATUS_SEQUENCE);
  const bool go = ok && !(same && p == b);
  src[b] = go ? p : -1;
  dst[b] = go ? b : -1;
}

// grid (sequence, layer x side x head): the first len[source] positions of a
// slab, which are contiguous (values of bf16 slabs in blocks of 8 positions)
__global__ __launch_bounds__(256) void k_fork_slabs(ForkSlab to, ForkSlab from, int H, int dh,
                                                    int elt, const int32_t *src, const int32_t *dst,
                                                    const int32_t *len) {
  const int b = blockIdx.x, s = src[b];
  if (dst[b] < 0) return;
  const int h = blockIdx.y % H, side = blockIdx.y / H % 2, layer = blockIdx.y / H / 2;
  const size_t row = (size_t)dh * elt;
  const size_t n16 = (size_t)min((len[s] + 7) / 8 * 8, min(to.kv_cap, from.kv_cap)) * row / 16;
  const uint4 *x = (const uint4 *)((side ? from.v : from.k) + layer * from.layer_bytes +
                                   ((size_t)s * H + h) * from.kv_cap * row);
  uint4 *y = (uint4 *)((side ? to.v : to.k) + layer * to.layer_bytes + ((size_t)b * H + h) * to.kv_cap * row);
  for (size_t i = threadIdx.x; i < n16; i += 256) y[i] = x[i];
}

__global__ __launch_bounds__(256) void k_fork_state(ForkSide to, ForkSide from, int same, const int32_t *src,
                                                    const int32_t *dst) {
  const int b = blockIdx.x, s = src[b];
  if (dst[b] < 0) {
    if (threadIdx.x == 0 && !same) {   // nothing to continue here: an empty, finished sequence
      to.n[b] = to.gen[b] = to.lenT[b] = to.lenD[b] = to.rnd[b] = to.zeros[b] = 0;
      to.done[b] = 1;
      to.ll[b] = 0.0;
      to.acc_stats[3 * b] = to.acc_stats[3 * b + 1] = to.acc_stats[3 * b + 2] = 0ull;
    }
    return;
  }
  const int n = from.n[s];
  for (int i = threadIdx.x; i < n; i += 256) {
    to.ev_t[(size_t)b * to.cap + i] = from.ev_t[(size_t)s * from.cap + i];
    to.ev_k[(size_t)b * to.cap + i] = from.ev_k[(size_t)s * from.cap + i];
  }
  if (threadIdx.x) return;
  to.n[b] = n;
  to.gen[b] = from.gen[s];
  to.lenT[b] = from.lenT[s];
  to.lenD[b] = from.lenD[s];
  to.done[b] = from.done[s];
  to.t_end[b] = from.t_end[s];
  to.ll[b] = from.ll[s];
  if (same) {
    // draws that the sequence has not made before, for itself or its source
    const uint32_t r = max((uint32_t)to.rnd[b], (uint32_t)from.rnd[s]);
    to.rnd[b] = (int32_t)(((r >> FORK_SHIFT) + 1u) << FORK_SHIFT);
  } else {
    to.rnd[b] = from.rnd[s];
    to.zeros[b] = 0;
    to.acc_stats[3 * b] = to.acc_stats[3 * b + 1] = to.acc_stats[3 * b + 2] = 0ull;
  }
}

__global__ __launch_bounds__(256) void k_fork_done(ForkSide to) {
  __shared__ int part[4];
  int c = 0;
  for (int i = threadIdx.x; i < to.B; i += 256) c += to.done[i] != 0;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) c += __shfl_down(c, d, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = c;
  __syncthreads();
  if (threadIdx.x == 0) *to.n_done = part[0] + part[1] + part[2] + part[3];
}

}  // namespace

void launch_fork_pairs(const ForkSide &to, const ForkSide &from, const int32_t *parent, int same, int32_t *src,
                       int32_t *dst, hipStream_t st) {
  if (!same) k_fork_clear<<<1, 1, 0, st>>>(to.status);
  k_fork_pairs<<<(to.B + 255) / 256, 256, 0, st>>>(to, from, parent, same, src, dst);
}

void launch_fork_slabs(const ForkSlab &to, const ForkSlab &from, int B, int L, int H, int dh, int elt,
                       const int32_t *src, const int32_t *dst, const int32_t *len, hipStream_t st) {
  k_fork_slabs<<<dim3(B, L * H * 2), 256, 0, st>>>(to, from, H, dh, elt, src, dst, len);
}

void launch_fork_state(const ForkSide &to, const ForkSide &from, int same, const int32_t *src, const int32_t *dst,
                       hipStream_t st) {
  k_fork_state<<<to.B, 256, 0, st>>>(to, from, same, src, dst);
  k_fork_done<<<1, 256, 0, st>>>(to);
}

}  // namespace tppsd
