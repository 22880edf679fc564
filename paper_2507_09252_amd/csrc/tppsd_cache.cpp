// Host side of the 8-bit paged cache: geometry, workspace layout, argument
// checks and the launches of each entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/tppsd.h"
#include "tppsd_cache.h"
#include "tppsd_internal.h"

using namespace tppsd;

static_assert(TPPSD_CACHE_BLOCK == CACHE_BLOCK && TPPSD_CACHE_RING == CACHE_RING, "public geometry");

struct tppsd_cache {
  CacheDev d{};
  bool ready = false;    // tppsd_cache_reset has run
  int B = 0, P = 0;      // the plan in progress (B 0: none)
};

namespace {

constexpr size_t ALIGN = 256;
constexpr int MAX_SEQS = 1 << 20, MAX_EVENTS = 1 << 30, MAX_PAGES = 1 << 26;
// entries of all sequences' tables: a plan sums pages over its rows in 32 bits
constexpr long long MAX_TABLE = 1LL << 30;
// products of the limits pass 64 bits: sizes are summed in 128, and no workspace has more bytes than this
typedef unsigned __int128 bytes_t;
constexpr bytes_t MAX_BYTES = (bytes_t)1 << 48;

struct Entry {
  const char *name;
  size_t off;
};
constexpr int N_ENTRIES = 6;
bytes_t view(CacheDev *c, char *ws, Entry *entries);

int check_cfg(const tppsd_cache_cfg *c, CacheDev *d) {
  if (!c) return fail(TPPSD_E_ARG, "null cache configuration");
  if (c->n_layers < 1 || c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads)
    return fail(TPPSD_E_CONFIG, "need n_layers >= 1 and n_heads a multiple of n_kv_heads >= 1");
  if (c->n_layers > 65534 || c->n_heads > 65535) return fail(TPPSD_E_CONFIG, "too many layers or heads");
  if (c->d_head != 16 && c->d_head != 32 && c->d_head != 64 && c->d_head != 128)
    return fail(TPPSD_E_CONFIG, "d_head %d not in {16, 32, 64, 128}", c->d_head);
  if (c->prec != TPPSD_PREC_FP32 && c->prec != TPPSD_PREC_BF16)
    return fail(TPPSD_E_CONFIG, "unsupported precision %d", c->prec);
  if (c->max_seqs < 1 || c->max_seqs > MAX_SEQS || c->max_events < 1 || c->max_events > MAX_EVENTS)
    return fail(TPPSD_E_ARG, "need 1 <= max_seqs <= %d and 1 <= max_events <= %d", MAX_SEQS, MAX_EVENTS);
  const long long np = (c->max_events + CACHE_BLOCK - 1LL) / CACHE_BLOCK;
  const long long pages = c->n_pages ? c->n_pages : np * c->max_seqs;
  if (pages < 1 || pages > MAX_PAGES) return fail(TPPSD_E_ARG, "%lld pages outside 1..%d", pages, MAX_PAGES);
  if (np * c->max_seqs > MAX_TABLE)
    return fail(TPPSD_E_ARG, "%d sequences of %lld pages: more than %lld table entries", c->max_seqs, np, MAX_TABLE);
  d->L = c->n_layers;
  d->H = c->n_heads;
  d->KV = c->n_kv_heads;
  d->dh = c->d_head;
  d->bf16 = c->prec == TPPSD_PREC_BF16;
  d->S = c->max_seqs;
  d->NP = (int)np;
  d->n_pages = (int)pages;
  d->max_events = c->max_events;
  if (view(d, nullptr, nullptr) > MAX_BYTES) return fail(TPPSD_E_ARG, "a workspace of more than 2^48 bytes");
  return TPPSD_OK;
}

bytes_t view(CacheDev *c, char *ws, Entry *entries) {
  bytes_t off = 0;
  int n = 0;
  auto take = [&](auto *&p, bytes_t bytes, const char *name = nullptr) {
    off = (off + ALIGN - 1) / ALIGN * ALIGN;
    p = ws ? (std::remove_reference_t<decltype(p)>)(ws + (size_t)off) : nullptr;
    if (name && entries) entries[n++] = {name, (size_t)off};
    off += bytes;
  };
  const bytes_t L = c->L, S = c->S, KV = c->KV, N = c->n_pages, dh = c->dh, e = c->bf16 ? 2 : 4;
  take(c->pages, L * N * KV * 2 * CACHE_BLOCK * dh, "pages");
  take(c->scales, L * N * KV * 2 * 4, "scales");
  take(c->tails, L * S * KV * 2 * CACHE_RING * dh * e, "tails");
  take(c->table, S * c->NP * 4, "table");
  take(c->lens, S * 4, "lens");
  take(c->refs, N * 4, "refs");
  take(c->held, S * 4);
  take(c->low, S * 4);
  take(c->pend, S * 4);
  take(c->planned, S * 4);
  take(c->came, L * S * 4);
  take(c->freeb, (N + 31) / 32 * 4);
  take(c->owner, S * 4);
  take(c->role, S * 4);
  take(c->list, N * 4);
  take(c->map, N * 4);
  take(c->mark, (N + 31) / 32 * 4);
  take(c->counts, 32);
  take(c->p_seq, S * 4);
  take(c->p_start, S * 4);
  take(c->p_count, S * 4);
  c->max_items = cache_max_items(c->S, c->KV);
  take(c->items, (bytes_t)c->max_items * sizeof(CacheItem));
  take(c->part, (bytes_t)cache_part_floats(*c) * 4);
  take(c->joins, CACHE_JOINS * 4);
  take(c->stash, S * KV * 2 * CACHE_BLOCK * dh * e);
  take(c->status, 4);
  return (off + ALIGN - 1) / ALIGN * ALIGN;
}

int check_ready(const tppsd_cache *c) {
  if (!c) return fail(TPPSD_E_ARG, "null cache");
  if (!c->ready) return fail(TPPSD_E_ORDER, "call tppsd_cache_reset first");
  return TPPSD_OK;
}

int check_planned(const tppsd_cache *c, int layer) {
  if (int rc = check_ready(c)) return rc;
  if (!c->B) return fail(TPPSD_E_ORDER, "call tppsd_cache_begin first");
  if (layer < 0 || layer >= c->d.L) return fail(TPPSD_E_ARG, "layer %d outside 0..%d", layer, c->d.L - 1);
  return TPPSD_OK;
}

int check_pairs(const tppsd_cache *c, int n, const void *a, const void *b) {
  if (!a || !b) return fail(TPPSD_E_ARG, "null sequence list");
  if (n < 1 || n > c->d.S) return fail(TPPSD_E_ARG, "%d sequences outside 1..%d", n, c->d.S);
  return TPPSD_OK;
}

int check_rows(const CacheDev &d, const void *p, int64_t ld, int heads, const char *what) {
  if (!p) return fail(TPPSD_E_ARG, "null %s", what);
  const int e = d.bf16 ? 2 : 4;
  if ((uintptr_t)p % 16 || ld * e % 16) return fail(TPPSD_E_ARG, "%s and its row stride must be multiples of 16 bytes", what);
  if (ld < (int64_t)heads * d.dh) return fail(TPPSD_E_ARG, "row stride of %s is shorter than its heads", what);
  return TPPSD_OK;
}

CacheRows packed_rows(const tppsd_cache *c, const tppsd_cache_rows *r) {
  CacheRows x{};
  x.k = r->k;
  x.v = r->v;
  x.k_sp = r->ldk;
  x.v_sp = r->ldv;
  x.k_sb = r->ldk * c->P;
  x.v_sb = r->ldv * c->P;
  x.k_sh = x.v_sh = c->d.dh;
  return x;
}

}  // namespace

namespace tppsd {
size_t cache_view(CacheDev *c, char *d_ws) { return (size_t)view(c, d_ws, nullptr); }
}  // namespace tppsd

extern "C" {

int tppsd_cache_bytes(const tppsd_cache_cfg *cfg, size_t *bytes) {
  CacheDev d{};
  if (int rc = check_cfg(cfg, &d)) return rc;
  if (!bytes) return fail(TPPSD_E_ARG, "null output pointer");
  *bytes = (size_t)view(&d, nullptr, nullptr);
  return TPPSD_OK;
}

int tppsd_cache_entry(const tppsd_cache_cfg *cfg, int index, const char **name, size_t *offset) {
  CacheDev d{};
  if (int rc = check_cfg(cfg, &d)) return rc;
  if (index < 0 || index >= N_ENTRIES) return fail(TPPSD_E_ARG, "cache entry %d out of range", index);
  Entry e[N_ENTRIES];
  view(&d, nullptr, e);
  if (name) *name = e[index].name;
  if (offset) *offset = e[index].off;
  return TPPSD_OK;
}

int tppsd_cache_create(const tppsd_cache_cfg *cfg, void *d_workspace, size_t ws_bytes, tppsd_cache **out) {
  CacheDev d{};
  if (int rc = check_cfg(cfg, &d)) return rc;
  if (!d_workspace || !out) return fail(TPPSD_E_ARG, "null workspace or output pointer");
  if ((uintptr_t)d_workspace % ALIGN) return fail(TPPSD_E_WORKSPACE, "workspace must be 256-byte aligned");
  const size_t need = (size_t)view(&d, nullptr, nullptr);
  if (ws_bytes < need) return fail(TPPSD_E_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, need);
  tppsd_cache *c = new (std::nothrow) tppsd_cache();
  if (!c) return fail(TPPSD_E_ARG, "no host memory");
  c->d = d;
  view(&c->d, (char *)d_workspace, nullptr);
  *out = c;
  return TPPSD_OK;
}

void tppsd_cache_destroy(tppsd_cache *c) { delete c; }

int tppsd_cache_reset(tppsd_cache *c, hipStream_t st) {
  if (!c) return fail(TPPSD_E_ARG, "null cache");
  launch_cache_reset(c->d, st);
  c->ready = true;
  c->B = 0;
  return hip_check("tppsd_cache_reset");
}

int tppsd_cache_begin(tppsd_cache *c, int B, int n_new, const int32_t *d_seqs, const int32_t *d_counts,
                      hipStream_t st) {
  if (int rc = check_ready(c)) return rc;
  if (B < 1 || B > c->d.S) return fail(TPPSD_E_ARG, "batch %d outside 1..%d", B, c->d.S);
  if (n_new < 1 || n_new > c->d.max_events)
    return fail(TPPSD_E_ARG, "n_new %d outside 1..%d", n_new, c->d.max_events);
  if (n_new / CACHE_BLOCK > 65000)
    return fail(TPPSD_E_ARG, "n_new %d too large", n_new);
  CacheBegin b{};
  b.B = B;
  b.P = n_new;
  b.seqs = d_seqs;
  b.counts = d_counts;
  b.split_target = cache_split_target(c->d, B, n_new);
  launch_cache_begin(c->d, b, st);
  c->B = B;
  c->P = n_new;
  return hip_check("tppsd_cache_begin");
}

int tppsd_cache_append(tppsd_cache *c, int layer, const tppsd_cache_rows *rows, hipStream_t st) {
  if (int rc = check_planned(c, layer)) return rc;
  if (!rows) return fail(TPPSD_E_ARG, "null rows");
  if (int rc = check_rows(c->d, rows->k, rows->ldk, c->d.KV, "k")) return rc;
  if (int rc = check_rows(c->d, rows->v, rows->ldv, c->d.KV, "v")) return rc;
  launch_cache_append(c->d, layer, c->B, c->P, packed_rows(c, rows), st);
  return hip_check("tppsd_cache_append");
}

int tppsd_cache_attend(tppsd_cache *c, int layer, const tppsd_cache_rows *rows, float scale, int sink,
                       hipStream_t st) {
  if (int rc = check_planned(c, layer)) return rc;
  if (!rows) return fail(TPPSD_E_ARG, "null rows");
  if (int rc = check_rows(c->d, rows->k, rows->ldk, c->d.KV, "k")) return rc;
  if (int rc = check_rows(c->d, rows->v, rows->ldv, c->d.KV, "v")) return rc;
  if (int rc = check_rows(c->d, rows->q, rows->ldq, c->d.H, "q")) return rc;
  if (int rc = check_rows(c->d, rows->o, rows->ldo, c->d.H, "o")) return rc;
  if (!(scale > 0.f) || !std::isfinite(scale * 1.4426950408889634f))   // (scores go to base 2)
    return fail(TPPSD_E_ARG, "scale and scale log2(e) must be positive and finite");
  if (cache_groups(c->d, c->P) > 65535)   // (a dimension of the grid)
    return fail(TPPSD_E_ARG, "%d positions of %d heads a key/value head are too many for one call", c->P, c->d.H / c->d.KV);
  CacheAttend a{};
  a.q = rows->q;
  a.o = rows->o;
  a.ldq = rows->ldq;
  a.ldo = rows->ldo;
  a.kv = packed_rows(c, rows);
  a.layer = layer;
  a.B = c->B;
  a.P = c->P;
  a.scale = scale;
  a.sink = sink != 0;
  launch_cache_attend(c->d, a, st);
  return hip_check("tppsd_cache_attend");
}

int tppsd_cache_commit(tppsd_cache *c, const int32_t *d_accept, hipStream_t st) {
  if (int rc = check_planned(c, 0)) return rc;
  launch_cache_commit(c->d, c->B, d_accept, st);
  c->B = 0;
  return hip_check("tppsd_cache_commit");
}

int tppsd_cache_truncate(tppsd_cache *c, int n, const int32_t *d_seqs, const int32_t *d_lens, hipStream_t st) {
  if (int rc = check_ready(c)) return rc;
  if (!d_seqs) return fail(TPPSD_E_ARG, "null sequence list");
  if (n < 1 || n > MAX_SEQS) return fail(TPPSD_E_ARG, "%d sequences outside 1..%d", n, MAX_SEQS);
  launch_cache_truncate(c->d, n, d_seqs, d_lens, st);
  c->B = 0;
  return hip_check("tppsd_cache_truncate");
}

int tppsd_cache_fork(tppsd_cache *c, int n, const int32_t *d_src, const int32_t *d_dst, hipStream_t st) {
  if (int rc = check_ready(c)) return rc;
  if (int rc = check_pairs(c, n, d_src, d_dst)) return rc;
  launch_cache_fork(c->d, n, d_src, d_dst, st);
  c->B = 0;
  return hip_check("tppsd_cache_fork");
}

int tppsd_cache_copy(tppsd_cache *to, tppsd_cache *from, int n, const int32_t *d_src, const int32_t *d_dst,
                     hipStream_t st) {
  if (int rc = check_ready(to)) return rc;
  if (int rc = check_ready(from)) return rc;
  if (to == from) return fail(TPPSD_E_ARG, "tppsd_cache_copy needs two caches (tppsd_cache_fork continues sequences of one)");
  if (to->d.L != from->d.L || to->d.KV != from->d.KV || to->d.dh != from->d.dh || to->d.bf16 != from->d.bf16)
    return fail(TPPSD_E_CONFIG, "caches differ in layers, key/value heads, d_head or precision");
  if (int rc = check_pairs(to, n, d_src, d_dst)) return rc;
  if ((long long)n * (1 + to->d.L) > (1LL << 30)) return fail(TPPSD_E_ARG, "too many sequences");
  launch_cache_copy(to->d, from->d, n, d_src, d_dst, st);
  to->B = 0;
  return hip_check("tppsd_cache_copy");
}

int tppsd_cache_read(tppsd_cache *c, int layer, int n, const int32_t *d_seqs, const int32_t *d_first, int count,
                     void *d_k, void *d_v, hipStream_t st) {
  if (int rc = check_ready(c)) return rc;
  if (layer < 0 || layer >= c->d.L) return fail(TPPSD_E_ARG, "layer %d outside 0..%d", layer, c->d.L - 1);
  if (n < 1 || (!d_seqs && n > c->d.S)) return fail(TPPSD_E_ARG, "%d sequences", n);
  if (count < 1 || count / CACHE_BLOCK > 65000) return fail(TPPSD_E_ARG, "count %d outside its range", count);
  if (!d_k || !d_v) return fail(TPPSD_E_ARG, "null output");
  if ((uintptr_t)d_k % 16 || (uintptr_t)d_v % 16) return fail(TPPSD_E_ARG, "outputs must be 16-byte aligned");
  launch_cache_read(c->d, layer, n, d_seqs, d_first, count, d_k, d_v, st);
  return hip_check("tppsd_cache_read");
}

int tppsd_cache_status(tppsd_cache *c, hipStream_t st, uint32_t *bits) {
  if (int rc = check_ready(c)) return rc;
  uint32_t b = 0;
  if (hipMemcpyAsync(&b, c->d.status, 4, hipMemcpyDeviceToHost, st) != hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return hip_check("tppsd_cache_status");
  if (bits) *bits = b;
  return TPPSD_OK;
}

}  // extern "C"
