// 8-bit paged key/value cache: device view, geometry and launchers
// (tppsd_cache.hip: bookkeeping, append, read, copies; tppsd_cache_attn.hip:
// attention). Not part of the public ABI.
//
// A page holds CACHE_BLOCK positions of every layer and key/value head as
// e4m3 codes, keys and values each under a power-of-two scale per (layer,
// head). A sequence owns floor(length / 64) whole pages; the rows of the block
// that is still open are kept as they came, in a ring of two blocks (slot =
// position mod 128), so that every element is rounded to 8 bits once, under
// the maximum of its whole block, whatever the calls that brought its rows.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tppsd {

constexpr int CACHE_BLOCK = 64;   // positions of a page (TPPSD_CACHE_BLOCK)
constexpr int CACHE_RING = 128;   // tail rows: two blocks
// Least exponent of a scale: 2^-100 keeps every code's value, and its product
// with the reciprocal scale, a normal fp32 (and bf16) number
constexpr int CACHE_E_MIN = -100;
// Waves of the attention that make a full chip (two per SIMD), the fewest pages
// of a piece of a row, and the most (row, head, group) triples of a batch whose
// rows are split
constexpr int CACHE_SPLIT_WAVES = 2048, CACHE_MIN_PIECE = 8, CACHE_JOINS = 4096;

// A work item of the attention: pages lo .. hi - 1 of a row of the batch. Rows
// in several pieces keep each piece's partial state in a slot.
struct CacheItem {
  int row, seq, start, count;   // row of the batch, its sequence, first new position and how many
  int lo, hi;
  int piece, pieces;            // this one of so many
  int slot0;                    // slot of the row's first piece
  int pad[3];
};

struct CacheDev {
  int L, H, KV, dh, bf16;
  int S, NP, n_pages, max_events;   // sequences, pages of a table row, pages of the pool
  uint8_t *pages;     // [L][n_pages][KV][2][64 dh] codes in fragment order (page_at)
  float *scales;      // [L][n_pages][KV][2]
  char *tails;        // [L][S][KV][2][128][dh] rows of the last blocks, in the model's type
  int32_t *table;     // [S][NP] pages of each sequence, -1 past those it holds
  int32_t *lens;      // [S] committed positions
  int32_t *refs;      // [n_pages] sequences that hold the page
  int32_t *held;      // [S] pages held (those of uncommitted blocks too)
  int32_t *low;       // [S] first block whose rows the ring holds
  int32_t *pend;      // [S] positions that the plan brings and that are not committed
  int32_t *planned;   // [S] twice the number of the last plan that brings the sequence any; 1: behind an open
                      // block that is not in the ring any more (which a commit settles)
  int32_t *came;      // [L][S] number of the last plan whose rows the layer has
  uint32_t *freeb;    // [ceil(n_pages / 32)] bit set: page is free
  int32_t *owner;     // [S] scratch: which row of a call names the sequence
  int32_t *role;      // [S] scratch of forks
  int32_t *list;      // [n_pages] scratch: pages in the order of a scan
  int32_t *map;       // [n_pages] scratch of copies: destination page
  uint32_t *mark;     // [ceil(n_pages / 32)] scratch of copies: pages to copy
  int32_t *counts;    // [8] items of the plan, pages to copy, a word of freeb before which no page is free,
                      // number of the plan (calls that drop a plan take one too)
  // plan of the call in progress, one row per sequence of the batch
  int32_t *p_seq, *p_start, *p_count;   // [S]
  CacheItem *items;
  int max_items;
  float *part;        // partial states of split rows
  int32_t *joins;     // [CACHE_JOINS] splits that have arrived; zero between calls
  char *stash;        // [S][KV][2][64][dh] rows of a long chunk's first block from before it
  uint32_t *status;
};

__host__ __device__ inline size_t page_tile(const CacheDev &c) { return (size_t)2 * CACHE_BLOCK * c.dh; }

// rows of the caller: element (row i of the batch, position p, head h, column j)
// at base + i sb + p sp + h sh + j
struct CacheRows {
  const void *k, *v;
  int64_t k_sb, k_sp, k_sh, v_sb, v_sp, v_sh;
  int v_blocked;      // values in 8-position blocks (bf16 slabs): + (p / 8) 8 dh + j 8 + p mod 8
};

// start_in: positions start_in[i] + start_off replace the committed lengths
// (and become them); done: rows to leave out
struct CacheBegin {
  int B, P;
  const int32_t *seqs, *counts, *start_in, *done;
  int start_off;
  int split_target;   // full chip: items of the batch, 0: one per row
};

struct CacheAttend {
  const void *q;
  void *o;
  int64_t ldq, ldo;   // elements between the positions of a row of the batch
  CacheRows kv;
  int layer, B, P;
  float scale;
  int sink;
  int zero;           // rows that are left out are written as zeros
  // set by the launcher:
  int whole;          // rows are not split: no work items
  int nt_pages;       // pages of a row from which they are read with the non-temporal hint
};

void launch_cache_reset(const CacheDev &c, hipStream_t st);
void launch_cache_begin(const CacheDev &c, const CacheBegin &b, hipStream_t st);
// (launch_cache_attend appends as well)
void launch_cache_append(const CacheDev &c, int layer, int B, int P, const CacheRows &r, hipStream_t st);
void launch_cache_commit(const CacheDev &c, int B, const int32_t *accept, hipStream_t st);
void launch_cache_truncate(const CacheDev &c, int n, const int32_t *seqs, const int32_t *lens, hipStream_t st);
void launch_cache_fork(const CacheDev &c, int n, const int32_t *src, const int32_t *dst, hipStream_t st);
void launch_cache_copy(const CacheDev &to, const CacheDev &from, int n, const int32_t *src, const int32_t *dst,
                       hipStream_t st);
void launch_cache_read(const CacheDev &c, int layer, int n, const int32_t *seqs, const int32_t *first, int count,
                       void *k, void *v, hipStream_t st);

// items that make a full chip for a batch of B rows of P positions, 0 where
// rows are not split
int cache_split_target(const CacheDev &c, int B, int P);
// groups of query rows of a call of P positions (one grid dimension)
int cache_groups(const CacheDev &c, int P);
int cache_max_items(int S, int KV);
size_t cache_part_floats(const CacheDev &c);
void launch_cache_attend(const CacheDev &c, const CacheAttend &a, hipStream_t st, hipEvent_t ev0 = nullptr,
                         hipEvent_t ev1 = nullptr);

// device view over a workspace (d_ws NULL: the sizes alone); returns its bytes
size_t cache_view(CacheDev *c, char *d_ws);

}  // namespace tppsd
