// What the kernels on paged caches take, and the arithmetic that their host and device
// sides share.
#pragma once

#include "launch.h"

namespace infllm {

constexpr int kMaxPaged = 256;  // sequences of one launch

// The sequences of a launch, packed one after another.
struct PagedSeqs {
  int n_seqs;
  int n_pages, page_size;
  FastDiv d_page;
  const int32_t* table;  // row of the launch's first sequence
  int64_t table_stride;
  int32_t start[kMaxPaged + 1];  // first new token, in the call's order; the end
  int32_t past[kMaxPaged];       // tokens before it
};

// The sequence of new token t (uniform over the wave): the last one that starts at or
// before it.  Every lane reads its sequences' entries at once.
__device__ __forceinline__ int paged_seq_of(const PagedSeqs& a, int t) {
  constexpr int CH = kMaxPaged / kWave;
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    if (j * kWave >= a.n_seqs) break;
    const int i = j * kWave + lane;
    n += __popcll(__ballot(i < a.n_seqs && a.start[i] <= t));
  }
  return __builtin_amdgcn_readfirstlane(n) - 1;
}

// Norms and rotation.  A token has n_q query rows, n_k key rows and n_v value rows, in this
// order; a wave has `rows_wave` of them.
struct RotateArgs {
  int first_token, n_tokens;  // of this launch
  int n_q, n_k, n_v;
  int rows_wave;
  FastDiv d_split;  // waves of a token
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  void* k_out;
  void* v_out;
  int64_t q_tok, q_head, kv_tok, kv_head, qo_tok, qo_head, ko_tok, ko_head;
  int64_t page_stride;  // (with pages, ko_tok and ko_head are those within a page)
  const int64_t* positions;
  int64_t first_position;
  int rotary_dim, interleaved, norm;
  float magnitude, eps;
  const void* q_weight;
  const void* k_weight;
  int head_dim;
  bool bf16;
  double rev[kMaxPairs];  // revolutions per position of pair i
};
// And the append to pages.  (Apart, for the 2 KB of sequences cost a launch 0.4 us on the host.)
struct AppendPagesArgs : RotateArgs {
  PagedSeqs seqs;
};
hipError_t launch_rotate(const RotateArgs& a, hipStream_t s);
hipError_t launch_rotate(const AppendPagesArgs& a, hipStream_t s);

// Attention over pages.  A row tile is a run of rows (query-major, the group's heads
// packed) of one sequence.  The key tiles that a row tile sees, in order, are those of the
// initial tokens that lie before the window, then [first of the window, diagonal]; they
// are cut into parts.  An item is a part of a row tile (the sequences in the order of the
// list, of a sequence the last row tile first, of a row tile its parts in order), a
// workgroup an item and a kv head.  Row tiles with several parts leave partial rows (see
// common.h), item_rows of them per item and kv head, and a merge.
// A sequence's row tiles are cut into parts of one length, the sequences listed by falling
// length of their parts, those without new tokens left out.
constexpr int kMaxAttend = 192;  // sequences of one launch
struct PagedArgs {
  int n_q_heads, n_kv_heads, head_dim;
  bool bf16;
  float sm_scale, softcap;
  int window, n_init;
  const float* slopes;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  int64_t q_tok, q_head, out_tok, out_head, lse_stride;
  int64_t head_stride;
  uint32_t page16, token16;  // strides of pages and their tokens in pieces of 16 bytes (modulo 2^32)
  int rows_log2;             // rows of a row tile
  int tile_queries;          // most queries with rows in one row tile
  int key_tile;              // keys of a tile
  int items, item_rows;
  FastDiv d_group, d_kv;
  void* part_o;
  float* part_lse;
  int32_t* part_exp;
  int n_pages, page_size;
  FastDiv d_page;
  const int32_t* table;
  int64_t table_stride;
  int n_seqs;
  int32_t first[kMaxAttend];       // first item of a sequence
  int32_t start[kMaxAttend];       // its first new token
  int32_t len[kMaxAttend];
  int32_t past[kMaxAttend];        // tokens before it
  uint8_t parts[kMaxAttend];       // most parts of its row tiles, less 1
  uint8_t table_row[kMaxAttend];   // its row of the page table
};
static_assert(sizeof(PagedArgs) <= 4096, "arguments of a launch");

// Keys of a row tile whose first and last queries are i0 and i1 of a sequence with `past`
// tokens before: tiles [0, sink) and [low, low + n - sink).
struct PagedRange {
  int sink, low, n;
};
__host__ __device__ inline PagedRange paged_range(const PagedArgs& a, int past, int i0, int i1) {
  PagedRange r;
  const int end = (past + i1) / a.key_tile + 1;
  r.low = a.window > 0 ? (past + i0 >= a.window ? past + i0 - a.window + 1 : 0) / a.key_tile : 0;
  const int init = a.n_init < past + i1 + 1 ? a.n_init : past + i1 + 1;
  r.sink = (init + a.key_tile - 1) / a.key_tile;
  if (r.sink > r.low) r.sink = r.low;
  r.n = r.sink + end - r.low;
  return r;
}
// Most tiles that a row tile of a sequence sees (its items are as many parts for each).
__host__ __device__ inline int paged_most_tiles(const PagedArgs& a, int past, int len) {
  const int total = past + len, whole = (total - 1) / a.key_tile + 1;
  if (a.window == 0) return whole;
  const int queries = a.tile_queries < len ? a.tile_queries : len;
  const int64_t keys = (int64_t)(a.window < total ? a.window : total) + queries - 1;
  const int init = a.n_init < total ? a.n_init : total;
  const int64_t most = (init + a.key_tile - 1) / a.key_tile + (keys - 1) / a.key_tile + 2;
  return most < whole ? (int)most : whole;
}
__host__ __device__ inline int paged_row_tiles(const PagedArgs& a, int group, int len) {
  return (int)(((int64_t)len * group + (1 << a.rows_log2) - 1) >> a.rows_log2);
}

// Where a workgroup of item `item` works.
struct PagedWork {
  int start, len, past;  // the sequence
  int table_row;
  int rt, part;
  int part_tiles;  // key tiles of a part
};
__device__ __forceinline__ PagedWork paged_work(const PagedArgs& a, int item) {
  PagedWork w;
  int first0, m;
  if (a.n_seqs == 1) {  // (no trip to memory beside the other arguments')
    first0 = 0;
    w.start = a.start[0];
    w.len = a.len[0];
    w.past = a.past[0];
    m = a.parts[0] | a.table_row[0] << 8;
  } else {
    constexpr int CH = kMaxAttend / kWave;
    static_assert(CH * kWave == kMaxAttend, "whole waves");
    const int lane = threadIdx.x & 63;
    int first[CH], start[CH], len[CH], past[CH], more[CH], n = 0;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (j * kWave >= a.n_seqs) break;
      const int i = j * kWave + lane;
      first[j] = a.first[i];
      start[j] = a.start[i];
      len[j] = a.len[i];
      past[j] = a.past[i];
      more[j] = a.parts[i] | a.table_row[i] << 8;
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      if (j * kWave >= a.n_seqs) break;
      n += __popcll(__ballot(j * kWave + lane < a.n_seqs && first[j] <= item));
    }
    const int s = __builtin_amdgcn_readfirstlane(n) - 1;
    auto pick = [&](const int (&x)[CH]) {
      int v = __builtin_amdgcn_readlane(x[0], s & 63);
#pragma unroll
      for (int j = 1; j < CH; ++j)
        if (s >> 6 == j) v = __builtin_amdgcn_readlane(x[j], s & 63);
      return v;
    };
    w.start = pick(start);
    w.len = pick(len);
    w.past = pick(past);
    m = pick(more);
    first0 = pick(first);
  }
  w.table_row = m >> 8;
  const int parts = (m & 255) + 1;
  const int tiles = paged_row_tiles(a, (int)a.d_group.d, w.len), u = item - first0;
  const int down = parts == 1 ? u : tiles == 1 ? 0 : u / parts;
  w.part = u - down * parts;
  w.rt = tiles - 1 - down;
  const int most = paged_most_tiles(a, w.past, w.len);
  w.part_tiles = parts == 1 ? most : (most + parts - 1) / parts;
  return w;
}
hipError_t launch_paged(const PagedArgs& a, hipStream_t s);
hipError_t launch_paged_merge(const PagedArgs& a, hipStream_t s);

}  // namespace infllm
