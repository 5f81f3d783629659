// What the kernels for packed prompts, shared documents and copies of sequences take, and
// the arithmetic that their host and device sides share.
#pragma once

#include "launch.h"

namespace infllm {

// Packed prompts: whole causal self-attention of sequences that lie one after another.
// Row (token t, head h) of a tensor starts at t * its token stride + h * its head
// stride elements.  The sequences are listed by falling length, empty ones left out.
// A row tile is a run of rows (query-major, the group's heads packed) of one sequence;
// tiles are numbered from the last row tile of the longest sequence down, level by
// level: the tiles that many sequences have at one level lie side by side, so that
// tile numbers fall by the keys a tile sees.  first[i] is the number of the first tile
// of the levels that exactly the i + 1 longest sequences reach.
//
// The row tiles that see the most keys are split along the keys: part p takes the key
// tiles [p * part_tiles, (p + 1) * part_tiles), and a tile has as many parts as its level
// can see.  The row tiles with a part p are the first ones, those whose part p is a full
// one of part_tiles the first full[p] of them.  So that the workgroups which start last
// are short ones, the items of the launch are numbered full parts first, by part, then the
// rest from the last part down to part 0 (row tiles that are whole).  Where a tile has
// several parts (the first split_tiles) they leave partial rows (see common.h), rows_wg of
// them per item and kv head, and a merge.
constexpr int kMaxPrompts = 256;  // of one launch
constexpr int kMaxPromptParts = 16;
struct PromptArgs {
  int n_seqs, n_q_heads, n_kv_heads, head_dim;
  int64_t q_tok, q_head, kv_tok, kv_head, out_tok, out_head;
  int64_t lse_stride;  // tokens of the whole call
  float sm_scale;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;  // nullable, [n_q_heads][lse_stride]
  int row_waves;  // waves of a workgroup that hold query rows, 32 each
  int n_tiles;
  int parts;       // most parts of a row tile
  int part_tiles;  // key tiles of a part
  int split_tiles;
  int items;
  int full[kMaxPromptParts];
  int full_begin[kMaxPromptParts + 1];  // first item of the full parts p; of the rest
  int rest_begin[kMaxPromptParts + 1];  // first item of the rest of part parts - 1 - x; all items
  void* part_o;
  float* part_lse;
  int32_t* part_exp;
  FastDiv d_group, d_kv;
  bool bf16;
  int32_t start[kMaxPrompts];
  int32_t len[kMaxPrompts];
  int32_t first[kMaxPrompts];
};
struct PromptTile {
  int start, len;  // the sequence
  int tile;        // row tile of it
};
// The part and row tile of an item, and back.
__host__ __device__ inline void prompt_item(const PromptArgs& a, int item, int& p, int& t) {
  const int* begin = item < a.full_begin[a.parts] ? a.full_begin : a.rest_begin;
  int x = 0;
  for (int i = 1; i < a.parts; ++i) x += item >= begin[i] ? 1 : 0;
  p = begin == a.full_begin ? x : a.parts - 1 - x;
  t = item - begin[x] + (begin == a.full_begin ? 0 : a.full[p]);
}
__host__ __device__ inline int prompt_item_of(const PromptArgs& a, int p, int t) {
  return t < a.full[p] ? a.full_begin[p] + t : a.rest_begin[a.parts - 1 - p] + t - a.full[p];
}
// Row tiles with a part p.
__host__ __device__ inline int prompt_part_count(const PromptArgs& a, int p) {
  return a.full[p] + a.rest_begin[a.parts - p] - a.rest_begin[a.parts - 1 - p];
}
// Rows that the items with partial rows take: those before the row tiles that are whole.
__host__ inline int64_t prompt_partial_rows(const PromptArgs& a) {
  return a.parts > 1 ? (int64_t)a.rest_begin[a.parts - 1] * a.n_kv_heads * 32 * a.row_waves : 0;
}
// Row tile number t (uniform over the wave).  Every lane reads its sequences' entries at
// once, so that one trip to memory serves the search and what it leads to.
__device__ __forceinline__ PromptTile prompt_tile(const PromptArgs& a, int t, int rows_log2) {
  constexpr int CH = kMaxPrompts / kWave;
  const int lane = threadIdx.x & 63;
  int first[CH], len[CH], start[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    if (j * kWave >= a.n_seqs) break;
    first[j] = a.first[j * kWave + lane];
    len[j] = a.len[j * kWave + lane];
    start[j] = a.start[j * kWave + lane];
  }
  int i = 0;  // sequences with tiles on the level of t
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    if (j * kWave >= a.n_seqs) break;
    i += __popcll(__ballot(j * kWave + lane < a.n_seqs && first[j] <= t));
  }
  i = __builtin_amdgcn_readfirstlane(i);
  auto pick = [&](const int (&x)[CH], int s) {
    int v = __builtin_amdgcn_readlane(x[0], s & 63);
#pragma unroll
    for (int j = 1; j < CH; ++j)
      if (s >> 6 == j) v = __builtin_amdgcn_readlane(x[j], s & 63);
    return v;
  };
  const int u = t - pick(first, i - 1), down = u / i, s = u - down * i;
  const int rows = pick(len, i - 1) * (int)a.d_group.d;
  return PromptTile{pick(start, s), pick(len, s), ((rows - 1) >> rows_log2) - down};
}
hipError_t launch_prompt(const PromptArgs& a, hipStream_t s);
hipError_t launch_prompt_merge(const PromptArgs& a, hipStream_t s);

// Attention of continuations over a document they share.  Three regions of keys, each
// with parts of its own:
//   shared: I and L of the document, met by the rows of all continuations together;
//   units : the looked-up units of one continuation (document store);
//   own   : the tokens of one continuation, X at their end (its own store, causal).
// A few current tokens (x_k given) are not in the own region: the merge meets them, and
// writes them to the own stores.
constexpr int kPrefixMergeTokens = 8;
struct PrefixArgs {
  int batch, n_q_heads, n_kv_heads, head_dim, n_q;
  int64_t prefix_capacity, own_capacity, q_head_stride, out_head_stride;
  float sm_scale;
  const void* q;
  const void* prefix_k;
  const void* prefix_v;
  const void* own_k;
  const void* own_v;
  const int32_t* idx;  // [batch][n_kv_heads][idx_stride]
  int n_init, n_units, n_sel, block_size, unit_base, idx_stride;
  int64_t local_begin, prefix_len;
  const void* x_k;  // [batch][n_kv_heads] heads of n_q rows with x_head_stride, or null
  const void* x_v;
  int64_t x_head_stride;
  int parts_s, parts_u, parts_o;  // of the regions; parts = their sum
  int parts;
  bool direct;                    // one part, whose rows are the output's
  int row_waves;                  // waves of a workgroup that hold query rows (matrix-core kernel)
  int tiles_s, tiles_p;           // row tiles of the shared region and of one continuation
  FastDiv d_group, d_block, d_kv, d_q, d_tiles_s, d_tiles_p, d_parts_u, d_parts_o;
  void* out;
  float* lse;
  void* part_o;
  float* part_lse;
  int32_t* part_exp;
  bool bf16;
  int64_t own_len[kMaxVarBatch];
};
// Where a workgroup of the prefix attention works.
struct PrefixWork {
  int region;  // 0 shared, 1 units, 2 own
  int g, b;    // b: the continuation (0 in the shared region)
  int tile;    // row tile
  int part;    // of the region's parts
};
__device__ __forceinline__ PrefixWork prefix_work(const PrefixArgs& a, int id) {
  PrefixWork w;
  int r = div_by(id, a.d_kv);
  w.g = id - r * (int)a.d_kv.d;
  const int n_shared = a.tiles_s * a.parts_s, n_units = a.batch * a.tiles_p * a.parts_u;
  if (r < n_shared) {
    w.region = 0;
    w.b = 0;
    w.part = div_by(r, a.d_tiles_s);
    w.tile = r - w.part * a.tiles_s;
    return w;
  }
  r -= n_shared;
  w.region = r < n_units ? 1 : 2;
  r -= w.region == 1 ? 0 : n_units;
  const int c = div_by(r, a.d_tiles_p);
  w.tile = r - c * a.tiles_p;
  w.b = w.region == 1 ? div_by(c, a.d_parts_u) : div_by(c, a.d_parts_o);
  w.part = c - w.b * (w.region == 1 ? a.parts_u : a.parts_o);
  return w;
}
// The keys of a region as a step's key axis; n_q = 0 where every row sees all of them.
__device__ __forceinline__ StepGeom prefix_geom(const PrefixArgs& a, const PrefixWork& w) {
  StepGeom g;
  g.n_units = a.n_units;
  g.unit_base = a.unit_base;
  g.idx_stride = a.idx_stride;
  g.block_size = w.region == 1 ? a.block_size : 8;
  g.n_init = w.region == 0 ? a.n_init : 0;
  g.n_sel = w.region == 1 ? a.n_sel : 0;
  g.local_begin = w.region == 0 ? a.local_begin : 0;
  g.n_q = w.region == 2 && a.x_k == nullptr ? a.n_q : 0;
  g.past_len = w.region == 2 ? a.own_len[w.b] : a.prefix_len;
  g.n_virtual = w.region == 1   ? a.n_sel * a.block_size
                : w.region == 0 ? (int32_t)(a.n_init + (a.prefix_len - a.local_begin))
                                : (int32_t)g.past_len + g.n_q;
  return g;
}
// First part of a region among all parts, and the workgroups of the launch.
__host__ __device__ inline int prefix_first_part(const PrefixArgs& a, int region) {
  return region == 0 ? 0 : a.parts_s + (region == 1 ? 0 : a.parts_u);
}
__host__ inline int prefix_workgroups(const PrefixArgs& a) {
  return a.n_kv_heads * (a.tiles_s * a.parts_s + a.batch * a.tiles_p * (a.parts_u + a.parts_o));
}
hipError_t launch_prefix(const PrefixArgs& a, hipStream_t s);
hipError_t launch_prefix_merge(const PrefixArgs& a, hipStream_t s);

// Copies of whole sequences between memories: the pairs are sorted by source, so that a
// source's bytes are read once for all its copies.
struct SeqCopyArgs {
  int n_pairs, n_sources, n_kv_heads, row_bytes;  // row_bytes: of a K or V row
  int64_t src_capacity, dst_capacity;
  int src_units, dst_units, src_ring, dst_ring;
  int repr_bytes;  // of a unit's representatives (0: none are kept)
  int cells;       // 16-byte cells of a unit's key sum (head_dim / 4)
  int ring_rows;   // rpart rows (head_dim / 8), 0 without rings
  const char* src_k;
  const char* src_v;
  const char* src_rot;
  const char* src_repr;
  const char* src_ksum;
  const char* src_qprefix;
  const char* src_rpart;
  char* dst_k;
  char* dst_v;
  char* dst_rot;
  char* dst_repr;
  char* dst_ksum;
  char* dst_qprefix;
  char* dst_rpart;
  int32_t pair_begin[kMaxVarBatch + 1];  // of a source
  int32_t block_begin[kMaxVarBatch + 1];
  int32_t src_seq[kMaxVarBatch];         // of a source
  int32_t dst_seq[kMaxVarBatch];         // of a pair
  int32_t built[kMaxVarBatch];
  int64_t len[kMaxVarBatch];
};
hipError_t launch_copy_sequences(const SeqCopyArgs& a, hipStream_t s);

struct PrefixScoreArgs {
  int batch, n_q_heads, n_kv_heads, head_dim, n_q, n_units, max_units;
  int64_t q_head_stride;
  const void* q;
  const float* unit_ksum;
  float* scores;      // [batch][n_kv_heads][n_units]
  float* qbar_parts;  // workspace: score_qbar_parts per (sequence, kv head)
  bool bf16;
};
hipError_t launch_prefix_score(const PrefixScoreArgs& a, hipStream_t s);

}  // namespace infllm
