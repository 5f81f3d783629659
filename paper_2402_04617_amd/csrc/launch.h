// Host-side launchers of the gfx950 kernels (internal to the library).  The C ABI
// in abi.cpp validates every argument, then calls these; each returns the
// hipError_t of its launch(es).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.h"

namespace infllm {

// Variable-length batches: sequence b has its own past length past[b] (all
// sequences append the same number of tokens).  Kernels derive each sequence's
// step geometry from it with the host's partition arithmetic.
constexpr int kMaxVarBatch = 64;
struct VarLen {
  int32_t on;
  int64_t past[kMaxVarBatch];
};

// Memory parts of a step split by the positional remap: the memory keys' share
// of `parts`, at least one part per non-empty region.
__host__ __device__ inline int split_parts_mem(int parts, int64_t mem_len, int64_t n_virtual) {
  if (mem_len <= 0 || parts < 2) return 0;
  int pm = (int)((parts * mem_len + n_virtual / 2) / n_virtual);
  return pm < 1 ? 1 : (pm > parts - 1 ? parts - 1 : pm);
}

// Step geometry of a sequence with past length `past` (the partition of
// Section 3.1): `base` supplies the shared fields (l_bs, l_I, k_m, l_X).
__host__ __device__ inline StepGeom seq_geom(const StepGeom& base, int n_local, int64_t past) {
  StepGeom g = base;
  g.n_init = (int32_t)(past < base.unit_base ? past : base.unit_base);
  const int64_t evicted = past - base.unit_base - n_local;
  const int64_t nu = evicted > 0 ? evicted / base.block_size : 0;
  g.n_units = (int32_t)nu;
  g.n_sel = (int32_t)(base.idx_stride < nu ? base.idx_stride : nu);
  g.local_begin = g.n_init + nu * base.block_size;
  g.past_len = past;
  g.n_virtual = (int32_t)(g.n_init + (int64_t)g.n_sel * base.block_size + (past - g.local_begin) + base.n_q);
  return g;
}

// Width of the dimension slices whose partial representative scores the append
// stores (rpart holds D / kRpartDims float64 values per token).
constexpr int kRpartDims = 8;

struct AppendArgs {
  int batch, n_q_heads, n_kv_heads, head_dim, n_q, ring, n_init, n_local;
  int64_t past_len, capacity, q_head_stride, kv_head_stride;
  const void* q;
  const void* k_src;
  const void* v_src;
  void* k_store;
  void* v_store;
  double* qprefix;
  double* rpart;  // [B*Hkv][D/kRpartDims][ring] partial representative scores
  void* k_rot;    // positional remap: keys rotated to their own positions (same layout as k_store)
  RopeArgs rope;
  VarLen var;      // per-sequence past lengths (var.on), else past_len for all
  bool mean_repr;  // units scored by their mean key: no query ring, no representative scores
  bool bf16;
};
// Past length of sequence b of an append.
__host__ __device__ inline int64_t seq_past(const AppendArgs& a, int b) { return a.var.on ? a.var.past[b] : a.past_len; }
struct BuildArgs;
int score_qbar_parts(int G, int n_q);
// qbar: optional float32 output of the chunk's group-query sums: [batch*Hkv][D]
// (the scan total), or with the mean representation [batch*Hkv][parts][D]
// partial sums, parts = score_qbar_parts(G, n_q).
// fused_build: optional unit construction carried by the same launch (its ring
// reads must not overlap the chunk's new ring slots).
hipError_t launch_append(const AppendArgs& a, hipStream_t s, float* qbar, const BuildArgs* fused_build);

struct BuildArgs {
  int batch, n_q_heads, n_kv_heads, head_dim, n_init, n_local, block_size, n_repr;
  int first_unit, n_new, max_units, ring;
  int64_t capacity;
  const void* k_store;
  const double* rpart;
  int32_t* repr_idx;
  float* unit_ksum;
  double* repr_score;  // nullable
  bool mean_repr;      // unit_ksum = mean of the unit's l_bs keys (no representatives)
  // Variable-length batches: sequence b builds units [first[b], first[b] + count[b])
  // (var_on); otherwise every sequence builds [first_unit, first_unit + n_new).
  int32_t var_on;
  int32_t var_first[kMaxVarBatch];
  int32_t var_count[kMaxVarBatch];
  bool bf16;
};
hipError_t launch_build_units(const BuildArgs& a, hipStream_t s);

struct ScoreArgs {
  int batch, n_q_heads, n_kv_heads, head_dim, n_q, n_units, max_units;
  int64_t q_head_stride;
  const void* q;
  const float* unit_ksum;
  float* scores;
  float* qbar_parts;  // workspace
  RopeArgs rope;      // positional remap: the query sum is turned by R(l_L)
  // Variable-length batches: sequence b scores var_units[b] units, rows of
  // `scores` strided by score_stride (var_on); otherwise n_units each, stride n_units.
  int32_t var_on;
  int32_t var_units[kMaxVarBatch];
  int32_t score_stride;
  bool bf16;
};
int score_qbar_parts(int G, int n_q);
hipError_t launch_score(const ScoreArgs& a, hipStream_t s);
// Scoring when a.qbar_parts already holds the query sums as `parts` partials.
hipError_t launch_score_given_qbar(const ScoreArgs& a, int parts, hipStream_t s);

hipError_t launch_select_topk(int rows, const float* scores, int n_units, int k, int32_t* idx,
                              hipStream_t s);
// Rows of different lengths: row r holds row_n[r / rows_per_seq] scores at stride
// `stride`; n_max bounds them.
struct TopkRows {
  int32_t rows_per_seq;
  int32_t row_n[kMaxVarBatch];
};
hipError_t launch_select_topk_var(int rows, const float* scores, int stride, int n_max, const TopkRows& tr, int k,
                                  int32_t* idx, hipStream_t s);

// Waves of 32 query rows in a workgroup of the bf16 matrix-core attention kernel,
// and the workgroups that run at a time (one per compute unit).
constexpr int kMfmaWaves = 8;
constexpr int kMfmaTargetWgs = 256;
// Workgroups the bf16 decode kernel aims for (two per compute unit), and the
// fewest keys * head_dim it gives one workgroup (64 keys of 128 dims).
constexpr int kDecodeTargetWgs = 512;
constexpr int kDecodeMinWork = 64 * 128;
constexpr int kDecodeWaves = 4;
// Keys that its waves take at a time: a tile of two loads of 64 / (head_dim / 8) keys each;
// up to so many tiles of a wave are all in flight at once.
constexpr int decode_step_keys(int head_dim) { return kDecodeWaves * 2 * 64 / (head_dim / 8); }
constexpr int kDecodeShortTiles = 4;
// Work of a short context (keys * head_dim * (group + 2): the keys' bytes and the group's
// products) up to which one workgroup takes all its keys: the merge's launch costs more than
// a split saves (337 keys of 64 dims, group 2, four sequences: 11.4 us per step, split 14.1).
// Either way costs the same at 1,024 keys of 64 dims and 512 of 128 (group 1), 430 of 64
// (group 4) and about 215 of 128.
constexpr int64_t kDecodeWholeWork = 192000;
// Most selected units the decode kernel stages in LDS; longer lookups decode on
// the matrix-core kernel.
constexpr int kDecodeMaxSel = 1024;
// Longest score row the decode kernel selects from itself (one wave).
constexpr int kDecodeSelMax = 1024;
// Most units a wave selects by ranking its candidates (see topk_select.h): about
// 64 ln(64 / (64 - k)) keys of a full row are left, 89 at 48, 107 at 52 and 133 at 56, and a
// wave ranks 128.  Past it the eight waves of a workgroup share a radix select, which the
// decode kernel (four waves) leaves to a launch of its own: by the one wave alone, bit by bit,
// it takes 11 us (64 units of 217 for one sequence at 32K: 36.3 us per step).
constexpr int kWaveSelMaxK = 48;

// Score rows the matrix-core attention selects from itself: rows of at most
// kFusedSelectShort units by one wave (up to kWaveSelMaxK of them) or with two keys per
// thread of all eight, longer rows up to kFusedSelectMax with sixteen; at most
// kFusedSelectMaxK units are looked up.
constexpr int kFusedSelectShort = 1024;
constexpr int kFusedSelectMax = 8192;
constexpr int kFusedSelectMaxK = 1024;

struct AttendArgs {
  int batch, n_q_heads, n_kv_heads, head_dim;
  int64_t capacity, q_head_stride, out_head_stride;
  float sm_scale;
  StepGeom geom;
  const void* q;
  const void* k_store;
  const void* v_store;
  // Positional remap: parts [0, parts_mem) cover the memory keys (virtual
  // indices [0, mem_len): I and the selected units) with unrotated keys from
  // k_store and queries turned by R(l_L); parts [parts_mem, parts) cover L and X
  // with keys from k_rot and queries at their own positions.  Without the remap
  // parts_mem = 0 and every part reads k_store.
  const void* k_rot;
  int parts_mem;
  int mem_len;
  RopeArgs rope;
  // Variable-length batches (var.on): each sequence's geometry, memory length and
  // memory parts are derived from var.past[b] (n_local is l_L); geom, mem_len and
  // parts_mem then only carry the shared fields.
  VarLen var;
  int n_local;
  const int32_t* idx;
  // Lookup inside the attention (idx_out non-null; matrix-core kernel,
  // n_units <= kFusedSelectMax, n_sel <= kFusedSelectMaxK; decode kernel, n_units <=
  // kDecodeSelMax): a workgroup whose tiles hold unit
  // keys selects its kv head's n_sel units from the score row itself, with the
  // select of infllm_select_topk, instead of reading idx; the workgroup of row
  // tile 0 and part 0 also writes the row to idx_out (the -1 padding included).
  const float* sel_scores;  // [batch * n_kv_heads][sel_stride]; not read for a sequence that looks up every unit or none
  int64_t sel_stride;
  int sel_units;            // most units in any score row (picks the select's keys per thread)
  int32_t* idx_out;         // [batch * n_kv_heads][geom.idx_stride]
  // Per-tile unit-mass partials (with sel_scores; null: off): for tile u of the
  // looked-up units (u < n_sel * l_bs / 64; l_I and l_bs multiples of 64) and
  // attention row r (query-major, r = i * G + h) of kv row bg:
  // mass_part[(bg * mass_tiles + u) * G * n_q + r] = (sum of P over the tile, m)
  // with P = exp2(z * log2(e) - m), z the logit.
  float2* mass_part;
  int mass_tiles;  // tiles per kv row in mass_part (k * l_bs / 64)
  void* out;     // final output (one part)
  float* lse;    // nullable
  // Split-key partials (parts > 1), see the layout in common.h: float32 rows for
  // float32 inputs; for bf16 inputs fp16 rows scaled by 2^-part_exp[row].
  void* part_o;        // [parts][rows][D]
  float* part_lse;     // [parts][rows]
  int32_t* part_exp;   // [parts][rows] (bf16 only)
  int parts;
  // Matrix-core kernel: waves of a workgroup that hold query rows (8, or 4 where the
  // rows are too few to fill the chip with 8); its launcher fills the divisors.
  int row_waves;
  FastDiv d_row_tiles, d_parts, d_kv, d_group, d_block;
  bool bf16;
};
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
__device__ __forceinline__ void prompt_item(const PromptArgs& a, int item, int& p, int& t) {
  const int* begin = item < a.full_begin[a.parts] ? a.full_begin : a.rest_begin;
  int x = 0;
  for (int i = 1; i < a.parts; ++i) x += item >= begin[i] ? 1 : 0;
  p = begin == a.full_begin ? x : a.parts - 1 - x;
  t = item - begin[x] + (begin == a.full_begin ? 0 : a.full[p]);
}
__device__ __forceinline__ int prompt_item_of(const PromptArgs& a, int p, int t) {
  return t < a.full[p] ? a.full_begin[p] + t : a.rest_begin[a.parts - 1 - p] + t - a.full[p];
}
// Row tiles with a part p.
__device__ __forceinline__ int prompt_part_count(const PromptArgs& a, int p) {
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

struct ThinScoreArgs {
  const float* unit_ksum;
  float* scores;
  int max_units, n_units, block_size;  // n_units: the largest of the batch
  int64_t score_stride;
};
// The append of a few tokens (at most kThinAppend, no units to build) and the scores
// of all units against them in one launch: a.rope must hold both tables.
constexpr int kThinAppend = 8;
hipError_t launch_append_score(const AppendArgs& a, const ThinScoreArgs& sc, hipStream_t s);

// The step of sequence b as a kernel sees it.
struct SeqStep {
  StepGeom geom;
  int mem_len;
  int parts_mem;
};
__host__ __device__ inline SeqStep seq_step(const AttendArgs& a, int b) {
  SeqStep r;
  if (!a.var.on) {
    r.geom = a.geom;
    r.mem_len = a.mem_len;
    r.parts_mem = a.parts_mem;
    return r;
  }
  r.geom = seq_geom(a.geom, a.n_local, a.var.past[b]);
  r.mem_len = r.geom.n_init + r.geom.n_sel * r.geom.block_size;
  r.parts_mem = a.rope.on ? split_parts_mem(a.parts, r.mem_len, r.geom.n_virtual) : 0;
  return r;
}
// Number of key parts the attention uses for this shape, limited by max_parts, and
// for the matrix-core kernel the waves of a workgroup that hold rows.
int attend_choose_parts(bool bf16, int batch, int n_q_heads, int n_kv_heads, int head_dim, int n_q, int n_sel,
                        int n_virtual, int max_parts, int* row_waves);
hipError_t launch_attend(const AttendArgs& a, hipStream_t s);
// Most scores a row may hold for the launch to select its units itself (see
// AttendArgs::idx_out); -1 where its kernel never does.
int attend_select_max(const AttendArgs& a);
// Whether launch_attend runs the matrix-core kernel for these arguments.
bool attend_uses_mfma(const AttendArgs& a);

struct MergeArgs {
  int rows, head_dim, parts, n_q, n_q_heads;
  int64_t out_head_stride;
  const void* part_o;
  const float* part_lse;
  const int32_t* part_exp;
  void* out;
  float* lse;
  bool bf16;
};
hipError_t launch_merge(const MergeArgs& a, hipStream_t s);

// Attention mass of the looked-up units and the frequency-score update.
constexpr int kMassMaxK = 1024;  // most lookup slots per row
struct MassArgs {
  int rows;  // batch * n_kv_heads
  int n_q_heads, n_kv_heads, head_dim;
  int n_q, k, n_units, max_units, block_size;
  int64_t n_init;  // l_I: first position of unit 0
  int64_t capacity, q_head_stride;
  float sm_scale, decay;
  const void* q;
  const void* k_store;
  const int32_t* idx;  // [rows][k]
  const float* lse;    // [batch][Hq][n_q] natural log
  float* mass;         // [rows][k]
  float* freq;         // [rows][max_units] or null
  RopeArgs rope;
  bool bf16;
};
hipError_t launch_unit_mass(const MassArgs& a, hipStream_t s);

// Unit masses from the attention's per-tile partials (AttendArgs::mass_part):
// for slot j < n_sel of kv row bg, mass = sum over the unit's tiles and the
// G * n_q rows of P_sum * exp2(m - lse * log2(e)), lse the step's merged
// natural-log normaliser; slots past n_sel get 0.  The frequency scores as in
// launch_unit_mass.
struct MassPartsArgs {
  int rows;  // batch * n_kv_heads
  int n_q_heads, n_kv_heads, n_q, k, n_sel, n_units, max_units;
  int tiles_per_unit, mass_tiles;
  float decay;
  const float2* mass_part;
  const int32_t* idx;  // [rows][k]
  const float* lse;    // [batch][Hq][n_q]
  float* mass;         // [rows][k]
  float* freq;         // [rows][max_units] or null
};
hipError_t launch_unit_mass_parts(const MassPartsArgs& a, hipStream_t s);

}  // namespace infllm
