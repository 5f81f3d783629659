// C ABI of what a batch over shared documents needs beside the step (declared in
// include/infllm.h): packed prompts, scoring and attention of the continuations of one
// document, copies of sequences between memories.  As in abi.cpp every check runs before
// the first HIP call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "abi_util.h"
#include "shared.h"

using namespace infllm;

namespace {

// Rows (token, head) of a tensor read or written in 16-byte pieces: `tok` and `head` are
// the strides in elements.
infllm_status check_strided(const infllm_params* p, const void* ptr, int64_t tok, int64_t head) {
  if (ptr == nullptr) return INFLLM_E_NULL;
  const int64_t piece = 16 / esize(p);
  if (tok < 0 || head < 0 || tok % piece != 0 || head % piece != 0 || !aligned16(ptr)) return INFLLM_E_SHAPE;
  return INFLLM_OK;
}

// Whether offsets into rows of head_dim elements, n1 by n2 of them with strides s1 and s2,
// stay within 62 bits: kernels and checks multiply them in 64.
bool span_fits(const infllm_params* p, int64_t n1, int64_t s1, int64_t n2 = 1, int64_t s2 = 0) {
  return ((__int128)(n1 - 1) * s1 + (__int128)(n2 - 1) * s2 + p->head_dim) * esize(p) <= (__int128)1 << 62;
}
bool store_fits(const infllm_params* p, const infllm_memory* m) {
  return (__int128)m->batch * p->n_kv_heads * m->capacity <= ((__int128)1 << 62) / (p->head_dim * esize(p));
}
// Whether the product of three numbers that are not negative fits 31 bits.
bool fits31(int64_t a, int64_t b, int64_t c) { return (__int128)a * b * c <= INT32_MAX; }

int key_tile(bool bf16) { return bf16 ? 64 : 32; }

// Whether a launch of so many workgroups stays within 2^32 threads.
bool launchable(int64_t wgs, int threads) { return wgs < (int64_t)(0xFFFFFFFFull / (uint64_t)threads); }

// Workgroups that run at a time: the bf16 kernel's by their LDS, the float32 kernel's by
// their registers.
int resident_wgs(const infllm_params* p, int row_waves) {
  if (p->dtype == INFLLM_BF16) return row_waves == kMfmaWaves ? kMfmaTargetWgs : 2 * kMfmaTargetWgs;
  return kMfmaTargetWgs * 4 / row_waves * (p->head_dim == 64 && row_waves > 1 ? 2 : 1);
}

// Lengths of all sequences; false where they are not valid.
struct PromptSizes {
  int64_t total, longest;
};
bool prompt_sizes(int32_t n_seqs, const int32_t* lens, PromptSizes* r) {
  r->total = r->longest = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (lens[i] < 0) return false;
    r->total += lens[i];
    r->longest = std::max<int64_t>(r->longest, lens[i]);
  }
  return true;
}

// Whether every row tile, part and kv head of such prompts has its number in 32 bits.
bool prompt_fits(const infllm_params* p, int32_t n_seqs, const PromptSizes& sizes) {
  const int64_t G = p->n_q_heads / p->n_kv_heads;
  return sizes.total <= INT32_MAX / G &&
         (sizes.total * G / 32 + n_seqs) * kMaxPromptParts <= INT32_MAX / p->n_kv_heads;
}

// Microseconds of a workgroup of the attention kernels, for each tile of keys and beside
// them (prologue, epilogue): with the whole chip at work, and of one that runs longer than
// the others (alone on its compute unit, at a higher clock).
struct ItemCost {
  float tile, item, lone_tile, lone_item;
};
ItemCost item_cost(const infllm_params* p, int row_waves) {
  const bool wide = p->head_dim == 128;
  if (p->dtype == INFLLM_BF16) {
    if (row_waves == kMfmaWaves) return wide ? ItemCost{1.72f, 10.f, 1.4f, 8.2f} : ItemCost{1.02f, 9.f, 0.87f, 7.5f};
    return wide ? ItemCost{1.76f, 9.f, 0.95f, 6.5f} : ItemCost{0.96f, 8.5f, 0.72f, 5.5f};
  }
  return wide ? ItemCost{6.6f, 12.f, 6.6f, 12.f} : row_waves > 1 ? ItemCost{6.2f, 10.f, 4.2f, 8.f} : ItemCost{3.7f, 8.f, 3.7f, 8.f};
}
constexpr float kMergeCost = 9.f;          // microseconds of a merge's launch
constexpr float kPartialByteCost = 2.5e-7f;  // of a byte of a partial row, written and read

// The sequences of the next launch, from lens[*i] on (first token *at): the shape fields,
// tile numbers and key parts of `a`.  False when none is left.
bool prompt_next(const infllm_params* p, int32_t n_seqs, const int32_t* lens, int* i, int64_t* at,
                 PromptArgs* a) {
  const int64_t G = p->n_q_heads / p->n_kv_heads;
  const bool bf16 = p->dtype == INFLLM_BF16;
  int n = 0;
  int32_t start[kMaxPrompts], len[kMaxPrompts];
  uint16_t order[kMaxPrompts];
  for (; *i < n_seqs && n < kMaxPrompts; *at += lens[(*i)++]) {
    if (lens[*i] == 0) continue;
    start[n] = (int32_t)*at;
    len[n] = lens[*i];
    order[n] = (uint16_t)n;
    ++n;
  }
  if (n == 0) return false;
  // the longest first, equal ones in their order
  std::sort(order, order + n, [&](uint16_t x, uint16_t y) { return len[x] != len[y] ? len[x] > len[y] : x < y; });
  a->n_seqs = n;
  a->n_kv_heads = p->n_kv_heads;
  for (int j = 0; j < n; ++j) {
    a->start[j] = start[order[j]];
    a->len[j] = len[order[j]];
  }
  const int kt = key_tile(bf16);
  int64_t rows_wg = 0;
  // Row tiles of sequence j; tiles of keys that a row tile of level R sees at most; the
  // first level that sees more than x of them; the row tiles of level R and above.
  auto tiles = [&](int j) { return j < n ? ((int64_t)a->len[j] * G + rows_wg - 1) / rows_wg : 0; };
  auto keys_of = [&](int64_t R) { return ((R + 1) * rows_wg - 1) / G / kt + 1; };
  auto level_past = [&](int64_t x) { return x * kt * G / rows_wg; };
  auto row_tiles_from = [&](int64_t R) {
    int64_t c = 0;
    for (int j = 0; j < n && tiles(j) > R; ++j) c += tiles(j) - R;
    return c;
  };
  // The rows of a workgroup and the parts along the keys.  The launch lasts as long as its
  // work shared over the workgroups that run at a time, or as a part, and where the parts
  // do not all start at once about half a part more; a split costs the merge.  Measured,
  // in us (bf16, D = 128): 16,000 tokens of 32 / 8 heads by 8 waves 1,716, by 4 1,757;
  // 4,000 126 and 132; 2,000 53 and 43; 1,000 28 and 23, in two parts 29 and 29; 16 of 300
  // 41 and 37; 4,000 of 4 / 1 heads by 4 waves 57, in 3 parts 35, in 8 43; 6,000 of 8 / 8
  // by 8 waves 130, in 2 parts 90.  Float32, 5 prompts up to 1,600 tokens of 8 / 2 heads
  // of 64: 174, in 6 parts 72.
  const int64_t most_rows = (int64_t)a->len[0] * G;
  const int least_waves = bf16 ? kMfmaWaves / 2 : most_rows > 64 ? 4 : most_rows > 32 ? 2 : 1;
  const int most_waves = bf16 ? kMfmaWaves : least_waves;
  float best_cost = -1.f;
  for (int waves = most_waves; waves >= least_waves; waves /= 2) {
    rows_wg = 32 * waves;
    const ItemCost cost = item_cost(p, waves);
    const float share = (float)p->n_kv_heads / (float)resident_wgs(p, waves);
    const int64_t longest = std::min(keys_of(tiles(0) - 1), ((int64_t)a->len[0] + kt - 1) / kt);
    float work = 0.f;  // tiles of keys of all row tiles
    for (int j = 0; j < n; ++j) work += (float)tiles(j) * (float)(keys_of(0) + keys_of(tiles(j) - 1)) * 0.5f;
    for (int c = 1; c <= kMaxPromptParts; ++c) {
      const int64_t T = (longest + c - 1) / c;
      if (c > 1 && T < 2) break;
      int64_t items = row_tiles_from(0), full = 0;
      for (int x = 1; x <= c; ++x) {
        if (x < c) items += row_tiles_from(level_past(x * T));
        full += row_tiles_from(level_past(x * T - 1));
      }
      const float even = share * (work * cost.tile + (float)items * cost.item);
      const float part = (float)T * cost.lone_tile + cost.lone_item;
      float t = std::max(even, part);
      if (c > 1) {
        if ((float)items * share > 1.f) t = std::max(even, part + 0.5f * (float)T * cost.tile + cost.item);
        t += kMergeCost + (float)(full * p->n_kv_heads * rows_wg) * (float)part_row_bytes(p) * kPartialByteCost;
      }
      if (best_cost < 0.f || t < best_cost) {
        best_cost = t;
        a->row_waves = waves;
        a->parts = c;
        a->part_tiles = (int)T;
      }
      if (even >= part) break;  // (more parts add nothing but workgroups)
    }
  }
  rows_wg = 32 * a->row_waves;
  // the levels that exactly the j + 1 longest sequences reach hold j + 1 tiles each
  a->n_tiles = 0;
  for (int j = 0; j < n; ++j) {
    a->first[j] = a->n_tiles;
    a->n_tiles += (int)((j + 1) * (tiles(j) - tiles(j + 1)));
  }
  int counts[kMaxPromptParts], parts = 0;
  const int64_t T = a->part_tiles;
  a->items = 0;
  for (int x = 0; x < a->parts; ++x) {
    counts[x] = x == 0 ? a->n_tiles : (int)row_tiles_from(level_past(x * T));
    if (counts[x] == 0) break;
    a->full[x] = (int)row_tiles_from(level_past((x + 1) * T - 1));
    a->full_begin[x] = a->items;
    a->items += a->full[x];
    parts = x + 1;
  }
  a->parts = parts;
  a->split_tiles = parts > 1 ? counts[1] : 0;
  a->full_begin[parts] = a->items;
  for (int x = 0; x < parts; ++x) {
    a->rest_begin[x] = a->items;
    a->items += counts[parts - 1 - x] - a->full[parts - 1 - x];
  }
  a->rest_begin[parts] = a->items;
  return true;
}

}  // namespace

extern "C" {

size_t infllm_prompt_workspace_bytes(const infllm_params* p, int32_t n_seqs, const int32_t* seq_lens) {
  PromptSizes sizes;
  if (check_params(p) != INFLLM_OK || n_seqs < 0 || (n_seqs > 0 && seq_lens == nullptr) ||
      !prompt_sizes(n_seqs, seq_lens, &sizes) || !prompt_fits(p, n_seqs, sizes))
    return 0;
  PromptArgs a;
  size_t most = 0;
  int64_t at = 0;
  for (int i = 0; prompt_next(p, n_seqs, seq_lens, &i, &at, &a);)
    most = std::max(most, (size_t)prompt_partial_rows(a) * part_row_bytes(p));
  return (most + 255) & ~(size_t)255;
}

infllm_status infllm_prompt_attend(const infllm_params* p, int32_t n_seqs, const int32_t* seq_lens, const void* q,
                                   int64_t q_token_stride, int64_t q_head_stride, const void* k, const void* v,
                                   int64_t kv_token_stride, int64_t kv_head_stride, void* out,
                                   int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if (remap(p)) return INFLLM_E_UNSUPPORTED;
  if (n_seqs < 0) return INFLLM_E_SHAPE;
  if (n_seqs == 0) return INFLLM_OK;
  if (seq_lens == nullptr) return INFLLM_E_NULL;
  const int G = p->n_q_heads / p->n_kv_heads;
  const bool bf16 = p->dtype == INFLLM_BF16;
  PromptSizes sizes;
  if (!prompt_sizes(n_seqs, seq_lens, &sizes)) return INFLLM_E_SHAPE;
  const int64_t total = sizes.total, longest = sizes.longest;
  if (total == 0) return INFLLM_OK;
  if (!prompt_fits(p, n_seqs, sizes)) return INFLLM_E_UNSUPPORTED;
  if ((st = check_strided(p, q, q_token_stride, q_head_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, k, kv_token_stride, kv_head_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, v, kv_token_stride, kv_head_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, out, out_token_stride, out_head_stride)) != INFLLM_OK) return st;
  // two rows of the output never share an element: one stride steps over all of the other's rows
  const int64_t D = p->head_dim;
  auto steps_over = [&](int64_t outer, int64_t inner, int64_t n) {  // outer >= (n - 1) * inner + D, in 64 bits
    return outer >= D && (n == 1 || inner <= (outer - D) / (n - 1));
  };
  const bool by_head = out_token_stride >= D && (p->n_q_heads == 1 || steps_over(out_head_stride, out_token_stride, total));
  const bool by_token = out_head_stride >= D && (total == 1 || steps_over(out_token_stride, out_head_stride, p->n_q_heads));
  if (!by_head && !by_token) return INFLLM_E_SHAPE;
  if (!span_fits(p, total, q_token_stride, p->n_q_heads, q_head_stride) ||
      !span_fits(p, total, kv_token_stride, p->n_kv_heads, kv_head_stride) ||
      !span_fits(p, total, out_token_stride, p->n_q_heads, out_head_stride))
    return INFLLM_E_UNSUPPORTED;
  // the bf16 kernel addresses the keys of a sequence with 32-bit byte offsets
  if (bf16 && ((uint64_t)kv_token_stride > 0x7FFFFFFFull ||
               (uint64_t)(longest - 1) * (uint64_t)kv_token_stride * 2u + (uint64_t)D * 2u > 0xFFFFFFFFull))
    return INFLLM_E_UNSUPPORTED;
  PromptArgs a;
  std::memset(&a, 0, sizeof(a));
  int launches = 0;
  int64_t at = 0;
  size_t need = 0;
  for (int i = 0; prompt_next(p, n_seqs, seq_lens, &i, &at, &a); ++launches) {
    need = std::max(need, (size_t)prompt_partial_rows(a) * part_row_bytes(p));
    if (!launchable((int64_t)a.items * p->n_kv_heads, 64 * a.row_waves)) return INFLLM_E_UNSUPPORTED;
  }
  if (need > 0) {
    if (workspace == nullptr || workspace_bytes < need) return INFLLM_E_WORKSPACE;
    if (!aligned16(workspace)) return INFLLM_E_SHAPE;
  }
  if ((st = check_device()) != INFLLM_OK) return st;

  a.n_q_heads = p->n_q_heads;
  a.n_kv_heads = p->n_kv_heads;
  a.head_dim = p->head_dim;
  a.q_tok = q_token_stride;
  a.q_head = q_head_stride;
  a.kv_tok = kv_token_stride;
  a.kv_head = kv_head_stride;
  a.out_tok = out_token_stride;
  a.out_head = out_head_stride;
  a.lse_stride = total;
  a.sm_scale = p->sm_scale;
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.lse = lse;
  a.bf16 = bf16;
  a.d_group = fast_div(G);
  a.d_kv = fast_div(p->n_kv_heads);
  at = 0;
  // (the shape of a call's only launch is there already)
  for (int i = 0, l = 0; l < launches && (launches == 1 || prompt_next(p, n_seqs, seq_lens, &i, &at, &a)); ++l) {
    const int64_t rows = prompt_partial_rows(a);
    if (rows > 0) partial_layout(p, workspace, 1, rows, &a.part_o, &a.part_lse, &a.part_exp);
    if ((st = launch_status(launch_prompt(a, (hipStream_t)stream))) != INFLLM_OK) return st;
    if (rows > 0 && (st = launch_status(launch_prompt_merge(a, (hipStream_t)stream))) != INFLLM_OK) return st;
  }
  return INFLLM_OK;
}

}  // extern "C"

namespace {

// Launch shape of the prefix attention.
struct PrefixPlan {
  int row_waves, tiles_s, tiles_p;   // row tiles of the shared region, and of one continuation
  int64_t keys_s, keys_u;            // tiles of keys
  int most_s, most_u, most_o;        // most parts of the regions
  int parts_s, parts_u, parts_o;
};

int64_t key_tiles(const infllm_params* p, int64_t keys) {
  const int kt = key_tile(p->dtype == INFLLM_BF16);
  return keys / kt + (keys % kt != 0);
}

// The part counts' bounds follow from the shape alone, so that the workspace does: a
// region takes at most one part more than fits a round of workgroups (300 row tiles on 512
// places: two; more row tiles than places: one).
PrefixPlan prefix_shape(const infllm_params* p, int batch, int n_q, int64_t shared_keys, int64_t unit_keys,
                        int64_t own_keys) {
  PrefixPlan r;
  const bool bf16 = p->dtype == INFLLM_BF16;
  const int64_t G = p->n_q_heads / p->n_kv_heads, rows_p = G * n_q, rows_s = rows_p * batch;
  const int64_t most_rows = shared_keys > 0 ? rows_s : rows_p;
  // (bf16: eight waves a workgroup are slower throughout, by up to 2 times with few rows;
  // of 3,200 rows over 68 tiles of keys 165 us against 163)
  r.row_waves = bf16 ? kMfmaWaves / 2 : most_rows > 64 ? 4 : most_rows > 32 ? 2 : 1;
  const int rows_wg = 32 * r.row_waves, at_a_time = resident_wgs(p, r.row_waves);
  r.tiles_s = (int)((rows_s + rows_wg - 1) / rows_wg);
  r.tiles_p = (int)((rows_p + rows_wg - 1) / rows_wg);
  r.keys_s = key_tiles(p, shared_keys);
  r.keys_u = key_tiles(p, unit_keys);
  auto most = [&](int64_t tiles, int64_t wgs) {
    return (int)std::min<int64_t>(tiles, at_a_time / std::max<int64_t>(1, wgs * p->n_kv_heads) + 1);
  };
  r.most_s = most(r.keys_s, r.tiles_s);
  r.most_u = most(r.keys_u, (int64_t)batch * r.tiles_p);
  r.most_o = most(key_tiles(p, own_keys), (int64_t)batch * r.tiles_p);
  r.parts_s = r.parts_u = r.parts_o = 0;
  return r;
}

// Parts of at most T tiles of keys each.  As for the prompts, the launch lasts as long as
// its work shared over the workgroups that run at a time, or as a part; where the last
// workgroups (the own tokens') have to wait for full parts of the other regions, as a part
// and one of theirs; the longer the parts, the longer its end, when few still run.  A tile of a row tile's own keys takes its share of the memory's
// rate, one that several row tiles read the matrix cores'; the merge adds its launch, a
// round trip for every eight parts of a lane group, and the partial rows' bytes.  Measured
// in us at T = 8, 12, 16, 24, 32, 48: 32 continuations of 64K tokens 89, 81, 79, 68, 70,
// 81; 8 of 8 tokens at 128K 48, 49, 41, 43, 46, 46; 64 of 8K tokens 34, 31, 32, 36, 46, 55.
void prefix_parts(const infllm_params* p, int batch, int n_q, const int64_t* own_lens, int64_t own_keys, PrefixPlan* r) {
  const bool bf16 = p->dtype == INFLLM_BF16, wide = p->head_dim == 128;
  const int Hkv = p->n_kv_heads, rows = batch * p->n_q_heads * n_q;
  const int64_t to = key_tiles(p, own_keys), pairs = (int64_t)batch * r->tiles_p;
  int64_t own_sum = 0;
  for (int b = 0; b < batch; ++b) own_sum += key_tiles(p, own_lens[b]);
  const float memory_tile = wide ? 2.8f : 1.4f, core_tile = item_cost(p, r->row_waves).tile;
  const float tile_s = bf16 && r->tiles_s < 2 ? memory_tile : core_tile;
  const float tile_p = bf16 && r->tiles_p < 2 ? memory_tile : core_tile;
  const float item = bf16 ? (r->tiles_s < 2 && r->tiles_p < 2 ? 5.f : 9.f) : 8.f;
  const float lone_tile = bf16 ? (wide ? 1.35f : 0.75f) : wide ? 5.9f : 3.4f, lone_item = bf16 ? 6.5f : wide ? 7.f : 5.f;
  const float share = (float)Hkv / (float)resident_wgs(p, r->row_waves);
  const int groups = 64 / (p->head_dim / (bf16 ? 8 : 4));  // lane groups of the merge
  const int64_t most_tiles = std::max<int64_t>(std::max(r->keys_s, r->keys_u), std::max<int64_t>(to, 1));
  auto parts = [](int64_t tiles, int64_t T, int most) { return (int)std::min<int64_t>((tiles + T - 1) / T, most); };
  auto longest = [](int64_t tiles, int n) { return n > 0 ? (tiles + n - 1) / n : 0; };
  const float work = ((float)(r->tiles_s * r->keys_s) * tile_s + (float)(pairs * r->keys_u + r->tiles_p * own_sum) * tile_p) * share;
  float best = -1.f;
  for (int64_t T = 1;; T += T < 6 ? 1 : T / 4) {  // (1 to 6, then steps of a quarter)
    T = std::min(T, most_tiles);
    const int ps = parts(r->keys_s, T, r->most_s), pu = parts(r->keys_u, T, r->most_u), po = parts(to, T, r->most_o);
    const int64_t full = (int64_t)r->tiles_s * ps + pairs * pu, items = full + pairs * po;
    const int64_t long_o = longest(to, po), long_p = std::max(std::max(longest(r->keys_s, ps), longest(r->keys_u, pu)), long_o);
    const float part = (float)long_p * lone_tile + lone_item;
    const float late = (float)items * share - 1.f;  // rounds of workgroups past the first
    float t = std::max(part, work + (float)items * share * item);
    if (late > 0.f && (float)full * share + late > 1.f) t = std::max(t, part + (float)long_o * lone_tile + lone_item);
    const int all = ps + pu + po;
    t += 0.2f * part + 4.f + 1.5f * (float)((all + 8 * groups - 1) / (8 * groups)) + (float)all * (float)rows * (float)part_row_bytes(p) * kPartialByteCost;
    if (best < 0.f || t < best) {
      best = t;
      r->parts_s = ps;
      r->parts_u = pu;
      r->parts_o = po;
    }
    if (T == most_tiles) break;
  }
}

// Keys of the shared region at document length `len`, and of the looked-up units.
void prefix_keys(const infllm_params* p, int64_t len, int k, Part* part, int64_t* shared, int64_t* units) {
  *part = partition(p, len);
  *shared = part->n_init + (len - part->local_begin);
  *units = (int64_t)std::min(k, part->n_units) * p->block_size;
}

}  // namespace

extern "C" {

size_t infllm_prefix_workspace_bytes(const infllm_params* p, int32_t batch, int32_t n_q, int64_t prefix_len,
                                     int64_t own_capacity) {
  if (check_params(p) != INFLLM_OK || batch < 1 || n_q < 0 || prefix_len < 0 || own_capacity < 0) return 0;
  if (!fits31(batch, p->n_q_heads, n_q)) return 0;
  Part part;
  int64_t shared, units;
  prefix_keys(p, prefix_len, p->topk, &part, &shared, &units);
  const PrefixPlan r = prefix_shape(p, batch, n_q, shared, units, own_capacity);
  const size_t a = attend_ws_bytes(p, batch, n_q, r.most_s + r.most_u + r.most_o);
  return (std::max(a, qbar_ws_bytes(p, batch, n_q)) + 255) & ~(size_t)255;
}

infllm_status infllm_prefix_score(const infllm_params* p, const infllm_memory* prefix, int32_t batch, const void* q,
                                  int64_t q_head_stride, int32_t n_q, int32_t n_units, float* scores, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if (remap(p)) return INFLLM_E_UNSUPPORTED;
  if (prefix == nullptr) return INFLLM_E_NULL;
  if (prefix->batch != 1 || batch < 1 || n_q < 0 || n_units < 0) return INFLLM_E_SHAPE;
  if (n_units > prefix->max_units) return INFLLM_E_RANGE;
  if (n_units == 0) return INFLLM_OK;
  if (prefix->unit_ksum == nullptr || scores == nullptr) return INFLLM_E_NULL;
  if (!aligned16(prefix->unit_ksum)) return INFLLM_E_SHAPE;
  if ((st = check_rows(p, q, q_head_stride, n_q)) != INFLLM_OK) return st;
  if ((int64_t)batch * p->n_kv_heads > 65535 || !fits31(batch, p->n_q_heads, n_q) ||
      !span_fits(p, (int64_t)batch * p->n_q_heads, q_head_stride))
    return INFLLM_E_UNSUPPORTED;
  if (workspace == nullptr) return INFLLM_E_NULL;
  if (workspace_bytes < qbar_ws_bytes(p, batch, n_q)) return INFLLM_E_WORKSPACE;
  if (!aligned16(workspace)) return INFLLM_E_SHAPE;
  if ((st = check_device()) != INFLLM_OK) return st;
  PrefixScoreArgs a;
  a.batch = batch;
  a.n_q_heads = p->n_q_heads;
  a.n_kv_heads = p->n_kv_heads;
  a.head_dim = p->head_dim;
  a.n_q = n_q;
  a.n_units = n_units;
  a.max_units = prefix->max_units;
  a.q_head_stride = q_head_stride;
  a.q = q;
  a.unit_ksum = prefix->unit_ksum;
  a.scores = scores;
  a.qbar_parts = (float*)workspace;
  a.bf16 = p->dtype == INFLLM_BF16;
  return launch_status(launch_prefix_score(a, (hipStream_t)stream));
}

infllm_status infllm_prefix_attend(const infllm_params* p, const infllm_memory* prefix, int64_t prefix_len,
                                   const infllm_memory* own, const int64_t* own_lens, const void* q,
                                   int64_t q_head_stride, const void* k, const void* v, int64_t kv_head_stride,
                                   int32_t n_q, const int32_t* idx, int32_t n_idx, void* out, int64_t out_head_stride,
                                   float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if (remap(p)) return INFLLM_E_UNSUPPORTED;
  if (own_lens == nullptr) return INFLLM_E_NULL;
  if ((st = check_store(p, prefix)) != INFLLM_OK) return st;
  if ((st = check_store(p, own)) != INFLLM_OK) return st;
  if (prefix->batch != 1 || prefix_len < 0 || n_q < 0 || n_idx < 0) return INFLLM_E_SHAPE;
  if (prefix_len > prefix->capacity) return INFLLM_E_RANGE;
  const int B = own->batch;
  if (B > kMaxVarBatch) return INFLLM_E_UNSUPPORTED;
  int64_t own_most = 0;
  for (int b = 0; b < B; ++b) {
    if (own_lens[b] < 0) return INFLLM_E_SHAPE;
    if (own_lens[b] > own->capacity - n_q) return INFLLM_E_RANGE;
    own_most = std::max(own_most, own_lens[b]);
  }
  if ((st = check_rows(p, q, q_head_stride, n_q)) != INFLLM_OK) return st;
  if ((st = check_rows(p, out, out_head_stride, n_q)) != INFLLM_OK) return st;
  if ((k == nullptr) != (v == nullptr)) return INFLLM_E_NULL;
  if (k != nullptr && ((st = check_rows(p, k, kv_head_stride, n_q)) != INFLLM_OK ||
                       (st = check_rows(p, v, kv_head_stride, n_q)) != INFLLM_OK))
    return st;
  Part part;
  int64_t shared, units;
  prefix_keys(p, prefix_len, n_idx, &part, &shared, &units);
  if (units > 0 && idx == nullptr) return INFLLM_E_NULL;
  const bool bf16 = p->dtype == INFLLM_BF16;
  const int64_t G = p->n_q_heads / p->n_kv_heads, D = p->head_dim;
  if (shared > INT32_MAX || units > INT32_MAX || own_most + n_q > INT32_MAX || !fits31(B, p->n_q_heads, n_q))
    return INFLLM_E_UNSUPPORTED;
  if (!store_fits(p, prefix) || !store_fits(p, own) || !span_fits(p, (int64_t)B * p->n_q_heads, q_head_stride) ||
      !span_fits(p, (int64_t)B * p->n_q_heads, out_head_stride) ||
      (k != nullptr && !span_fits(p, (int64_t)B * p->n_kv_heads, kv_head_stride)))
    return INFLLM_E_UNSUPPORTED;
  // the bf16 kernel addresses one (sequence, kv head) slice of a store with 32-bit byte offsets
  const int64_t most_rows = (int64_t)(0xFFFFFFFFull / (uint64_t)(2 * D));
  if (bf16 && (prefix->capacity > most_rows || own->capacity > most_rows))
    return INFLLM_E_UNSUPPORTED;
  if (n_q == 0) return INFLLM_OK;
  PrefixPlan r = prefix_shape(p, B, n_q, shared, units, own->capacity);
  // a few current tokens are met by the merge, and not in the own region
  const bool merge_x = k != nullptr && n_q <= kPrefixMergeTokens;
  prefix_parts(p, B, n_q, own_lens, own_most + (merge_x ? 0 : n_q), &r);
  const int parts = r.parts_s + r.parts_u + r.parts_o;
  if (!launchable((int64_t)p->n_kv_heads * ((int64_t)r.tiles_s * r.parts_s + (int64_t)B * r.tiles_p * (r.parts_u + r.parts_o)),
                  64 * r.row_waves) ||
      !launchable(((int64_t)B * p->n_q_heads * n_q + 3) / 4, 256))
    return INFLLM_E_UNSUPPORTED;
  const bool direct = parts == 1 && !merge_x;
  if (parts > 0 && !direct) {
    if (workspace == nullptr || workspace_bytes < attend_ws_bytes(p, B, n_q, parts)) return INFLLM_E_WORKSPACE;
    if (!aligned16(workspace)) return INFLLM_E_SHAPE;
  }
  if ((st = check_device()) != INFLLM_OK) return st;
  hipStream_t s = (hipStream_t)stream;
  if (k != nullptr && !merge_x) {
    // X joins the own stores: the copy role of the append (no ring, no scores)
    AppendArgs aa;
    std::memset(&aa, 0, sizeof(aa));
    aa.batch = B;
    aa.n_q_heads = p->n_q_heads;
    aa.n_kv_heads = p->n_kv_heads;
    aa.head_dim = p->head_dim;
    aa.n_q = n_q;
    aa.capacity = own->capacity;
    aa.q_head_stride = q_head_stride;
    aa.kv_head_stride = kv_head_stride;
    aa.q = q;
    aa.k_src = k;
    aa.v_src = v;
    aa.k_store = own->k;
    aa.v_store = own->v;
    aa.var.on = 1;
    for (int b = 0; b < B; ++b) aa.var.past[b] = own_lens[b];
    aa.mean_repr = true;
    aa.bf16 = bf16;
    if ((st = launch_status(launch_append(aa, s, nullptr, nullptr))) != INFLLM_OK) return st;
  }
  PrefixArgs a;
  std::memset(&a, 0, sizeof(a));
  a.batch = B;
  a.n_q_heads = p->n_q_heads;
  a.n_kv_heads = p->n_kv_heads;
  a.head_dim = p->head_dim;
  a.n_q = n_q;
  a.prefix_capacity = prefix->capacity;
  a.own_capacity = own->capacity;
  a.q_head_stride = q_head_stride;
  a.out_head_stride = out_head_stride;
  a.sm_scale = p->sm_scale;
  a.q = q;
  a.prefix_k = prefix->k;
  a.prefix_v = prefix->v;
  a.own_k = own->k;
  a.own_v = own->v;
  a.idx = idx;
  a.n_init = (int)part.n_init;
  a.n_units = part.n_units;
  a.n_sel = std::min(n_idx, part.n_units);
  a.block_size = p->block_size;
  a.unit_base = p->n_init;
  a.idx_stride = n_idx;
  a.local_begin = part.local_begin;
  a.prefix_len = prefix_len;
  a.parts_s = r.parts_s;
  a.parts_u = r.parts_u;
  a.parts_o = r.parts_o;
  a.parts = parts;
  a.direct = direct;
  if (merge_x) {
    a.x_k = k;
    a.x_v = v;
    a.x_head_stride = kv_head_stride;
  }
  a.row_waves = r.row_waves;
  a.tiles_s = r.tiles_s;
  a.tiles_p = r.tiles_p;
  a.d_group = fast_div((int)G);
  a.d_block = fast_div(p->block_size);
  a.d_kv = fast_div(p->n_kv_heads);
  a.d_q = fast_div(n_q);
  a.d_tiles_s = fast_div(r.tiles_s);
  a.d_tiles_p = fast_div(r.tiles_p);
  a.d_parts_u = fast_div(std::max(1, r.parts_u));
  a.d_parts_o = fast_div(std::max(1, r.parts_o));
  a.out = out;
  a.lse = lse;
  a.bf16 = bf16;
  for (int b = 0; b < B; ++b) a.own_len[b] = own_lens[b];
  if (!direct) partial_layout(p, workspace, parts, (int64_t)B * p->n_q_heads * n_q, &a.part_o, &a.part_lse, &a.part_exp);
  if (parts > 0 && (st = launch_status(launch_prefix(a, s))) != INFLLM_OK) return st;
  return direct ? INFLLM_OK : launch_status(launch_prefix_merge(a, s));
}

infllm_status infllm_copy_sequences(const infllm_params* p, const infllm_memory* dst, const infllm_memory* src, int32_t n,
                                    const int32_t* dst_seq, const int32_t* src_seq, const int64_t* lens,
                                    const int32_t* units_built, void* stream) {
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if ((st = check_store(p, dst)) != INFLLM_OK) return st;
  if ((st = check_store(p, src)) != INFLLM_OK) return st;
  if (n < 0) return INFLLM_E_SHAPE;
  if (n == 0) return INFLLM_OK;
  if (n > kMaxVarBatch) return INFLLM_E_UNSUPPORTED;
  if (dst_seq == nullptr || src_seq == nullptr || lens == nullptr || units_built == nullptr) return INFLLM_E_NULL;
  const bool rings = !mean_repr(p);
  int units = 0;
  for (int i = 0; i < n; ++i) {
    if (lens[i] < 0 || units_built[i] < 0) return INFLLM_E_SHAPE;
    if (dst_seq[i] < 0 || dst_seq[i] >= dst->batch || src_seq[i] < 0 || src_seq[i] >= src->batch) return INFLLM_E_RANGE;
    if (lens[i] > dst->capacity || lens[i] > src->capacity) return INFLLM_E_RANGE;
    if (units_built[i] > partition(p, lens[i]).n_units) return INFLLM_E_SHAPE;
    if (units_built[i] > dst->max_units || units_built[i] > src->max_units) return INFLLM_E_RANGE;
    units = std::max(units, units_built[i]);
  }
  for (const infllm_memory* m : {dst, src}) {
    if (units > 0 && (st = check_units(p, m)) != INFLLM_OK) return st;
    if (rings) {
      if (m->qprefix == nullptr || m->rpart == nullptr) return INFLLM_E_NULL;
      if (!aligned16(m->qprefix) || m->ring < 1) return INFLLM_E_SHAPE;
      if (!fits31(p->n_kv_heads, m->ring, p->head_dim / 2)) return INFLLM_E_UNSUPPORTED;
    }
    if (!fits31(p->n_kv_heads, units, std::max(p->head_dim / 4, p->n_repr)) || !store_fits(p, m)) return INFLLM_E_UNSUPPORTED;
  }
  // a copy goes to a slot of its own, which no pair reads
  const int64_t row = (int64_t)p->head_dim * esize(p);
  auto slot = [&](const infllm_memory* m, int s) { return (const char*)m->k + (int64_t)s * p->n_kv_heads * m->capacity * row; };
  auto meet = [&](const infllm_memory* x, int i, const infllm_memory* y, int j) {
    const char *a = slot(x, i), *b = slot(y, j);
    return a < b + p->n_kv_heads * y->capacity * row && b < a + p->n_kv_heads * x->capacity * row;
  };
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j)
      if ((j != i && dst_seq[i] == dst_seq[j]) || meet(dst, dst_seq[i], src, src_seq[j])) return INFLLM_E_SHAPE;
  if ((st = check_device()) != INFLLM_OK) return st;
  SeqCopyArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_pairs = n;
  a.n_kv_heads = p->n_kv_heads;
  a.row_bytes = (int)row;
  a.src_capacity = src->capacity;
  a.dst_capacity = dst->capacity;
  a.src_units = src->max_units;
  a.dst_units = dst->max_units;
  a.src_ring = rings ? src->ring : 1;
  a.dst_ring = rings ? dst->ring : 1;
  a.repr_bytes = mean_repr(p) ? 0 : p->n_repr * 4;
  a.cells = p->head_dim / 4;
  a.ring_rows = rings ? p->head_dim / kRpartDims : 0;
  a.src_k = (const char*)src->k;
  a.src_v = (const char*)src->v;
  a.src_rot = remap(p) ? (const char*)src->k_rot : nullptr;
  a.src_repr = (const char*)src->repr_idx;
  a.src_ksum = (const char*)src->unit_ksum;
  a.src_qprefix = (const char*)src->qprefix;
  a.src_rpart = (const char*)src->rpart;
  a.dst_k = (char*)dst->k;
  a.dst_v = (char*)dst->v;
  a.dst_rot = remap(p) ? (char*)dst->k_rot : nullptr;
  a.dst_repr = (char*)dst->repr_idx;
  a.dst_ksum = (char*)dst->unit_ksum;
  a.dst_qprefix = (char*)dst->qprefix;
  a.dst_rpart = (char*)dst->rpart;
  // pairs by source, and by length within a source
  int order[kMaxVarBatch];
  for (int i = 0; i < n; ++i) order[i] = i;
  std::sort(order, order + n, [&](int x, int y) {
    return src_seq[x] != src_seq[y] ? src_seq[x] < src_seq[y] : lens[x] != lens[y] ? lens[x] > lens[y] : x < y;
  });
  for (int i = 0; i < n; ++i) {
    const int o = order[i];
    if (i == 0 || src_seq[o] != a.src_seq[a.n_sources - 1]) {
      a.src_seq[a.n_sources] = src_seq[o];
      a.pair_begin[a.n_sources++] = i;
    }
    a.dst_seq[i] = dst_seq[o];
    a.len[i] = lens[o];
    a.built[i] = units_built[o];
  }
  a.pair_begin[a.n_sources] = n;
  return launch_status(launch_copy_sequences(a, (hipStream_t)stream));
}

}  // extern "C"
