// C ABI of what a batch over shared documents needs beside the step (declared in
// include/infllm.h): packed prompts, scoring and attention of the continuations of one
// document, copies of sequences between memories.  As in abi.cpp every check runs before
// the first HIP call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "abi_util.h"

using namespace infllm;

namespace {

// Rows (token, head) of a tensor read or written in 16-byte pieces: `tok` and `head` are
// the strides in elements.
infllm_status check_strided(const infllm_params* p, const void* ptr, int64_t tok, int64_t head) {
  if (ptr == nullptr) return INFLLM_E_NULL;
  if (tok < 0 || head < 0 || ((tok * esize(p)) & 15) != 0 || ((head * esize(p)) & 15) != 0 || !aligned16(ptr))
    return INFLLM_E_SHAPE;
  return INFLLM_OK;
}

// Waves of 32 query rows of a workgroup of the prompt attention.  bf16: 8, or 4 where 8
// leave compute units without a workgroup; float32: as the rows of the longest sequence fill.
int prompt_row_waves(bool bf16, int64_t rows8, int64_t longest_rows) {
  if (bf16) return rows8 < kMfmaTargetWgs ? kMfmaWaves / 2 : kMfmaWaves;
  return longest_rows > 64 ? 4 : longest_rows > 32 ? 2 : 1;
}

}  // namespace

extern "C" {

size_t infllm_prompt_workspace_bytes(const infllm_params* p, int32_t n_seqs, const int32_t* seq_lens) {
  (void)seq_lens;
  (void)n_seqs;
  (void)p;
  return 0;
}

infllm_status infllm_prompt_attend(const infllm_params* p, int32_t n_seqs, const int32_t* seq_lens, const void* q,
                                   int64_t q_token_stride, int64_t q_head_stride, const void* k, const void* v,
                                   int64_t kv_token_stride, int64_t kv_head_stride, void* out,
                                   int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  (void)workspace;
  (void)workspace_bytes;
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if (remap(p)) return INFLLM_E_UNSUPPORTED;
  if (n_seqs < 0) return INFLLM_E_SHAPE;
  if (n_seqs == 0) return INFLLM_OK;
  if (seq_lens == nullptr) return INFLLM_E_NULL;
  const int G = p->n_q_heads / p->n_kv_heads;
  const bool bf16 = p->dtype == INFLLM_BF16;
  int64_t total = 0, tiles8 = 0, longest = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (seq_lens[i] < 0) return INFLLM_E_SHAPE;
    total += seq_lens[i];
    tiles8 += ((int64_t)seq_lens[i] * G + 32 * kMfmaWaves - 1) / (32 * kMfmaWaves);
    longest = std::max<int64_t>(longest, seq_lens[i]);
  }
  if (total == 0) return INFLLM_OK;
  if (total > INT32_MAX || total * G > INT32_MAX || (total * G / 32 + n_seqs) * p->n_kv_heads > INT32_MAX)
    return INFLLM_E_UNSUPPORTED;
  if ((st = check_strided(p, q, q_token_stride, q_head_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, k, kv_token_stride, kv_head_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, v, kv_token_stride, kv_head_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, out, out_token_stride, out_head_stride)) != INFLLM_OK) return st;
  // two rows of the output never share an element: one stride steps over all of the other's rows
  const int64_t D = p->head_dim;
  const bool by_head = out_token_stride >= D && (p->n_q_heads == 1 || out_head_stride >= (total - 1) * out_token_stride + D);
  const bool by_token = out_head_stride >= D && (total == 1 || out_token_stride >= (p->n_q_heads - 1) * out_head_stride + D);
  if (!by_head && !by_token) return INFLLM_E_SHAPE;
  // the bf16 kernel addresses the keys of a sequence with 32-bit byte offsets
  if (bf16 && ((uint64_t)kv_token_stride > 0x7FFFFFFFull ||
               (uint64_t)(longest - 1) * (uint64_t)kv_token_stride * 2u + (uint64_t)D * 2u > 0xFFFFFFFFull))
    return INFLLM_E_UNSUPPORTED;
  if ((st = check_device()) != INFLLM_OK) return st;

  PromptArgs a;
  std::memset(&a, 0, sizeof(a));
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
  a.row_waves = prompt_row_waves(bf16, tiles8 * p->n_kv_heads, longest * G);
  const int rows_wg = 32 * a.row_waves;
  int64_t at = 0;
  for (int i0 = 0; i0 < n_seqs;) {
    // the next sequences that are not empty, the longest first (equal ones in their order)
    int n = 0;
    int32_t start[kMaxPrompts], len[kMaxPrompts];
    uint16_t order[kMaxPrompts];
    for (; i0 < n_seqs && n < kMaxPrompts; at += seq_lens[i0++]) {
      if (seq_lens[i0] == 0) continue;
      start[n] = (int32_t)at;
      len[n] = seq_lens[i0];
      order[n] = (uint16_t)n;
      ++n;
    }
    if (n == 0) break;
    std::sort(order, order + n, [&](uint16_t x, uint16_t y) { return len[x] != len[y] ? len[x] > len[y] : x < y; });
    a.n_seqs = n;
    a.n_tiles = 0;
    auto tiles = [&](int j) { return (int)(((int64_t)a.len[j] * G + rows_wg - 1) / rows_wg); };
    for (int j = 0; j < n; ++j) {
      a.start[j] = start[order[j]];
      a.len[j] = len[order[j]];
    }
    for (int j = 0; j < n; ++j) {
      // the levels that exactly the j + 1 longest sequences reach hold j + 1 tiles each
      a.first[j] = a.n_tiles;
      a.n_tiles += (j + 1) * (tiles(j) - (j + 1 < n ? tiles(j + 1) : 0));
    }
    if ((st = launch_status(launch_prompt(a, (hipStream_t)stream))) != INFLLM_OK) return st;
  }
  return INFLLM_OK;
}

}  // extern "C"

namespace {

// Launch shape of the prefix attention.
struct PrefixPlan {
  int row_waves, tiles_s, tiles_p;
  int most_s, most_u, most_o;  // most parts of the regions
  int parts_s, parts_u, parts_o;
};

int key_tile(bool bf16) { return bf16 ? 64 : 32; }
int prefix_target(bool bf16, int row_waves) { return bf16 ? kMfmaTargetWgs : kMfmaTargetWgs * 4 / row_waves; }

// The part counts' bounds follow from the shape alone, so that the workspace does.
PrefixPlan prefix_shape(const infllm_params* p, int batch, int n_q, int64_t shared_keys, int64_t unit_keys,
                        int64_t own_keys) {
  PrefixPlan r;
  const bool bf16 = p->dtype == INFLLM_BF16;
  const int64_t G = p->n_q_heads / p->n_kv_heads, rows_p = G * n_q, rows_s = rows_p * batch;
  const int64_t most_rows = shared_keys > 0 ? rows_s : rows_p;
  r.row_waves = bf16 ? (most_rows > 32 * kMfmaWaves / 2 ? kMfmaWaves : kMfmaWaves / 2)
                     : (most_rows > 64 ? 4 : most_rows > 32 ? 2 : 1);
  const int rows_wg = 32 * r.row_waves, target = prefix_target(bf16, r.row_waves);
  r.tiles_s = (int)((rows_s + rows_wg - 1) / rows_wg);
  r.tiles_p = (int)((rows_p + rows_wg - 1) / rows_wg);
  auto most = [&](int64_t keys, int64_t wgs) {
    const int64_t tiles = (keys + key_tile(bf16) - 1) / key_tile(bf16);
    return (int)std::min<int64_t>(tiles, 2 * target / std::max<int64_t>(1, wgs * p->n_kv_heads) + 1);
  };
  r.most_s = most(shared_keys, r.tiles_s);
  r.most_u = most(unit_keys, (int64_t)batch * r.tiles_p);
  r.most_o = std::max(1, most(own_keys, (int64_t)batch * r.tiles_p));
  r.parts_s = r.parts_u = r.parts_o = 0;
  return r;
}

// Parts of at most T tiles each, T the least that keeps the workgroups within a number of
// rounds: of one to four rounds the one whose time, a prologue and T tiles for each, is least.
void prefix_parts(const infllm_params* p, int batch, int64_t shared_keys, int64_t unit_keys, int64_t own_keys,
                  PrefixPlan* r) {
  const bool bf16 = p->dtype == INFLLM_BF16;
  const int kt = key_tile(bf16), target = prefix_target(bf16, r->row_waves);
  const int64_t ts = (shared_keys + kt - 1) / kt, tu = (unit_keys + kt - 1) / kt, to = (own_keys + kt - 1) / kt;
  auto parts = [](int64_t tiles, int64_t T, int most) { return (int)std::min<int64_t>((tiles + T - 1) / T, most); };
  auto wgs = [&](int64_t T) {
    return p->n_kv_heads * ((int64_t)r->tiles_s * parts(ts, T, r->most_s) +
                            (int64_t)batch * r->tiles_p * (parts(tu, T, r->most_u) + parts(to, T, r->most_o)));
  };
  auto longest = [&](int64_t T) {  // tiles of the longest part, under the bounds
    int64_t x = 0;
    if (ts > 0) x = std::max(x, (ts + parts(ts, T, r->most_s) - 1) / parts(ts, T, r->most_s));
    if (tu > 0) x = std::max(x, (tu + parts(tu, T, r->most_u) - 1) / parts(tu, T, r->most_u));
    if (to > 0) x = std::max(x, (to + parts(to, T, r->most_o) - 1) / parts(to, T, r->most_o));
    return x;
  };
  const int64_t most_tiles = std::max(std::max(ts, tu), std::max<int64_t>(to, 1));
  constexpr int kPartCost = 5;  // prologue and epilogue of a workgroup, in tiles
  int64_t best = most_tiles, best_cost = -1;
  for (int rounds = 1; rounds <= 4; ++rounds) {
    int64_t lo = 1, hi = most_tiles;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (wgs(mid) <= (int64_t)rounds * target) hi = mid;
      else lo = mid + 1;
    }
    const int64_t real = (wgs(lo) + target - 1) / target;
    const int64_t cost = real * (kPartCost + longest(lo));
    if (best_cost < 0 || cost < best_cost) {
      best = lo;
      best_cost = cost;
    }
  }
  r->parts_s = ts > 0 ? parts(ts, best, r->most_s) : 0;
  r->parts_u = tu > 0 ? parts(tu, best, r->most_u) : 0;
  r->parts_o = std::max(1, parts(to, best, r->most_o));
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
  if ((int64_t)batch * p->n_kv_heads > 65535 || (int64_t)(p->n_q_heads / p->n_kv_heads) * n_q > INT32_MAX)
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
    if (own_lens[b] + n_q > own->capacity) return INFLLM_E_RANGE;
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
  if (shared > INT32_MAX || units > INT32_MAX || own_most + n_q > INT32_MAX || G * n_q * B > INT32_MAX)
    return INFLLM_E_UNSUPPORTED;
  // the bf16 kernel addresses one (sequence, kv head) slice of a store with 32-bit byte offsets
  if (bf16 && ((uint64_t)prefix->capacity * D * 2u > 0xFFFFFFFFull || (uint64_t)own->capacity * D * 2u > 0xFFFFFFFFull))
    return INFLLM_E_UNSUPPORTED;
  if (n_q == 0) return INFLLM_OK;
  PrefixPlan r = prefix_shape(p, B, n_q, shared, units, own->capacity);
  prefix_parts(p, B, shared, units, own_most + n_q, &r);
  const int parts = r.parts_s + r.parts_u + r.parts_o;
  if (parts > 1) {
    if (workspace == nullptr || workspace_bytes < attend_ws_bytes(p, B, n_q, parts)) return INFLLM_E_WORKSPACE;
    if (!aligned16(workspace)) return INFLLM_E_SHAPE;
  }
  if ((st = check_device()) != INFLLM_OK) return st;
  hipStream_t s = (hipStream_t)stream;
  if (k != nullptr) {
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
  a.d_parts_o = fast_div(r.parts_o);
  a.out = out;
  a.lse = lse;
  a.bf16 = bf16;
  for (int b = 0; b < B; ++b) a.own_len[b] = own_lens[b];
  if (parts > 1) partial_layout(p, workspace, parts, (int64_t)B * p->n_q_heads * n_q, &a.part_o, &a.part_lse, &a.part_exp);
  if ((st = launch_status(launch_prefix(a, s))) != INFLLM_OK) return st;
  if (parts == 1) return INFLLM_OK;
  MergeArgs ma = merge_args(p, B, n_q, parts, workspace, out, out_head_stride, lse);
  return launch_status(launch_merge(ma, s));
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
      if ((int64_t)p->n_kv_heads * m->ring * p->head_dim / 2 > INT32_MAX) return INFLLM_E_UNSUPPORTED;
    }
    if ((int64_t)p->n_kv_heads * units * std::max(p->head_dim / 4, p->n_repr) > INT32_MAX) return INFLLM_E_UNSUPPORTED;
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
