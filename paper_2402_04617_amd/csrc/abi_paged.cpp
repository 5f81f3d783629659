// C ABI of the calls on paged caches (declared in include/infllm.h): rotary frequencies,
// norms and rotation, the append to pages, attention over them.  As in abi.cpp every check
// runs before the first HIP call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "abi_util.h"
#include "paged.h"

using namespace infllm;

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr int64_t kMostTokens = INT32_MAX - 255;  // of a sequence: tile ends past them stay in 31 bits

infllm_status check_rotary(const infllm_params* p, const infllm_rotary* r) {
  if (r == nullptr) return INFLLM_E_NULL;
  if (r->rotary_dim < 0 || r->rotary_dim > p->head_dim || r->rotary_dim % 2 != 0) return INFLLM_E_SHAPE;
  if (r->rotary_dim > 0) {
    if (r->inv_freq == nullptr) return INFLLM_E_NULL;
    if (!std::isfinite(r->magnitude)) return INFLLM_E_SHAPE;
    for (int i = 0; i < r->rotary_dim / 2; ++i)
      if (!std::isfinite(r->inv_freq[i]) || r->inv_freq[i] < 0.0) return INFLLM_E_SHAPE;
  }
  if (r->norm != 0) {
    if (!std::isfinite(r->norm_eps) || r->norm_eps < 0.f) return INFLLM_E_SHAPE;
    if (!aligned16(r->q_weight) || !aligned16(r->k_weight)) return INFLLM_E_SHAPE;
  }
  return INFLLM_OK;
}

// Rows (i, j), i < n1, j < n2, with strides s1 and s2: whether no two share an element.
bool apart(int64_t D, int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
  auto over = [&](int64_t outer, int64_t inner, int64_t n) {  // outer steps over n inner rows, in 64 bits
    return outer >= D && (n == 1 || inner <= (outer - D) / (n - 1));
  };
  const bool i_outer = (n2 == 1 || s2 >= D) && (n1 == 1 || over(s1, s2, n2));
  const bool j_outer = (n1 == 1 || s1 >= D) && (n2 == 1 || over(s2, s1, n1));
  return i_outer || j_outer;
}

infllm_status check_out(const infllm_params* p, const void* ptr, int64_t n_tokens, int64_t tok, int64_t n_heads, int64_t head) {
  infllm_status st = check_strided(p, ptr, tok, head);
  if (st != INFLLM_OK) return st;
  return apart(p->head_dim, n_tokens, tok, n_heads, head) ? INFLLM_OK : INFLLM_E_SHAPE;
}

// The pages: three strides, each of which steps over all rows of the smaller ones.
infllm_status check_pages(const infllm_params* p, const infllm_pages* g) {
  if (g == nullptr || g->k == nullptr || g->v == nullptr) return INFLLM_E_NULL;
  if (g->n_pages < 1 || g->page_size < 1) return INFLLM_E_SHAPE;
  infllm_status st;
  if ((st = check_strided(p, g->k, g->page_stride, g->token_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, g->v, g->head_stride, 0)) != INFLLM_OK) return st;
  struct Axis {
    int64_t n, s;
  } ax[3] = {{g->n_pages, g->page_stride}, {g->page_size, g->token_stride}, {p->n_kv_heads, g->head_stride}};
  std::sort(ax, ax + 3, [](const Axis& x, const Axis& y) { return x.s < y.s; });
  __int128 extent = p->head_dim;  // elements that the axes so far span
  for (const Axis& x : ax) {
    if (x.n == 1) continue;
    if (x.s < extent) return INFLLM_E_SHAPE;
    extent += (__int128)(x.n - 1) * x.s;
  }
  return extent * esize(p) <= (__int128)1 << 62 ? INFLLM_OK : INFLLM_E_UNSUPPORTED;
}

// The sequences' lengths: their sum, and whether they fit the table.
infllm_status check_seqs(const infllm_pages* g, int32_t n_seqs, const int32_t* lens, const int64_t* pasts,
                         int64_t table_stride, int64_t* total) {
  *total = 0;
  if (n_seqs < 0) return INFLLM_E_SHAPE;
  if (n_seqs == 0) return INFLLM_OK;
  if (lens == nullptr || pasts == nullptr) return INFLLM_E_NULL;
  if (table_stride < 0) return INFLLM_E_SHAPE;
  infllm_status st = INFLLM_OK;
  for (int i = 0; i < n_seqs; ++i) {
    if (lens[i] < 0 || pasts[i] < 0) return INFLLM_E_SHAPE;
    *total += lens[i];
    if (lens[i] == 0) continue;
    if (pasts[i] > kMostTokens - lens[i]) st = INFLLM_E_UNSUPPORTED;
    else if (st == INFLLM_OK && (pasts[i] + lens[i] - 1) / g->page_size >= table_stride) st = INFLLM_E_RANGE;
  }
  if (st == INFLLM_OK && (*total > INT32_MAX || (__int128)n_seqs * table_stride > (__int128)1 << 59)) st = INFLLM_E_UNSUPPORTED;
  return st;
}

// The sequences [i, i + kMaxPaged) of the call, the first of which starts at token `at`.
void fill_seqs(const infllm_pages* g, int32_t n_seqs, const int32_t* lens, const int64_t* pasts, const int32_t* table,
               int64_t table_stride, int i, int64_t at, PagedSeqs* s) {
  s->n_seqs = std::min(n_seqs - i, kMaxPaged);
  s->n_pages = g->n_pages;
  s->page_size = g->page_size;
  s->d_page = fast_div(g->page_size);
  s->table = table + i * table_stride;
  s->table_stride = table_stride;
  for (int j = 0; j < s->n_seqs; ++j) {
    s->start[j] = (int32_t)at;
    s->past[j] = lens[i + j] > 0 ? (int32_t)pasts[i + j] : 0;
    at += lens[i + j];
  }
  s->start[s->n_seqs] = (int32_t)at;
}

void set_rotary(const infllm_params* p, const infllm_rotary* r, RotateArgs* a) {
  a->head_dim = p->head_dim;
  a->bf16 = p->dtype == INFLLM_BF16;
  if (r == nullptr) return;
  a->rotary_dim = r->rotary_dim;
  a->interleaved = r->interleaved != 0;
  a->magnitude = r->magnitude;
  for (int i = 0; i < r->rotary_dim / 2; ++i) a->rev[i] = r->inv_freq[i] / kTwoPi;
  a->norm = r->norm != 0;
  a->eps = r->norm_eps;
  a->q_weight = r->q_weight;
  a->k_weight = r->k_weight;
}

// Whether a rotation's launch (a wave per token, more only where tokens are few) stays within
// 2^32 threads.
bool rotate_fits(int64_t tokens) { return tokens < (1 << 26) - 8192; }

// Microseconds of a workgroup of the attention, for each tile of keys and beside them: with
// the whole chip at work, and of one that runs nearly alone.  Row tiles of few rows read
// their keys at the memory's rate, of many they share them in the cache.  Fitted, with the
// rest of the model in `plan`, to 143 batches (1 to 190 sequences, single tokens, chunks of up
// to 5,000 and both together, up to 30,000 tokens before them, 64 and 128 dims, 1 to 8 kv
// heads, both types), each at a dozen part lengths: the length it chooses is on average
// within 1.3 % of the best in bf16 (3.5 % where single tokens and chunks meet), 3 % in float32.
// None of those batches had a cap, a bias or a window: a capped tile, which takes a quarter
// longer, is priced as a plain one.  So the row tiles of 700, 1,500 and 64 tokens with a cap and a
// window of 4,096 (192 of 66 key tiles, 376 of 12) stay whole, and the 192 run alone for half of
// the call.
// It takes the host 1 us for one sequence, 2.7, 8.4 and 27 for 16, 64 and 192.
struct ItemCost {
  float tile, item, lone_tile, lone_item;
};
ItemCost item_cost(const PagedArgs& a, bool thin) {
  const bool wide = a.head_dim == 128;
  if (a.bf16) {
    if (thin) return wide ? ItemCost{2.25f, 2.8f, 0.785f, 3.5f} : ItemCost{0.875f, 2.8f, 0.64f, 3.5f};
    return wide ? ItemCost{1.49f, 4.8f, 0.9f, 8.8f} : ItemCost{0.675f, 4.8f, 0.5f, 8.8f};
  }
  if (thin) return wide ? ItemCost{6.f, 5.f, 5.3f, 4.3f} : ItemCost{5.5f, 5.f, 2.7f, 4.3f};
  return wide ? ItemCost{5.5f, 6.4f, 5.2f, 3.7f} : ItemCost{7.5f, 6.4f, 2.5f, 3.7f};
}
// Of a merge: its launch, and for each item, byte of a partial row (written and read) and
// part that a row's threads take in turn.
struct MergeCost {
  float launch, item, byte, part;
};
MergeCost merge_cost(const PagedArgs& a) { return a.bf16 ? MergeCost{4.7f, 3.4e-3f, 2.6e-7f, 0.187f} : MergeCost{3.4f, 0.f, 4.2e-7f, 0.1f}; }
// Workgroups that run at a time: by their LDS (bf16 two to a compute unit), float32 by
// their registers too.
int resident_wgs(const PagedArgs& a) {
  if (a.bf16) return 512;
  if (a.head_dim == 128) return a.rows_log2 == 7 ? 256 : 512;
  return a.rows_log2 == 7 ? 512 : 1024;
}
constexpr int kMostParts = 256;              // of a row tile

// The sequences of the next launch, from lens[*i] on (first token *at): their parts and item
// numbers.  False where none is left, or (*ok) an item or its partial rows have no number.
// A row tile of n key tiles has ceil(n / T) parts of one length.  The items start in the
// order of their length.  Of as many as fill whole rounds of the workgroups that run at a
// time the launch takes their work's share; the others, the shortest, run side by side at
// a speed that grows as they end, up to that of one alone; a split costs the merge.
bool plan(const infllm_params* p, int32_t n_seqs, const int32_t* lens, const int64_t* pasts, int* i, int64_t* at, PagedArgs* a,
          bool* ok) {
  const int G = (int)a->d_group.d, Hkv = a->n_kv_heads;
  int n = 0;
  int32_t start[kMaxAttend], len[kMaxAttend], past[kMaxAttend];
  uint8_t row[kMaxAttend];
  *ok = true;
  a->table += *i * a->table_stride;
  int64_t most_rows = 0;
  const int from = *i;
  for (; *i < n_seqs && *i - from < kMaxAttend; *at += lens[(*i)++]) {
    if (lens[*i] == 0) continue;
    start[n] = (int32_t)*at;
    len[n] = lens[*i];
    past[n] = (int32_t)pasts[*i];
    row[n] = (uint8_t)(*i - from);
    most_rows = std::max(most_rows, (int64_t)lens[*i] * G);
    ++n;
  }
  a->n_seqs = n;
  a->items = 0;
  if (n == 0) return *i < n_seqs;
  a->key_tile = a->bf16 ? 64 : 32;
  a->rows_log2 = a->bf16 || most_rows > 64 ? 7 : most_rows > 32 ? 6 : 5;
  const int rows_wg = 1 << a->rows_log2;
  a->tile_queries = (rows_wg - 1) / G + 2;
  a->item_rows = (int)std::min<int64_t>(rows_wg, (most_rows + 7) / 8 * 8);
  // by sequence: row tiles, most key tiles of one, and the share of them that a causal one
  // sees on average; rows of an item
  int tiles[kMaxAttend], keys[kMaxAttend], rows[kMaxAttend], most = 0;
  float seen[kMaxAttend];
  for (int j = 0; j < n; ++j) {
    tiles[j] = paged_row_tiles(*a, G, len[j]);
    keys[j] = paged_most_tiles(*a, past[j], len[j]);
    rows[j] = (int)std::min<int64_t>(rows_wg, (int64_t)len[j] * G);
    const int first = paged_range(*a, past[j], 0, std::min(len[j], a->tile_queries) - 1).n;
    seen[j] = 0.5f * (float)(first + keys[j]) / (float)keys[j];
    most = std::max(most, keys[j]);
  }
  const int64_t slots = resident_wgs(*a);
  const ItemCost thin = item_cost(*a, true), thick = item_cost(*a, false);
  const MergeCost merge = merge_cost(*a);
  const int groups = a->item_rows > 16 ? 1 : 64 / (a->head_dim / (a->bf16 ? 8 : 4));  // that share a row's parts
  constexpr int kBins = 32;  // of item lengths
  float best = -1.f;
  int best_T = most;
  // (fewer lengths are looked at for many sequences, whose parts balance anyway: 192 of them
  // took the host 41 us)
  for (int T = most, c = 1; c <= kMostParts; c = std::max(c + 1, n > 48 ? c * 7 / 4 : c * 4 / 3)) {
    if (c > 1) {
      const int next = (most + c - 1) / c;
      if (next == T) {
        if (T == 1) break;
        continue;
      }
      T = next;
    }
    struct Bin {
      int64_t n;
      float time, work, lone;  // sums
    } bins[kBins] = {};
    float longest = 0.f, longest_alone = 0.f, bytes = 0.f;
    int turns = 0;
    const float per_T = 1.f / (float)T, top = (float)T * std::max(thin.tile, thick.tile) + std::max(thin.item, thick.item);
    int64_t items = 0;
    for (int j = 0; j < n; ++j) {
      const ItemCost& cost = rows[j] <= 32 ? thin : thick;
      // (a row tile of far fewer keys than T has its one part all the same)
      const int parts = std::max(1, (int)((float)keys[j] * per_T + 0.9985f));
      const int length = (int)((float)keys[j] / (float)parts + 0.9985f);
      const float time = (float)length * cost.tile + cost.item, lone = (float)length * cost.lone_tile + cost.lone_item;
      const int64_t count = (int64_t)tiles[j] * parts * Hkv;
      if (parts > 1) {
        bytes += (float)count * (float)rows[j];
        turns = std::max(turns, parts / groups);
      }
      Bin& b = bins[std::min(kBins - 1, (int)(time / top * kBins))];
      b.n += count;
      b.time += (float)count * time;
      b.work += (float)count * ((float)length * cost.tile * seen[j] + cost.item);
      b.lone += (float)count * lone / time;
      if (time > longest) {
        longest = time;
        longest_alone = lone;
      }
      items += count;
    }
    float t = 0.f;
    int64_t whole = items / slots * slots;  // items of full rounds
    int x = kBins - 1;
    for (; whole > 0; --x) {
      Bin& b = bins[x];
      if (b.n == 0) continue;
      const int64_t take = std::min(b.n, whole);
      const float part = (float)take / (float)b.n;
      t += b.work * part / (float)slots;
      b.time *= 1.f - part;
      b.lone *= 1.f - part;
      b.n -= take;
      whole -= take;
      if (b.n > 0) break;
    }
    const float full = t;  // for as long the chip is full
    int64_t left = items - items / slots * slots;
    float done = 0.f;
    for (int y = 0; y < kBins && left > 0; ++y) {
      const Bin& b = bins[y];
      if (y > x || b.n == 0) continue;
      const float time = b.time / (float)b.n;
      t += std::max(0.f, time - done) * std::max(b.lone / (float)b.n, (float)left / (float)slots);
      done = std::max(done, time);
      left -= b.n;
    }
    // (the longest runs alone from where the others leave off)
    t = std::max(t, longest_alone + std::min(full, longest) * (1.f - longest_alone / longest));
    if (bytes > 0.f)
      t += merge.launch + (float)items * merge.item + bytes * (float)(a->head_dim * (a->bf16 ? 2 : 4) + 8) * merge.byte +
           (float)turns * merge.part;
    if (best < 0.f || t < best) {
      best = t;
      best_T = T;
    }
    if (T == 1) break;
  }
  uint8_t order[kMaxAttend];
  int length[kMaxAttend];  // of a sequence's parts
  for (int j = 0; j < n; ++j) {
    const int parts = std::min(kMostParts, (keys[j] + best_T - 1) / best_T);
    length[j] = (keys[j] + parts - 1) / parts;
    order[j] = (uint8_t)j;
  }
  std::sort(order, order + n, [&](int x, int y) { return length[x] != length[y] ? length[x] > length[y] : x < y; });
  int64_t items = 0;
  for (int x = 0; x < n; ++x) {
    const int j = order[x], parts = (keys[j] + length[j] - 1) / length[j];
    a->first[x] = (int32_t)items;
    a->start[x] = start[j];
    a->len[x] = len[j];
    a->past[x] = past[j];
    a->parts[x] = (uint8_t)(parts - 1);
    a->table_row[x] = row[j];
    items += (int64_t)tiles[j] * parts;
    if (items * Hkv * 128 > INT32_MAX) *ok = false;
  }
  a->items = *ok ? (int)items : 0;
  return true;
}
// Partial rows of a launch (0 where no row tile has several parts).
int64_t partial_rows(const PagedArgs& a) {
  for (int i = 0; i < a.n_seqs; ++i)
    if (a.parts[i] > 0) return (int64_t)a.items * a.n_kv_heads * a.item_rows;
  return 0;
}

bool numbers_fit(const infllm_params* p, int64_t total) {
  return (__int128)total * p->n_q_heads <= INT32_MAX && total * (p->n_q_heads / p->n_kv_heads) <= INT32_MAX - 127;
}

// The shape fields of `a`, without the sequences.
void set_shape(const infllm_params* p, const infllm_pages* pages, const infllm_score_form* score, PagedArgs* a) {
  std::memset(a, 0, sizeof(*a));
  a->n_q_heads = p->n_q_heads;
  a->n_kv_heads = p->n_kv_heads;
  a->head_dim = p->head_dim;
  a->bf16 = p->dtype == INFLLM_BF16;
  a->sm_scale = p->sm_scale;
  if (score != nullptr) {
    a->softcap = score->softcap;
    a->window = score->window;
    a->n_init = score->n_init;
    a->slopes = score->slopes;
  }
  a->d_group = fast_div(p->n_q_heads / p->n_kv_heads);
  a->d_kv = fast_div(p->n_kv_heads);
  a->head_stride = pages->head_stride;
  a->page16 = (uint32_t)(pages->page_stride * esize(p) / 16);
  a->token16 = (uint32_t)(pages->token_stride * esize(p) / 16);
  a->n_pages = pages->n_pages;
  a->page_size = pages->page_size;
  a->d_page = fast_div(pages->page_size);
}

infllm_status check_score(const infllm_params* p, const infllm_score_form* s) {
  if (s == nullptr) return INFLLM_OK;
  if (!std::isfinite(s->softcap) || s->softcap < 0.f || s->window < 0 || s->n_init < 0) return INFLLM_E_SHAPE;
  if (s->softcap > 0.f && !std::isfinite(4.f * p->sm_scale / s->softcap)) return INFLLM_E_SHAPE;  // (the kernels form it)
  return (reinterpret_cast<uintptr_t>(s->slopes) & 3u) == 0 ? INFLLM_OK : INFLLM_E_SHAPE;
}

}  // namespace

extern "C" {

infllm_status infllm_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor,
                                      int64_t original_len, double slow, double fast, double* inv_freq) {
  if (rotary_dim < 0 || rotary_dim % 2 != 0) return INFLLM_E_SHAPE;
  if (!std::isfinite(base) || !(base > 0.0)) return INFLLM_E_SHAPE;
  if (scaling < INFLLM_ROPE_PLAIN || scaling > INFLLM_ROPE_PARTS) return INFLLM_E_SHAPE;
  if (scaling != INFLLM_ROPE_PLAIN && (!std::isfinite(factor) || !(factor > 0.0))) return INFLLM_E_SHAPE;
  if (scaling == INFLLM_ROPE_BASE && rotary_dim <= 2) return INFLLM_E_SHAPE;
  if (scaling == INFLLM_ROPE_PARTS && (original_len < 1 || !std::isfinite(slow) || !std::isfinite(fast) || !(slow < fast)))
    return INFLLM_E_SHAPE;
  if (rotary_dim == 0) return INFLLM_OK;
  if (inv_freq == nullptr) return INFLLM_E_NULL;
  const double r = rotary_dim, b = scaling == INFLLM_ROPE_BASE ? base * std::pow(factor, r / (r - 2.0)) : base;
  if (!std::isfinite(b) || !(b > 0.0)) return INFLLM_E_SHAPE;
  // (the largest frequency is the first or the last: no output is written where one passes float64)
  const double most = std::max(1.0, std::pow(b, -(r - 2.0) / r));
  if (!std::isfinite(scaling == INFLLM_ROPE_LINEAR || scaling == INFLLM_ROPE_PARTS ? most / std::min(1.0, factor) : most)) return INFLLM_E_SHAPE;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double theta = std::pow(b, -2.0 * i / r);
    if (scaling == INFLLM_ROPE_LINEAR) theta /= factor;
    if (scaling == INFLLM_ROPE_PARTS) {
      const double g = std::min(1.0, std::max(0.0, ((double)original_len * theta / kTwoPi - slow) / (fast - slow)));
      theta *= g + (1.0 - g) / factor;
    }
    inv_freq[i] = theta;
  }
  return INFLLM_OK;
}

infllm_status infllm_rotate(const infllm_params* p, const infllm_rotary* rot, int32_t n_tokens,
                            const int64_t* positions, int64_t first_position, const void* q, int64_t q_token_stride,
                            int64_t q_head_stride, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
                            const void* k, int64_t k_token_stride, int64_t k_head_stride, void* k_out,
                            int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream) {
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if (remap(p)) return INFLLM_E_UNSUPPORTED;
  if ((st = check_rotary(p, rot)) != INFLLM_OK) return st;
  if (n_tokens < 0) return INFLLM_E_SHAPE;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr)) return INFLLM_E_NULL;
  if (n_tokens == 0 || (q == nullptr && k == nullptr)) return INFLLM_OK;
  if ((reinterpret_cast<uintptr_t>(positions) & 7u) != 0) return INFLLM_E_SHAPE;
  if (q != nullptr) {
    if ((st = check_strided(p, q, q_token_stride, q_head_stride)) != INFLLM_OK) return st;
    if ((st = check_out(p, q_out, n_tokens, q_out_token_stride, p->n_q_heads, q_out_head_stride)) != INFLLM_OK) return st;
    if (!span_fits(p, n_tokens, q_token_stride, p->n_q_heads, q_head_stride) ||
        !span_fits(p, n_tokens, q_out_token_stride, p->n_q_heads, q_out_head_stride))
      return INFLLM_E_UNSUPPORTED;
  }
  if (k != nullptr) {
    if ((st = check_strided(p, k, k_token_stride, k_head_stride)) != INFLLM_OK) return st;
    if ((st = check_out(p, k_out, n_tokens, k_out_token_stride, p->n_kv_heads, k_out_head_stride)) != INFLLM_OK) return st;
    if (!span_fits(p, n_tokens, k_token_stride, p->n_kv_heads, k_head_stride) ||
        !span_fits(p, n_tokens, k_out_token_stride, p->n_kv_heads, k_out_head_stride))
      return INFLLM_E_UNSUPPORTED;
  }
  const int n_q = q != nullptr ? p->n_q_heads : 0, n_k = k != nullptr ? p->n_kv_heads : 0;
  if (!rotate_fits(n_tokens)) return INFLLM_E_UNSUPPORTED;
  if ((st = check_device()) != INFLLM_OK) return st;
  RotateArgs a;
  std::memset(&a, 0, sizeof(a));
  set_rotary(p, rot, &a);
  a.n_tokens = n_tokens;
  a.n_q = n_q;
  a.n_k = n_k;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_tok = q_token_stride;
  a.q_head = q_head_stride;
  a.kv_tok = k_token_stride;
  a.kv_head = k_head_stride;
  a.qo_tok = q_out_token_stride;
  a.qo_head = q_out_head_stride;
  a.ko_tok = k_out_token_stride;
  a.ko_head = k_out_head_stride;
  a.positions = positions;
  a.first_position = first_position;
  return launch_status(launch_rotate(a, (hipStream_t)stream));
}

infllm_status infllm_paged_append(const infllm_params* p, const infllm_rotary* rot, const infllm_pages* pages,
                                  int32_t n_seqs, const int32_t* seq_lens, const int64_t* past_lens,
                                  const int32_t* page_table, int64_t table_stride, const void* q,
                                  int64_t q_token_stride, int64_t q_head_stride, void* q_out,
                                  int64_t q_out_token_stride, int64_t q_out_head_stride, const void* k, const void* v,
                                  int64_t kv_token_stride, int64_t kv_head_stride, void* stream) {
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if (remap(p)) return INFLLM_E_UNSUPPORTED;
  if (rot != nullptr && (st = check_rotary(p, rot)) != INFLLM_OK) return st;
  if ((st = check_pages(p, pages)) != INFLLM_OK) return st;
  int64_t total;
  if ((st = check_seqs(pages, n_seqs, seq_lens, past_lens, table_stride, &total)) != INFLLM_OK) return st;
  if ((q == nullptr) != (q_out == nullptr)) return INFLLM_E_NULL;
  if (total == 0) return INFLLM_OK;
  if (page_table == nullptr) return INFLLM_E_NULL;
  if ((reinterpret_cast<uintptr_t>(page_table) & 3u) != 0) return INFLLM_E_SHAPE;
  if ((st = check_strided(p, k, kv_token_stride, kv_head_stride)) != INFLLM_OK) return st;
  if ((st = check_strided(p, v, kv_token_stride, kv_head_stride)) != INFLLM_OK) return st;
  if (!span_fits(p, total, kv_token_stride, p->n_kv_heads, kv_head_stride)) return INFLLM_E_UNSUPPORTED;
  if (q != nullptr) {
    if ((st = check_strided(p, q, q_token_stride, q_head_stride)) != INFLLM_OK) return st;
    if ((st = check_out(p, q_out, total, q_out_token_stride, p->n_q_heads, q_out_head_stride)) != INFLLM_OK) return st;
    if (!span_fits(p, total, q_token_stride, p->n_q_heads, q_head_stride) ||
        !span_fits(p, total, q_out_token_stride, p->n_q_heads, q_out_head_stride))
      return INFLLM_E_UNSUPPORTED;
  }
  const int n_q = q != nullptr ? p->n_q_heads : 0;
  if (!rotate_fits(total)) return INFLLM_E_UNSUPPORTED;
  if ((st = check_device()) != INFLLM_OK) return st;
  AppendPagesArgs a;
  std::memset(&a, 0, sizeof(a));
  set_rotary(p, rot, &a);
  a.n_q = n_q;
  a.n_k = a.n_v = p->n_kv_heads;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.k_out = pages->k;
  a.v_out = pages->v;
  a.q_tok = q_token_stride;
  a.q_head = q_head_stride;
  a.kv_tok = kv_token_stride;
  a.kv_head = kv_head_stride;
  a.qo_tok = q_out_token_stride;
  a.qo_head = q_out_head_stride;
  a.page_stride = pages->page_stride;
  a.ko_tok = pages->token_stride;
  a.ko_head = pages->head_stride;
  int64_t at = 0;
  for (int i = 0; i < n_seqs; i += kMaxPaged) {
    fill_seqs(pages, n_seqs, seq_lens, past_lens, page_table, table_stride, i, at, &a.seqs);
    a.first_token = (int)at;
    at = a.seqs.start[a.seqs.n_seqs];
    a.n_tokens = (int)at - a.first_token;
    if (a.n_tokens > 0 && (st = launch_status(launch_rotate(a, (hipStream_t)stream))) != INFLLM_OK) return st;
  }
  return INFLLM_OK;
}

size_t infllm_paged_workspace_bytes(const infllm_params* p, const infllm_pages* pages, int32_t n_seqs,
                                    const int32_t* seq_lens, const int64_t* past_lens, const infllm_score_form* score) {
  int64_t total;
  if (check_params(p) != INFLLM_OK || remap(p) || check_pages(p, pages) != INFLLM_OK || check_score(p, score) != INFLLM_OK ||
      check_seqs(pages, n_seqs, seq_lens, past_lens, INT32_MAX, &total) != INFLLM_OK || !numbers_fit(p, total))
    return 0;
  PagedArgs a;
  set_shape(p, pages, score, &a);
  size_t most = 0;
  int64_t at = 0;
  bool ok;
  for (int i = 0; plan(p, n_seqs, seq_lens, past_lens, &i, &at, &a, &ok);) {
    if (!ok) return 0;
    most = std::max(most, (size_t)partial_rows(a) * part_row_bytes(p));
  }
  return (most + 255) & ~(size_t)255;
}

infllm_status infllm_paged_attend(const infllm_params* p, const infllm_pages* pages, int32_t n_seqs,
                                  const int32_t* seq_lens, const int64_t* past_lens, const int32_t* page_table,
                                  int64_t table_stride, const infllm_score_form* score, const void* q,
                                  int64_t q_token_stride, int64_t q_head_stride, void* out, int64_t out_token_stride,
                                  int64_t out_head_stride, float* lse, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  infllm_status st;
  if ((st = check_params(p)) != INFLLM_OK) return st;
  if (remap(p)) return INFLLM_E_UNSUPPORTED;
  if ((st = check_pages(p, pages)) != INFLLM_OK) return st;
  if ((st = check_score(p, score)) != INFLLM_OK) return st;
  int64_t total;
  if ((st = check_seqs(pages, n_seqs, seq_lens, past_lens, table_stride, &total)) != INFLLM_OK) return st;
  if (total == 0) return INFLLM_OK;
  if (page_table == nullptr) return INFLLM_E_NULL;
  if ((reinterpret_cast<uintptr_t>(page_table) & 3u) != 0 || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return INFLLM_E_SHAPE;
  if ((st = check_strided(p, q, q_token_stride, q_head_stride)) != INFLLM_OK) return st;
  if ((st = check_out(p, out, total, out_token_stride, p->n_q_heads, out_head_stride)) != INFLLM_OK) return st;
  if (!span_fits(p, total, q_token_stride, p->n_q_heads, q_head_stride) ||
      !span_fits(p, total, out_token_stride, p->n_q_heads, out_head_stride))
    return INFLLM_E_UNSUPPORTED;
  if (!numbers_fit(p, total)) return INFLLM_E_UNSUPPORTED;
  // (keys are addressed by 16-byte pieces in 32 bits; the last number stands for no row)
  const __int128 span = (__int128)(pages->n_pages - 1) * pages->page_stride + (__int128)(pages->page_size - 1) * pages->token_stride;
  if (span * esize(p) / 16 >= 0xFFFFFFFFll - p->head_dim) return INFLLM_E_UNSUPPORTED;
  if (pages->page_size > 1 && pages->token_stride * esize(p) / 16 >= 1 << 24) return INFLLM_E_UNSUPPORTED;
  PagedArgs a;
  set_shape(p, pages, score, &a);
  a.q = q;
  a.k = pages->k;
  a.v = pages->v;
  a.out = out;
  a.lse = lse;
  a.q_tok = q_token_stride;
  a.q_head = q_head_stride;
  a.out_tok = out_token_stride;
  a.out_head = out_head_stride;
  a.lse_stride = total;
  a.table_stride = table_stride;
  // every launch is planned before the first is enqueued
  size_t need = 0;
  int64_t at = 0;
  int launches = 0;
  bool ok, planned = false;  // whether `a` holds the call's only launch
  a.table = page_table;
  for (int i = 0; plan(p, n_seqs, seq_lens, past_lens, &i, &at, &a, &ok); ++launches) {
    if (!ok) return INFLLM_E_UNSUPPORTED;
    need = std::max(need, (size_t)partial_rows(a) * part_row_bytes(p));
    if (i == n_seqs && launches == 0) {
      planned = true;
      ++launches;
      break;
    }
    a.table = page_table;
  }
  if (need > 0) {
    if (workspace == nullptr || workspace_bytes < need) return INFLLM_E_WORKSPACE;
    if (!aligned16(workspace)) return INFLLM_E_SHAPE;
  }
  if ((st = check_device()) != INFLLM_OK) return st;
  at = 0;
  for (int i = 0, l = 0; l < launches; ++l) {
    if (!planned) {
      a.table = page_table;
      plan(p, n_seqs, seq_lens, past_lens, &i, &at, &a, &ok);
    }
    if (a.items == 0) continue;
    const int64_t rows = partial_rows(a);
    if (rows > 0) partial_layout(p, workspace, 1, rows, &a.part_o, &a.part_lse, &a.part_exp);
    if ((st = launch_status(launch_paged(a, (hipStream_t)stream))) != INFLLM_OK) return st;
    if (rows > 0 && (st = launch_status(launch_paged_merge(a, (hipStream_t)stream))) != INFLLM_OK) return st;
  }
  return INFLLM_OK;
}

}  // extern "C"
