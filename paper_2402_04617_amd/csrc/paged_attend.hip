// Causal attention of new tokens over paged keys and values (infllm_paged_attend), bf16 on
// CDNA4 matrix cores (v_mfma_f32_32x32x16_bf16), fp32 accumulation.
//
//   O_i = sum_t softmax_t(z_it) v_t,  z_it = f(sm_scale q_i . k_t) - slope (p_i - t)
//
// over the visible keys t of the sequence, f the cap c tanh(x / c) or nothing.
//
// A workgroup has a row tile of 128 (query, head) rows of one kv head (four waves of 32)
// and a part of the key tiles that it sees; two workgroups share a compute unit.  Keys come
// in tiles of 64 through two LDS buffers of K and of V, loaded directly, each lane from an
// address of its own: the page of every group of 8 keys (of every key, where the page size
// is no multiple of 8) is looked up ahead into a table in LDS, as the place of the row in
// pieces of 16 bytes, which 32 bits hold up to 64 GiB of pages.
// Per wave and key tile, as in the step's attention: S^T = K Q^T with the keys from LDS and
// the query rows in registers, so that a lane has 16 scores of one row for each of two key
// blocks; P^T = exp2(z - m) is the B operand of O^T += V^T P^T as it stands, V^T read
// transposed.  Products of one tile run beside the exponentials of another.
//
// What bounds it: a long chunk the matrix cores at the clock that the power limit leaves
// (2,048 tokens after 64,000, 32 query heads of 128, 8 kv heads: 1.86 to 2.02 ms by card, 1.08
// to 1.17 PFLOP/s, 85 to 92 % of a library product of 8,192^3 on the same card; the matrix
// cores busy 68 % of the cycles, 5.2 vector instructions for each of theirs).  The cap adds
// an exponential and a reciprocal to a score (10.8 vector instructions for one matrix
// instruction) and makes the vector ALU the bound where the chip is full: 2,048 tokens after
// 30,000 take 1,165 us with it, 0.89 PFLOP/s, 919 without; with a bias (7.8) 888.  Batches of few
// row tiles are bound by how these fill the chip, which the host's model does not foresee for
// either form: 700, 1,500 and 64 tokens, capped, with a window of 4,096 107 to 114 us (the
// same tiles evenly spread: 81), 300, 800, 25 and two single ones with a bias 115 and 11 to 13 for the
// merge.  Single tokens beside chunks read their keys from memory while chunks have theirs in the
// caches: 512 and 300 new tokens and 30 single ones (613 MB) 164 us and 10.6 for the merge.  A few
// rows: see few_rows.
#include <type_traits>

#include "mfma_tile.h"
#include "paged.h"

namespace infllm {

namespace {

constexpr int kCap = 1, kSlopes = 2, kWideCap = 4;  // what scores become (see Scores; a cap is either kind)
constexpr int kTable = 1024;          // key groups whose places are in LDS
constexpr int kAhead = 3;             // a step looks up the tile that many ahead

// Places of the first rows of a window's key groups in pieces of 16 bytes (0, which is
// there, for a page that is not), and whether they are there, a bit each.
struct KeyTable {
  uint32_t place[kTable];
  uint64_t there[kTable / 64];
};

template <int D>
struct PagedSmem {
  bf16_t k[2][KB * D];
  bf16_t v[2][KB * D];
  KeyTable table;
  int bad[4];  // whether a wave met a page that is not there
};

// The kernel's arguments, read where they are used rather than held through the loop.
typedef const __attribute__((address_space(4))) PagedArgs LateArgs;
__device__ __forceinline__ LateArgs& late_args() {
  LateArgs* p = (LateArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *p;
}

// A sequence's row of the page table.
struct PageRow {
  const int32_t* table;
  FastDiv d_page;
  int page_size, n_pages;
  uint32_t page16, token16;
  // Place of a key in pieces of 16 bytes, given its page's entry x; kNoRow where that is not followed.
  __device__ __forceinline__ uint32_t place(int key, int x, int32_t page) const {
    const bool there = page >= 0 && page < n_pages;
    return there ? (uint32_t)page * page16 + (uint32_t)(key - x * page_size) * token16 : kNoRow;
  }
  __device__ __forceinline__ uint32_t place(int key) const {
    const int x = div_by(key, d_page);
    return place(key, x, table[x]);
  }
};
__device__ __forceinline__ PageRow page_row(int row) {
  LateArgs& a = late_args();
  return PageRow{a.table + row * a.table_stride, FastDiv{a.d_page.d, a.d_page.mul}, a.page_size, a.n_pages, a.page16, a.token16};
}

// The key tiles of a workgroup's part, in the order they are taken, and the table of their
// rows' places.  BACK: from the diagonal backwards.
template <int KT, int THREADS, bool BACK>
struct KeyTiles {
  int sink, shift;      // tile t < sink of the row tile's is at t * KT, others at (t + shift) * KT
  int t_begin, t_end;   // the part's
  int last;             // the sequence's last key
  int table_row;
  int gshift;           // keys of a table entry: 8, or 1
  int w0;               // first tile of the table's window
  __device__ __forceinline__ int key_of(int t) const {
    if (BACK) t = t_begin + t_end - 1 - t;
    return (t < sink ? t : t + shift) * KT;
  }
  // First key of the part's lowest tile.
  __device__ __forceinline__ int lowest() const { return key_of(BACK ? t_end - 1 : t_begin); }
  // The tiles [*a, *b) of all but the sink's, counted from key 0, in the order they are taken.
  __device__ __forceinline__ void range(int* a, int* b) const {
    const int x = max(*a - shift, t_begin), y = min(*b - shift, t_end);
    *a = BACK ? t_begin + t_end - y : x;
    *b = BACK ? t_begin + t_end - x : y;
  }
  __device__ __forceinline__ int tile_groups() const { return KT >> gshift; }
  __device__ __forceinline__ int window() const { return kTable / tile_groups(); }
  // Fills the table from tile `first` on; whether a page was not there.
  __device__ __forceinline__ bool fill(KeyTable& table, int first) {
    w0 = first;
    const PageRow pr = page_row(table_row);
    const int gmask = (1 << gshift) - 1, count = min(kTable, (t_end - first) * tile_groups());
    bool bad = false;
    for (int i = threadIdx.x; i - (int)(threadIdx.x & 63) < count; i += THREADS) {  // (whole waves)
      const int j = min(i, count - 1);
      const int key = min(key_of(first + (j << gshift) / KT) + ((j << gshift) & (KT - 1)), last & ~gmask);
      const uint32_t p = pr.place(key);
      table.place[i] = p == kNoRow ? 0u : p;
      const uint64_t there = __ballot(p != kNoRow);
      if ((i & 63) == 0) table.there[i >> 6] = there;
      bad |= p == kNoRow;
    }
    return bad;
  }
  // The same for the part's first window, and for the pages of the part behind it.
  __device__ __forceinline__ bool fill_first(KeyTable& table) {
    bool bad = fill(table, t_begin);
    if (t_begin + window() < t_end) {
      const PageRow pr = page_row(table_row);
      const int one = key_of(t_begin + window()), other = key_of(t_end - 1);
      const int from = div_by(min(one, other), pr.d_page);
      const int to = div_by(min(max(one, other) + KT - 1, last), pr.d_page);
      for (int x = from + (int)threadIdx.x; x <= to; x += THREADS) {
        const int32_t page = pr.table[x];
        bad |= page < 0 || page >= pr.n_pages;
      }
    }
    return bad;
  }
  // Which keys of tile t are there.
  __device__ __forceinline__ uint64_t there(const KeyTable& table, int t) const {
    const int i = (t - w0) * tile_groups() + (min((int)(threadIdx.x & 63), min(KT - 1, last - key_of(t))) >> gshift);
    return __ballot(((table.there[i >> 6] >> (i & 63)) & 1u) != 0);
  }
};

// What a row sees of a tile's keys from k0 on: a bit for each, the window and the initial
// tokens taken into account.
__device__ __forceinline__ uint64_t seen_keys(int pos, int k0, int window, int n_init) {
  auto below = [](int x) {  // the first x of 64 bits
    const int n = min(max(x, 0), 64);
    return n == 0 ? 0ull : ~0ull >> (64 - n);
  };
  uint64_t vis = below(pos - k0 + 1);
  if (window > 0) vis &= ~below(max(0, pos - window + 1) - k0) | below(n_init - k0);
  return vis;
}

// One row formed by its wave from the keys that it sees in the tiles [t_begin, t_end), for
// rows that a masked value which is not finite has reached: sum_t weight(q . k_t, t) v_t,
// DPL dims a lane.
template <typename T, int D, int KT, int THREADS, bool BACK, typename Weight>
__device__ __forceinline__ void form_row(const KeyTiles<KT, THREADS, BACK>& keys, const char* kbase, const char* vbase, const T* qp,
                                         int pos, int window, int n_init, Weight weight, float (&acc)[D / 64]) {
  constexpr int DPL = D / 64;
  const int lane = threadIdx.x & 63;
  const PageRow pr = page_row(keys.table_row);
#pragma unroll
  for (int e = 0; e < DPL; ++e) acc[e] = 0.f;
  for (int t = keys.t_begin; t < keys.t_end; ++t) {
    const int k0 = keys.key_of(t), key = k0 + lane;
    uint32_t at = kNoRow;
    if (lane < KT && ((seen_keys(pos, k0, window, n_init) >> lane) & 1u) != 0) at = pr.place(key);
    float p = 0.f;
    if (at != kNoRow) {
      const T* kp = (const T*)(kbase + (uint64_t)at * 16);
      float s = 0.f;
      for (int d = 0; d < D; ++d) s = __builtin_fmaf(Elem<T>::load(kp + d), Elem<T>::load(qp + d), s);
      p = weight(s, key);
    }
    for (uint64_t left = __ballot(at != kNoRow); left != 0; left &= left - 1) {
      const int j = __builtin_ctzll(left);
      const uint32_t aj = (uint32_t)__builtin_amdgcn_readlane((int)at, j);
      const float pj = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(p), j));
      const T* vp = (const T*)(vbase + (uint64_t)aj * 16) + DPL * lane;
#pragma unroll
      for (int e = 0; e < DPL; ++e) acc[e] = __builtin_fmaf(pj, Elem<T>::load(vp + e), acc[e]);
    }
  }
}

// Scores in the base-2 domain.  The scale, the cap and the bias are part of the
// exponential's argument: c tanh(x / c) = c - 2 c r with r = 1 / (1 + e^{2 x / c}), and a score
// to be capped becomes its r first (kCap).  That is off by some 2^-23 of c, 2^-20 at most, however
// small the score is, so it is for caps up to kMostFolded alone: 6e-5 there, thirty times less
// than rounding P to bf16 does.  Above (kWideCap) a score is capped by itself, off by its own
// roundings: x (1 - u^2 / 3 + 2 u^4 / 15 - 17 u^6 / 315), u = x / c, where |u| < 3 / 16 (the series'
// next term is 2^-25 there), else c (1 - 2 r).
constexpr float kMostFolded = 64.f;
template <int MOD>
struct Scores {
  float scale, cap_in, cap2, u_in, cap_s;
  static constexpr float kHidden = MOD & kCap ? __builtin_inff() : -__builtin_inff();  // what a hidden key's score becomes
  __device__ __forceinline__ explicit Scores(const PagedArgs& a)
      : scale(a.sm_scale * 1.4426950408889634f), cap_in(0.f), cap2(0.f), u_in(0.f), cap_s(0.f) {
    if constexpr (MOD & (kCap | kWideCap)) {
      cap_in = 2.f * scale / a.softcap;
      cap2 = a.softcap * 1.4426950408889634f;
    }
    if constexpr (MOD & kCap) scale = -2.f * cap2;
    if constexpr (MOD & kWideCap) {
      u_in = a.sm_scale / a.softcap;
      cap_s = a.softcap / a.sm_scale;
    }
  }
  static constexpr float kSeries = 0.1875f;
  __device__ __forceinline__ float series(float s) const {
    const float u = s * u_in, u2 = u * u;
    return s * __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(-17.f / 315.f, u2, 2.f / 15.f), u2, -1.f / 3.f), u2, 1.f);
  }
  __device__ __forceinline__ float saturated(float s) const {
    return __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + fast_exp2(s * cap_in)), 1.f) * cap_s;
  }
  __device__ __forceinline__ float form(float s) const {
    if constexpr (MOD & kCap) return __builtin_amdgcn_rcpf(1.f + fast_exp2(s * cap_in));
    if constexpr (MOD & kWideCap) return fabsf(s * u_in) < kSeries ? series(s) : saturated(s);
    return s;
  }
  // N scores: where the series does for all of the wave's, nothing else is formed (chunks of
  // 700, 1,500 and 64 tokens under a cap of 65: 107 to 110 us, folded 103 to 106; with scores up
  // to the cap 156, and 151 with both for every score).
  template <int N>
  __device__ __forceinline__ void form_all(float (&s)[N]) const {
    if constexpr (MOD & kWideCap) {
      float most = 0.f, x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        most = fmaxf(most, fabsf(s[i]));
        x[i] = series(s[i]);
      }
      if (__builtin_expect(__ballot(most * u_in >= kSeries) != 0, 0)) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = form(s[i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = x[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = form(s[i]);
    }
  }
  // What is added to every score: b, and the cap's own part.
  __device__ __forceinline__ float base(float b) const { return MOD & kCap ? b + cap2 : b; }
  __device__ __forceinline__ float exponent(float formed, float base) const { return __builtin_fmaf(formed, scale, base); }
};

// A head's slope in the base-2 domain, finite: times a distance of 0 it is 0.
__device__ __forceinline__ float slope_of(float slope) {
  return fminf(fmaxf(slope * 1.4426950408889634f, -3.402823466e38f), 3.402823466e38f);
}

// This wave's LDS accesses before it come before those after it.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// A part of a row tile of at most 16 rows (single tokens, a few guessed ones): the waves
// share the keys instead of the rows.  Wave w takes the 16 keys of every tile that it loads
// itself, so that the waves run without a barrier, each with its next two tiles' keys and
// values in flight, and join their shares in LDS at the end.  S^T = K Q^T with
// v_mfma_f32_16x16x32_bf16: a lane has keys 4 (lane / 16) .. + 3 of row lane % 16, which is
// the B operand of v_mfma_f32_16x16x16_bf16 as it stands; V^T read transposed.  Bound by
// memory: 48 sequences of up to 20,000 tokens (1.98 GB) take 338 us, 5.85 TB/s, and 346 with
// the merge.  One wave of four with all rows of the tile (of 32, four used) takes 351.5 there,
// 99.2 instead of 93.6 with a cap and a window of 4,096 keys, 13.8 instead of 13.2 for one
// sequence of 2,000.  Up to 32 rows this way (two blocks of them) were slower than the row
// tile's one wave: 32 sequences of 8 tokens after 4,000 100 and 97 us, 64 of one token with 32
// heads to a kv head 120 and 112, 4 of 5 tokens 23.8 and 20.6.
template <int D, int MOD, bool GROUPS>
__device__ __forceinline__ void few_rows(const PagedArgs& a, PagedSmem<D>& sm, const PagedWork& w, const PagedRange& range, int g, int i0,
                                         int i1) {
  constexpr int CH = D / 8, KSTEPS = D / 32, DBLK = D / 16;
  constexpr int RPI = 64 / CH, NI = 16 / RPI;
  constexpr uint32_t kTileBytes = KB * D * 2;
  typedef KeyTiles<KB, 256, (MOD & kSlopes) != 0> Keys;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, q4 = lane >> 4;
  const int G = (int)a.d_group.d, R = G * w.len;
  const int t_begin = w.part * w.part_tiles, t_end = min(t_begin + w.part_tiles, range.n);
  const bool one_part = range.n <= w.part_tiles;
  const int last = w.past + w.len - 1;
  const Keys keys{range.sink, range.low - range.sink, t_begin, t_end, last, w.table_row, GROUPS ? 3 : 0, t_begin};
  const PageRow pr = page_row(w.table_row);
  const char* kbase = (const char*)a.k + g * a.head_stride * 2;
  const char* vbase = (const char*)a.v + g * a.head_stride * 2;

  // Places of the wave's key groups (keys) of the next 32 (4) tiles, one a lane, and of the
  // 32 (4) after them, requested a window ahead.
  constexpr int kPer = GROUPS ? 2 : 16, kWindow = 64 / kPer;
  auto look_up = [&](int t0) -> uint32_t {
    const int t = min(t0 + lane / kPer, t_end - 1), first = keys.key_of(t) + 16 * wave;
    const int key = GROUPS ? min(first + 8 * (lane & 1), last & ~7) : min(first + (lane & 15), last);
    return pr.place(key);
  };
  uint32_t here = look_up(t_begin), ahead = 0;
  int w0 = t_begin;
  if (w0 + kWindow < t_end) ahead = look_up(w0 + kWindow);

  const int lrow = 16 * wave + lane / CH;
  const uint32_t piece0 = (uint32_t)(lane % CH) ^ (uint32_t)swz<D>(lrow);
  auto piece_of = [&](int j) { return D == 128 ? piece0 ^ (uint32_t)j : piece0; };
  uint32_t voff[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) voff[j] = 16u * (piece_of(j) + __umul24((uint32_t)(RPI * j + lane / CH) & 7u, a.token16));
  const uint32_t lds_k0 = (uint32_t)(uintptr_t)(INFLLM_LDS bf16_t*)sm.k[0];
  const uint32_t lds_v0 = (uint32_t)(uintptr_t)(INFLLM_LDS bf16_t*)sm.v[0];
  const uint32_t lds_k = lds_k0 + NI * wave * 1024, lds_v = lds_v0 + NI * wave * 1024;
  // which of the tile's keys are there: a bit for each of the wave's 16
  auto there_of = [&](uint32_t window, int t) -> uint32_t {
    const uint64_t ok = __ballot(window != kNoRow) >> (kPer * (t - w0));
    if constexpr (GROUPS) return ((ok & 1) ? 0xFFu : 0u) | ((ok & 2) ? 0xFF00u : 0u);
    return (uint32_t)ok & 0xFFFFu;
  };
  // Requests the wave's rows of tile t, which the window holds.
  auto issue = [&](int t) {
    const uint32_t buf = (uint32_t)((t - t_begin) & 1) * kTileBytes;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the buffer has been read)
    if constexpr (GROUPS) {
      uint64_t base[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)here, 2 * (t - w0) + i);
        base[i] = (uint64_t)(p == kNoRow ? 0u : p) << 4;
      }
#pragma unroll
      for (int j = 0; j < NI; ++j) lds_load(lds_k + buf + j * 1024, kbase + base[RPI * j / 8], voff[j]);
#pragma unroll
      for (int j = 0; j < NI; ++j) lds_load(lds_v + buf + j * 1024, vbase + base[RPI * j / 8], voff[j]);
    } else {
      uint64_t off[NI];
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const uint32_t p = __shfl(here, 16 * (t - w0) + RPI * j + lane / CH);
        off[j] = (uint64_t)((p == kNoRow ? 0u : p) + piece_of(j)) * 16;
      }
#pragma unroll
      for (int j = 0; j < NI; ++j) lds_load_lane(lds_k + buf + j * 1024, kbase + off[j]);
#pragma unroll
      for (int j = 0; j < NI; ++j) lds_load_lane(lds_v + buf + j * 1024, vbase + off[j]);
    }
  };
  issue(t_begin);
  uint32_t ok0 = there_of(here, t_begin), ok1 = 0xFFFFu;
  if (t_begin + 1 < t_end) {
    issue(t_begin + 1);
    ok1 = there_of(here, t_begin + 1);
  }

  const int row = min(c, R - 1), qi = div_by(row, a.d_group), qh = g * G + row - qi * G, pos = w.past + qi;
  bf16x8 qreg[KSTEPS];
  {
    const bf16_t* qp = (const bf16_t*)a.q + (int64_t)(w.start + qi) * a.q_tok + (int64_t)qh * a.q_head + 8 * q4;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) qreg[s] = *(const bf16x8*)(qp + 32 * s);
  }
  float slope = 0.f, m = -__builtin_inff(), neg_m = 0.f, l = 0.f;
  if constexpr (MOD & kSlopes) slope = slope_of(a.slopes[qh]);
  f32x4 o[DBLK];
#pragma unroll
  for (int db = 0; db < DBLK; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  const Scores<MOD> score(a);
  // LDS offsets of the fragments, XOR-related under the swizzle: K, k-step s: ^ 64 s; V^T,
  // block db: ^ 32 db
  const int kr = 16 * wave + c, vr = 16 * wave + 4 * q4 + (c >> 2);
  const uint32_t koff = 2u * D * kr + 16u * (q4 ^ swz<D>(kr));
  const uint32_t voff0 = 2u * D * vr + 16u * (((lane & 3) >> 1) ^ swz<D>(vr)) + 8u * (lane & 1);
  int plain0 = a.window > 0 ? (max(0, w.past + i1 - a.window + 1) + KB - 1) / KB : 0;
  int plain1 = (w.past + i0 + 1) / KB;
  keys.range(&plain0, &plain1);

  for (int t = t_begin; t < t_end; ++t) {
    const uint32_t buf = (uint32_t)((t - t_begin) & 1) * kTileBytes;
    const bool more = t + 1 < t_end;
    if (more) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(3 * NI) : "memory");  // this tile's keys have landed
    else asm volatile("s_waitcnt vmcnt(%0)" : : "n"(NI) : "memory");
    f32x4 s;
    const uint32_t ka = lds_k0 + buf + koff;
#pragma unroll
    for (int k = 0; k < KSTEPS; ++k) {
      const bf16x8 kf = *(const INFLLM_LDS bf16x8*)(uintptr_t)(ka ^ (64u * k));
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qreg[k], k == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s, 0, 0, 0);
    }
    const int k0 = keys.key_of(t) + 16 * wave;
    const bool plain = t >= plain0 && t < plain1 && ok0 == 0xFFFFu;
    if constexpr (MOD & (kCap | kWideCap)) {
      float x[4] = {s[0], s[1], s[2], s[3]};
      score.form_all(x);
      s = f32x4{x[0], x[1], x[2], x[3]};
    }
    if (!plain) {
      const uint32_t see = ((uint32_t)seen_keys(pos, k0, a.window, a.n_init) & ok0) >> (4 * q4);
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = (see >> j) & 1u ? s[j] : Scores<MOD>::kHidden;
    }
    const float distance = (float)(k0 + 4 * q4 - pos), base = score.base(0.f);
    float e[4], sum;
    auto exponent = [&](int j, float more) {
      if constexpr (MOD & kSlopes) return score.exponent(s[j], __builtin_fmaf(slope, fminf(distance + (float)j, 0.f), base)) + more;
      return score.exponent(s[j], base + more);
    };
    auto weights = [&]() {
#pragma unroll
      for (int j = 0; j < 4; ++j) e[j] = fast_exp2(exponent(j, neg_m));
      sum = (e[0] + e[1]) + (e[2] + e[3]);
    };
    weights();
    // the running maximum, raised only where a sum passes 2^16 or nothing has been seen yet
    if (__ballot(m == -__builtin_inff() || sum > 65536.f) != 0) {
      float mx = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 4; ++j) mx = fmaxf(mx, exponent(j, 0.f));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32)));
      const float alpha = mx == -__builtin_inff() ? 1.f : fast_exp2(m - mx);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DBLK; ++db) o[db] *= alpha;
      m = mx;
      neg_m = mx == -__builtin_inff() ? 0.f : -mx;
      weights();
    }
    l += sum;
    bf16x4 pb;
#pragma unroll
    for (int j = 0; j < 4; ++j) pb[j] = (__bf16)e[j];  // (by at most 2^-8 of each; the sums take them unrounded)
    const i16x4 p = __builtin_bit_cast(i16x4, pb);
    if (more) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * NI) : "memory");  // its values
    else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    const uint32_t va = lds_v0 + buf + voff0;
    if (GROUPS && k0 + 15 > last) {
      // rows behind the sequence's end: whatever the page holds meets weights of 0
      for (int i = max(0, last - k0 + 1) * CH + lane; i < 16 * CH; i += 64)
        *(INFLLM_LDS u32x4*)(uintptr_t)(lds_v0 + buf + 16 * wave * 2 * D + 16u * i) = u32x4{0, 0, 0, 0};
      wave_lds_order();
    }
#pragma unroll
    for (int db = 0; db < DBLK; ++db) {
      const i16x4 vf = __builtin_amdgcn_ds_read_tr16_b64_v4i16((INFLLM_LDS i16x4*)(uintptr_t)(va ^ (32u * db)));
      o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf, p, o[db], 0, 0, 0);
    }
    ok0 = ok1;
    if (t + 2 < t_end) {
      if (t + 2 >= w0 + kWindow) {
        here = ahead;
        w0 += kWindow;
        if (w0 + kWindow < t_end) ahead = look_up(w0 + kWindow);
      }
      issue(t + 2);
      ok1 = there_of(here, t + 2);
    }
  }

  // The waves' shares through LDS: [wave][row] of D values (padded), then maxima and sums.
  constexpr int kRow = D * 4 + 16, kRows = 16;
  static_assert(4 * kRows * (kRow + 8) <= (int)sizeof(sm), "the shares fit");
  INFLLM_LDS char* share = (INFLLM_LDS char*)(INFLLM_LDS PagedSmem<D>*)&sm;
  INFLLM_LDS float* stats = (INFLLM_LDS float*)(share + 4 * kRows * kRow);  // [wave][row]{m, l}
  lds_barrier();  // every wave is done with its tiles (its loads have landed)
#pragma unroll
  for (int db = 0; db < DBLK; ++db)
    *(INFLLM_LDS f32x4*)(share + (wave * kRows + c) * kRow + 4 * (16 * db + 4 * q4)) = o[db];
  {
    float sum = l;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (q4 == 0) {
      stats[2 * (wave * kRows + c)] = m;
      stats[2 * (wave * kRows + c) + 1] = sum;
    }
  }
  lds_barrier();
  constexpr int TPR = D / 8;  // threads of a row
  static_assert(256 / TPR >= kRows, "all rows at once");
  const int64_t prow0 = (int64_t)blockIdx.x * a.item_rows;
  const int r = tid / TPR, d = 8 * (tid % TPR);
  if ((tid & ~63) / TPR >= R) return;  // (whole waves)
  const int rc = min(r, kRows - 1);
  float M = -__builtin_inff(), L = 0.f, acc[8] = {};
#pragma unroll
  for (int v = 0; v < 4; ++v) M = fmaxf(M, stats[2 * (v * kRows + rc)]);
  const float base = M == -__builtin_inff() ? 0.f : M;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float mv = stats[2 * (v * kRows + rc)], lv = stats[2 * (v * kRows + rc) + 1];
    const float f = mv == -__builtin_inff() ? 0.f : fast_exp2(mv - base);
    const bool live = mv != -__builtin_inff() || lv != lv;
    L += live ? lv * (lv != lv ? 1.f : f) : 0.f;
    const INFLLM_LDS f32x4* x = (const INFLLM_LDS f32x4*)(share + (v * kRows + rc) * kRow + 4 * d);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += live ? f * x[e >> 2][e & 3] : 0.f;
  }
  const bool row_ok = r < R && r < kRows;
  const int i = div_by(min(r, R - 1), a.d_group), h = g * G + min(r, R - 1) - i * G;
  float inv = L > 0.f ? 1.f / L : 0.f;
  float lse_v = L > 0.f ? (M + __log2f(L)) * 0.6931471805599453f : -__builtin_inff();
  if (L != L) {  // a NaN among the row's scores is the row's, through the merge as well
    inv = L;
    lse_v = one_part ? L : __builtin_inff();
  }
  float z = 0.f, amax = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    z = __builtin_fmaf(acc[e], 0.f, z);
    acc[e] *= inv;
    amax = fmaxf(amax, fabsf(acc[e]));
  }
#pragma unroll
  for (int x = 1; x < TPR; x <<= 1) {
    z += __shfl_xor(z, x);
    amax = fmaxf(amax, __shfl_xor(amax, x));
  }
  // A row that a masked value which is not finite has reached (0 times it) is formed again
  // by the wave from the keys that it sees.
  const bool apart = row_ok && !(z == 0.f) && L == L;
  uint64_t odd = __ballot(apart && tid % TPR == 0);
  const int ex = one_part ? 0 : partial_row_exponent(amax);
  if (row_ok && !apart) {
    const float sc = exp2_int(-ex);
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[e] = one_part ? (uint32_t)f32_to_bf16(acc[2 * e]) | ((uint32_t)f32_to_bf16(acc[2 * e + 1]) << 16)
                      : pack_f16x2(acc[2 * e] * sc, acc[2 * e + 1] * sc);
    if (!one_part) *(u32x4*)((char*)a.part_o + (prow0 + r) * (D * 2) + 2 * d) = x;
    else *(u32x4*)((bf16_t*)a.out + (int64_t)(w.start + i) * a.out_tok + (int64_t)h * a.out_head + d) = x;
    if (d == 0 && !one_part) a.part_exp[prow0 + r] = ex;
  }
  if (row_ok && d == 0) {
    if (!one_part) a.part_lse[prow0 + r] = lse_v;
    else if (a.lse != nullptr) a.lse[h * a.lse_stride + w.start + i] = lse_v;
  }
  for (; odd != 0; odd &= odd - 1) {
    const int src = __builtin_ctzll(odd), rr = __shfl(r, src), p_r = w.past + __shfl(i, src);
    const float nm = -__shfl(base, src), inv_r = __shfl(inv, src);
    const int hr = __shfl(h, src);
    const bf16_t* qp = (const bf16_t*)a.q + (int64_t)(p_r - w.past + w.start) * a.q_tok + (int64_t)hr * a.q_head;
    float slope_r = 0.f;
    if constexpr (MOD & kSlopes) slope_r = slope_of(a.slopes[hr]);
    constexpr int DPL = D / 64;
    float again[DPL], top = 0.f;
    form_row<bf16_t, D>(keys, kbase, vbase, qp, p_r, a.window, a.n_init, [&](float x, int key) {
      return fast_exp2(score.exponent(score.form(x), score.base(slope_r * (float)(key - p_r))) + nm);
    }, again);
#pragma unroll
    for (int e = 0; e < DPL; ++e) {
      again[e] *= inv_r;
      const float x = fabsf(again[e]);
      top = x < __builtin_inff() ? fmaxf(top, x) : top;  // (of the finite ones, which keep their precision)
    }
    const int ex_r = one_part ? 0 : partial_row_exponent(wave_max(top));
    uint16_t* to = one_part ? (uint16_t*)a.out + (int64_t)(p_r - w.past + w.start) * a.out_tok + (int64_t)hr * a.out_head
                            : (uint16_t*)a.part_o + (prow0 + rr) * D;
#pragma unroll
    for (int e = 0; e < DPL; ++e)
      to[DPL * lane + e] = one_part ? f32_to_bf16(again[e]) : (uint16_t)(pack_f16x2(again[e] * exp2_int(-ex_r), 0.f) & 0xFFFFu);
    if (!one_part && lane == 0) a.part_exp[prow0 + rr] = ex_r;
  }
}

// GROUPS: pages of a multiple of 8 tokens.  The rows of a load instruction then lie in one
// group of 8 keys, whose place is uniform: its base goes through scalar registers, and a
// lane's offset from it is the same for every tile.  (With an address formed by every lane
// for every load the loop had 6.4 vector instructions for a matrix instruction instead of
// 5.)  Rows of the last group behind the sequence's end are loaded with it, whatever the
// page holds there, and those values are cleared in LDS.
template <int D, int MOD, bool GROUPS>
__global__ void __launch_bounds__(256, 2) paged_mfma_kernel(PagedArgs a) {
  constexpr int CH = D / 8;                       // 16-byte pieces of a row
  constexpr int KSTEPS = D / 16, DBLK = D / 32;
  constexpr int RPI = 64 / CH;                    // tile rows per load instruction
  constexpr int NI = KB * D * 2 / (4 * 1024);     // load instructions per wave and tile (K or V)
  constexpr uint32_t kTileBytes = KB * D * 2;
  __shared__ __attribute__((aligned(256))) PagedSmem<D> sm;
  static_assert(sizeof(sm) <= 80 * 1024, "two workgroups share a compute unit's LDS");

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, gsel = lane >> 5;
  const int G = (int)a.d_group.d;
  // the kv heads side by side (8 of them: one per XCD, whose L2 then holds its keys)
  const int item = div_by(blockIdx.x, a.d_kv), g = (int)blockIdx.x - item * (int)a.d_kv.d;
  const PagedWork w = paged_work(a, item);
  const int R = G * w.len, tile0 = w.rt * 128;
  const int i0 = div_by(tile0, a.d_group), i1 = div_by(min(R, tile0 + 128) - 1, a.d_group);
  const PagedRange range = paged_range(a, w.past, i0, i1);
  const int t_begin = w.part * w.part_tiles, t_end = min(t_begin + w.part_tiles, range.n);
  if (t_begin >= t_end) return;  // (the parts of a sequence are as many for each of its row tiles)
  if (R <= 16) {
    few_rows<D, MOD, GROUPS>(a, sm, w, range, g, i0, i1);
    return;
  }
  const bool one_part = range.n <= w.part_tiles;
  const int last = w.past + w.len - 1;
  KeyTiles<KB, 256, (MOD & kSlopes) != 0> keys{range.sink, range.low - range.sink, t_begin, t_end, last, w.table_row, GROUPS ? 3 : 0, t_begin};
  auto key_of = [&](int t) { return keys.key_of(t); };  // first key of tile t

  const int row0 = tile0 + wave * 32, row = row0 + n;
  const bool active = row0 < R;  // a wave without rows loads its share of the tiles
  const int row_c = min(row, R - 1);
  const int qi = div_by(row_c, a.d_group), qh = g * G + row_c - qi * G;
  const int pos = w.past + qi;

  const char* kbase = (const char*)a.k + g * a.head_stride * 2;
  const char* vbase = (const char*)a.v + g * a.head_stride * 2;
  // Load instruction j of wave w fills pieces [(NI*w + j)*64, +64) of a tile: rows lrow +
  // RPI*j; a lane's slot holds piece (lane % CH) ^ swz(row) of its row.
  const int lrow = KB / 4 * wave + lane / CH;
  // (swz(lrow + RPI * j) is swz(lrow) ^ j at D = 128, swz(lrow) at D = 64)
  const uint32_t piece0 = (uint32_t)(lane % CH) ^ (uint32_t)swz<D>(lrow);
  auto piece_of = [&](int j) { return D == 128 ? piece0 ^ (uint32_t)j : piece0; };
  const uint32_t lds_k0 = (uint32_t)(uintptr_t)(INFLLM_LDS bf16_t*)sm.k[0];
  const uint32_t lds_v0 = (uint32_t)(uintptr_t)(INFLLM_LDS bf16_t*)sm.v[0];
  const uint32_t lds_k = lds_k0 + NI * wave * 1024, lds_v = lds_v0 + NI * wave * 1024;
  // Places of a tile's rows: of the wave's two groups, or of the row of each load.
  constexpr int NP = GROUPS ? 2 : NI;
  struct Places {
    uint32_t o[NP];
  };
  uint32_t voff[NI];  // bytes from a group's place to this lane's piece
#pragma unroll
  for (int j = 0; j < NI; ++j) voff[j] = 16u * (piece_of(j) + __umul24((uint32_t)(RPI * j + lane / CH) & 7u, a.token16));
  auto load = [&](uint32_t lds, const char* base, const Places& f, int j) {
    if constexpr (GROUPS) lds_load(lds, base + ((uint64_t)f.o[RPI * j / 8] << 4), voff[j]);
    else lds_load_lane(lds, base + (uint64_t)(f.o[j] + piece_of(j)) * 16);
  };
  auto load_k = [&](int buf, const Places& f, int j) { load(lds_k + buf * kTileBytes + j * 1024, kbase, f, j); };
  auto load_v = [&](int buf, const Places& f, int j) { load(lds_v + buf * kTileBytes + j * 1024, vbase, f, j); };

  // The first tile's pages, the table's, and the query rows are requested at once.
  Places f0;
  {
    const PageRow pr = page_row(w.table_row);
    int key[NP], x[NP], page[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      key[j] = GROUPS ? min(key_of(t_begin) + KB / 4 * wave + 8 * j, last & ~7) : min(key_of(t_begin) + lrow + RPI * j, last);
      x[j] = div_by(key[j], pr.d_page);
      page[j] = pr.table[x[j]];
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const uint32_t p = pr.place(key[j], x[j], page[j]);
      f0.o[j] = p == kNoRow ? 0u : p;  // (a row that is not there: page 0's, masked)
      if constexpr (GROUPS) f0.o[j] = (uint32_t)__builtin_amdgcn_readfirstlane((int)f0.o[j]);
    }
  }
  bf16x8 qreg[KSTEPS];
  if (active) {
    const bf16_t* qp = (const bf16_t*)a.q + (int64_t)(w.start + qi) * a.q_tok + (int64_t)qh * a.q_head + 8 * gsel;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) qreg[s] = *(const bf16x8*)(qp + 16 * s);
  }
  float slope = 0.f;
  if constexpr (MOD & kSlopes) slope = slope_of(a.slopes[qh]);

  const bool bad = keys.fill_first(sm.table);
#pragma unroll
  for (int j = 0; j < NI; ++j) load_k(0, f0, j);
#pragma unroll
  for (int j = 0; j < NI; ++j) load_v(0, f0, j);
  {
    const bool any = __ballot(bad) != 0;
    if (lane == 0) sm.bad[wave] = any;
  }
  lds_barrier();
  // (A page that is not there, seen by a row or not, has every tile of the part masked.  A window
  // whose pages between it and the initial tokens are freed comes to that where a tile holds both
  // kinds: 2,048 tokens after 30,000, window 4,096, 152 us with pages of 16 and 100 initial tokens, 137
  // where all are there; 139 either way with pages of 64 and 128.)
  const bool has_bad = (sm.bad[0] | sm.bad[1] | sm.bad[2] | sm.bad[3]) != 0;

  // Places of the wave's rows of tile t (past the part's end: of its last tile again,
  // whose keys come from the cache and are not used).
  const uint32_t lds_rows = (uint32_t)(uintptr_t)(INFLLM_LDS uint32_t*)sm.table.place;
  struct Entries {
    uint32_t e[NP];
  };
  auto read_entries = [&](int t, Entries& en) {
    const uint32_t at = lds_rows + 4u * (uint32_t)((min(t, t_end - 1) - keys.w0) * keys.tile_groups());
    if constexpr (GROUPS) {
      const u32x2 x = *(const INFLLM_LDS u32x2*)(uintptr_t)(at + 8u * wave);
      en.e[0] = x[0];
      en.e[1] = x[1];
    } else {
#pragma unroll
      for (int j = 0; j < NP; ++j) en.e[j] = *(const INFLLM_LDS uint32_t*)(uintptr_t)(at + 4u * (uint32_t)(lrow + RPI * j));
    }
  };
  auto to_places = [&](const Entries& en, Places& f) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      if constexpr (GROUPS) f.o[j] = (uint32_t)__builtin_amdgcn_readfirstlane((int)en.e[j]);
      else f.o[j] = opaque_v(en.e[j]);
    }
  };
  auto places = [&](int t, Places& f) {
    Entries en;
    read_entries(t, en);
    to_places(en, f);
  };

  // LDS offsets of the fragments; under the swizzle they are XOR-related (see attend_mfma).
  constexpr uint32_t VX = D == 128 ? 32 : 0;
  const uint32_t koff0 = 2u * tile_off<D>(n, gsel);
  uint32_t voff0;
  {
    const int h = lane >> 4, q = (lane & 15) >> 2, m = lane & 3;
    const int vr = 4 * (h >> 1) + q, d0 = 16 * (h & 1) + 4 * m;
    voff0 = 2u * (tile_off<D>(vr, d0 >> 3) + (d0 & 7));
  }
  auto kfrag_at = [&](uint32_t kaddr, int kb, int s) {
    return *(const INFLLM_LDS bf16x8*)(uintptr_t)((kaddr ^ (32u * s)) + kb * 64u * D);
  };
  auto vfrag_at = [&](uint32_t vaddr, int db, int j) {
    const uint32_t a0 = (vaddr ^ (64u * db)) + j * 32u * D;
    const uint32_t a1 = ((vaddr ^ (64u * db) ^ VX) + 16u * D) + j * 32u * D;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((INFLLM_LDS i16x4*)(uintptr_t)a0);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((INFLLM_LDS i16x4*)(uintptr_t)a1);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto kaddr_of = [&](int buf) { return opaque_s(lds_k0 + buf * kTileBytes) + koff0; };
  auto vaddr_of = [&](int buf) { return opaque_s(lds_v0 + buf * kTileBytes) + voff0; };

  f32x16 oacc[DBLK];
#pragma unroll
  for (int db = 0; db < DBLK; ++db)
#pragma unroll
    for (int j = 0; j < 16; ++j) oacc[db][j] = 0.f;
  float m_run = -__builtin_inff(), neg_m = 0.f, l_run = 0.f;

  // With a bias the tiles are taken from the diagonal backwards, where it falls (forwards,
  // the maximum of a steep one grew with every tile).
  const Scores<MOD> score(a);
  // Key place c of a tile (element e = 16 kb + j of a lane: 32 kb + 8 (j / 4) + j % 4, its
  // half's 4 gsel aside).
  auto place_of = [](int e) { return 32 * (e >> 4) + 8 * ((e & 15) >> 2) + (e & 3); };
  // What a score is given besides its scale.  NEAR, with a bias: each key's own bias from its
  // distance (0 for keys behind the query, whose bias must not grow), the maximum taken off the
  // rounded score, so that a score is off by its own rounding, whatever the slope, and none
  // passes a maximum formed alike.  Else from the bias of this half's first key, with
  // the maximum taken off that (two instructions a score, not five): off by at most twice a score's own
  // rounding where every key of the tile is 64 and more away.
  struct Bias {
    float b, distance, more;
  };
  auto bias_of = [&](int t, auto near, float more) {
    Bias x{score.base(more), 0.f, more};
    if constexpr (MOD & kSlopes) {
      x.distance = (float)(key_of(t) + 4 * gsel - (int)opaque_v((uint32_t)pos));  // (the 32 sums of two tiles' places would not fit)
      if constexpr (!decltype(near)::value) x.b = score.base(slope * x.distance) + more;
    }
    return x;
  };
  // The exponent of element e of a tile.
  auto exponent = [&](float s, int e, const Bias& x, auto near) {
    if constexpr ((MOD & kSlopes) == 0) return score.exponent(s, x.b);
    else if constexpr (decltype(near)::value)
      return score.exponent(s, __builtin_fmaf(slope, fminf(x.distance + (float)place_of(e), 0.f), score.base(0.f))) + x.more;
    else return score.exponent(s, __builtin_fmaf(slope, (float)place_of(e), x.b));
  };
  // What a row sees of a tile: a bit for each key of this lane's half from its first on.
  struct Lims {
    uint32_t vis[2];
  };
  auto lims_of = [&](int t, bool masked) {
    Lims l{};
    const int k0 = key_of(t);
    if (masked) {
      uint64_t vis = seen_keys(pos, k0, a.window, a.n_init);
      if (has_bad) vis &= keys.there(sm.table, t);
      vis >>= 4 * gsel;
      l.vis[0] = (uint32_t)vis;
      l.vis[1] = (uint32_t)(vis >> 32);
    }
    return l;
  };
  // Elements [8i, 8i + 8) of a tile's scores: formed, and hidden where the row does not see the key.
  auto form8 = [&](f32x16 (&s)[2], int i, const Lims& l, bool masked) {
    float x[8];
#pragma unroll
    for (int e = 8 * i; e < 8 * i + 8; ++e) x[e - 8 * i] = s[e >> 4][e & 15];
    score.form_all(x);
#pragma unroll
    for (int e = 8 * i; e < 8 * i + 8; ++e) {
      const int c = place_of(e);
      float z = x[e - 8 * i];
      if (masked) {
        const uint32_t see = (uint32_t)((int32_t)(l.vis[e >> 4] << (31 - (c & 31))) >> 31);  // all ones or none
        z = __uint_as_float((__float_as_uint(z) & see) | (__builtin_bit_cast(uint32_t, Scores<MOD>::kHidden) & ~see));
      }
      s[e >> 4][e & 15] = z;
    }
  };
  auto tile_max = [&](const f32x16 (&s)[2], int t) {
    float mx = Scores<MOD>::kHidden;
    const std::true_type near;
    const Bias b = bias_of(t, near, 0.f);
    if constexpr (MOD & kSlopes) {
      mx = -__builtin_inff();
#pragma unroll
      for (int e = 0; e < 32; ++e) mx = fmaxf(mx, exponent(s[e >> 4][e & 15], e, b, near));
    } else {
#pragma unroll
      for (int e = 0; e < 32; ++e) mx = MOD & kCap ? fminf(mx, s[e >> 4][e & 15]) : fmaxf(mx, s[e >> 4][e & 15]);
      mx = score.exponent(mx, b.b);
    }
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
  };
  // Lazy running maximum, as in the step's attention: a tile's P is formed against the
  // maximum so far, and only where a row's sum of P passes 2^16 (or it has met no visible
  // key yet) is the tile's own maximum taken and the row rescaled.
  constexpr float kLazy = 65536.f;
  float bound = 0.f;
  auto set_max = [&](float mx) {
    m_run = mx;
    neg_m = mx == -__builtin_inff() ? 0.f : -mx;
    // (a row that sees none of the part's keys: its P are 0)
    bound = mx != -__builtin_inff() ? kLazy : (int)opaque_v((uint32_t)pos) < keys.lowest() ? 0.f : -1.f;
  };
  auto outgrown = [&](float l_tile, const f32x16 (&s)[2], int t) -> bool {
    if (__ballot(l_tile > bound) == 0) return false;
    const float mx = tile_max(s, t);
    if (__ballot(bound < 0.f ? mx != -__builtin_inff() : l_tile > bound) == 0) return false;
    const float m_new = fmaxf(m_run, mx);
    const float alpha = m_new == -__builtin_inff() ? 1.f : fast_exp2(m_run - m_new);
    l_run *= alpha;
#pragma unroll
    for (int db = 0; db < DBLK; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) oacc[db][j] *= alpha;
    set_max(m_new);
    return true;
  };
  // Two weights as a bf16 pair; the row sums add them unrounded.  (Rounded by at most 2^-8
  // of each: the instruction takes bf16 weights with bf16 values.)
  auto p_pair = [&](float z0, float z1, int e, const Bias& b, auto near, float (&acc)[2], bool first) -> uint32_t {
    const float e0 = fast_exp2(exponent(z0, e, b, near)), e1 = fast_exp2(exponent(z1, e + 1, b, near));
    acc[0] = first ? e0 : acc[0] + e0;
    acc[1] = first ? e1 : acc[1] + e1;
    bf16x2 pr;
    pr[0] = (__bf16)e0;
    pr[1] = (__bf16)e1;
    return opaque_v(__builtin_bit_cast(uint32_t, pr));
  };
  auto half_p = [&](const f32x16 (&s)[2], int h, int t, u32x4 (&p)[2]) {
    float ps[2];
    const std::true_type near;
    const Bias b = bias_of(t, near, neg_m);
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i >> 2][i & 3] = p_pair(s[h][2 * i], s[h][2 * i + 1], 16 * h + 2 * i, b, near, ps, i == 0);
    return ps[0] + ps[1];
  };
  auto as_frag = [](const u32x4& x) { return __builtin_bit_cast(bf16x8, x); };

  // Tiles all of whose keys every row of the workgroup sees: [plain0, plain1).  With a bias those
  // among them whose keys are 64 positions and more before every row; what comes before plain0 is
  // near then, and so is tile plain0 as the current one of its step.
  int plain0 = a.window > 0 ? (max(0, w.past + i1 - a.window + 1) + KB - 1) / KB : 0;
  int plain1 = max(0, w.past + i0 + (MOD & kSlopes ? 1 - KB : 1)) / KB;
  if constexpr (MOD & kSlopes) {
    // (scores past 2^24, whose roundings pass 1: each is formed the near way, or the maximum could
    // lie so far from them that their exponentials overflow)
    if (__ballot(fabsf(slope) * (float)(pos - keys.lowest()) > 16777216.f) != 0) plain1 = 0;
  }
  keys.range(&plain0, &plain1);
  if constexpr (MOD & kSlopes) ++plain0;
  if (has_bad) plain1 = 0;  // (none; never past t_end, where the plain pairs would not stop)

  // Step of tile t: QK(t+1) beside the second half of P(t), then PV(t) beside the form, mask
  // and first half of P of tile t+1.  At its top K(t+1) and V(t) have landed; it requests
  // K(t+2) and V(t+1) into the buffers that the barrier freed.
  f32x16 sA[2], sB[2];
  u32x4 p0[2];
  float l_pend = 0.f;
  Places f1, f2;  // of tiles t+1 and t+2
  auto top = [&](int t) {
    __builtin_amdgcn_s_setprio(0);
    publish_barrier<0>();
    if (GROUPS && key_of(t) + KB - 1 > last) {
      // V rows behind the sequence's end: whatever the page holds meets weights of 0
      for (int i = (last - key_of(t) + 1) * CH + tid; i < KB * CH; i += 256)
        *(INFLLM_LDS u32x4*)(uintptr_t)(lds_v0 + ((t - t_begin) & 1) * kTileBytes + 16u * i) = u32x4{0, 0, 0, 0};
      lds_barrier();
    }
    // (the table's readers are past the barrier; it keeps tile t+1, whose mask may ask it)
    if (t + kAhead >= keys.w0 + keys.window() && t + kAhead < t_end) {
      keys.fill(sm.table, t + 1);
      publish_barrier<0>();
    }
    __builtin_amdgcn_s_setprio(1);
  };
  auto step = [&](int t, f32x16 (&cur)[2], f32x16 (&nxt)[2], auto next_masked, auto near) {
    constexpr bool MASK = decltype(next_masked)::value;
    const int bc = (t - t_begin) & 1, bn = bc ^ 1;
    u32x4 w1[2];
    float ps1[2];
    bf16x8 va[DBLK];
    const uint32_t vaddr = vaddr_of(bc);
    const Bias bc_m = bias_of(t, near, neg_m);
    {
      const uint32_t ka = kaddr_of(bn);
      bf16x8 a0[2], a1[2];
      a0[0] = kfrag_at(ka, 0, 0);
      a1[0] = kfrag_at(ka, 1, 0);
      constexpr int EPC = 16 / KSTEPS;
      static_assert(EPC % 2 == 0 && 2 * NI <= KSTEPS, "pairs, and one load per chunk");
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) {
        if (s + 1 < KSTEPS) {
          a0[(s + 1) & 1] = kfrag_at(ka, 0, s + 1);
          a1[(s + 1) & 1] = kfrag_at(ka, 1, s + 1);
        } else {
#pragma unroll
          for (int db = 0; db < DBLK; ++db) va[db] = vfrag_at(vaddr, db, 0);
        }
        if (s == 0) {
          const f32x16 zero = {};
          nxt[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a0[0], qreg[0], zero, 0, 0, 0);
          nxt[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a1[0], qreg[0], zero, 0, 0, 0);
        } else {
          nxt[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a0[s & 1], qreg[s], nxt[0], 0, 0, 0);
          nxt[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a1[s & 1], qreg[s], nxt[1], 0, 0, 0);
        }
        if (s < NI) load_k(bc, f2, s);
        else if (s < 2 * NI) load_v(bn, f1, s - NI);
#pragma unroll
        for (int i = 0; i < EPC; i += 2) {
          const int x = (EPC * s + i) >> 1;
          w1[x >> 2][x & 3] = p_pair(cur[1][2 * x], cur[1][2 * x + 1], 16 + 2 * x, bc_m, near, ps1, x == 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    float l_tile = l_pend + (ps1[0] + ps1[1]);
    if (outgrown(l_tile, cur, t)) {
      l_tile = half_p(cur, 0, t, p0);
      l_tile += half_p(cur, 1, t, w1);
    }
    l_run += l_tile;
    u32x4 q0[2];
    float ps0[2];
    {
      const Lims l = lims_of(t + 1, MASK);
      const Bias bn_m = bias_of(t + 1, near, neg_m);
      Entries en;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j == 0) {
          f1 = f2;
          read_entries(t + kAhead, en);
        } else if (j == 2) {
          to_places(en, f2);
        }
#pragma unroll
        for (int db = 0; db < DBLK; ++db) {
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[db], as_frag(j < 2 ? p0[j & 1] : w1[j & 1]), oacc[db], 0, 0, 0);
          if (j + 1 < 4) va[db] = vfrag_at(vaddr, db, j + 1);
        }
        form8(nxt, j, l, MASK);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int x = 2 * j + i;
          q0[x >> 2][x & 3] = p_pair(nxt[0][2 * x], nxt[0][2 * x + 1], 2 * x, bn_m, near, ps0, x == 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    p0[0] = q0[0];
    p0[1] = q0[1];
    l_pend = __uint_as_float(opaque_v(__float_as_uint(ps0[0] + ps0[1])));
  };
  places(t_begin + 1, f1);
  places(t_begin + 2, f2);
#pragma unroll
  for (int j = 0; j < NI; ++j) load_k(1, f1, j);
  // K(t0) and V(t0) have landed, K(t0 + 1) is in flight
  publish_barrier<NI>();
  if (!active) {
    int t = t_begin;
    for (; t + 1 < t_end; ++t) {
      top(t);
      const int bc = (t - t_begin) & 1;
#pragma unroll
      for (int j = 0; j < NI; ++j) load_k(bc, f2, j);
#pragma unroll
      for (int j = 0; j < NI; ++j) load_v(bc ^ 1, f1, j);
      f1 = f2;
      places(t + kAhead, f2);
    }
    top(t);
  } else {
    {
      const uint32_t ka = kaddr_of(0);
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) {
        const f32x16 zero = {};
        sA[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kfrag_at(ka, 0, s), qreg[s], s == 0 ? zero : sA[0], 0, 0, 0);
        sA[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kfrag_at(ka, 1, s), qreg[s], s == 0 ? zero : sA[1], 0, 0, 0);
      }
    }
    {
      const bool mk = t_begin < plain0 || t_begin >= plain1;
      const Lims l = lims_of(t_begin, mk);
#pragma unroll
      for (int i = 0; i < 4; ++i) form8(sA, i, l, mk);
    }
    set_max(tile_max(sA, t_begin));  // the first tile's maximum
    l_pend = half_p(sA, 0, t_begin, p0);
    int t = t_begin;
    // pairs whose next tiles need a mask (with a bias: or are near), plain pairs, pairs that need one again
    const std::true_type yes;
    const std::false_type no;
    for (; t + 2 < t_end && t + 1 < plain0; t += 2) {
      top(t);
      step(t, sA, sB, yes, yes);
      top(t + 1);
      step(t + 1, sB, sA, yes, yes);
    }
    for (; t + 2 < plain1; t += 2) {
      top(t);
      step(t, sA, sB, no, no);
      top(t + 1);
      step(t + 1, sB, sA, no, no);
    }
    for (; t + 2 < t_end; t += 2) {
      top(t);
      step(t, sA, sB, yes, no);
      top(t + 1);
      step(t + 1, sB, sA, yes, no);
    }
    if (t + 1 < t_end) {
      top(t);
      step(t, sA, sB, yes, yes);
      sA[0] = sB[0];
      sA[1] = sB[1];
      ++t;
    }
    top(t);
    // the last tile's P and PV
    u32x4 w1[2];
    float l_tile = l_pend + half_p(sA, 1, t, w1);
    if (outgrown(l_tile, sA, t)) {
      l_tile = half_p(sA, 0, t, p0);
      l_tile += half_p(sA, 1, t, w1);
    }
    l_run += l_tile;
    const uint32_t vaddr = vaddr_of((t - t_begin) & 1);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int db = 0; db < DBLK; ++db)
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vfrag_at(vaddr, db, j), as_frag(j < 2 ? p0[j & 1] : w1[j & 1]), oacc[db], 0, 0, 0);
  }
  publish_barrier<0>();  // no load in flight, every wave done with the tile buffers
  __builtin_amdgcn_s_setprio(0);

  // Epilogue: the row's sum, its rows staged through LDS so that a store moves 16 bytes of
  // a row and a wave's store whole rows.
  // What it needs of the arguments and the row is formed again rather than held through the
  // loop.
  LateArgs& late = late_args();
  const FastDiv d_group{late.d_group.d, late.d_group.mul};
  const int lane_e = (int)opaque_v((uint32_t)lane), n_e = lane_e & 31, row_e = row0 + n_e;
  const bool row_ok = row_e < R;
  const float l_tot = l_run + __shfl_xor(l_run, 32);
  float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
  float lse_v = m_run == -__builtin_inff() || l_tot <= 0.f ? -__builtin_inff() : (m_run + __log2f(l_tot)) * 0.6931471805599453f;
  if (l_tot != l_tot) {  // a NaN among the row's scores is the row's, through the merge as well
    inv = l_tot;
    lse_v = one_part ? l_tot : __builtin_inff();
  }
  float sc = inv;
  int ex = 0;
  if (!one_part) {
    float amax = 0.f;
#pragma unroll
    for (int db = 0; db < DBLK; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) amax = fmaxf(amax, fabsf(oacc[db][j]));
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(amax), __float_as_uint(amax), false, false);
    ex = partial_row_exponent(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * inv);
    sc = inv * exp2_int(-ex);
  }
  constexpr int kStageRow = D * 2 + 16;  // padded: the 32 rows of a wave spread over the LDS banks
  static_assert(4 * 32 * kStageRow <= (int)(sizeof(sm.k) + sizeof(sm.v)), "staging fits the tile buffers");
  INFLLM_LDS char* stage = (INFLLM_LDS char*)(INFLLM_LDS bf16_t*)sm.k[0] + wave * 32 * kStageRow;
#pragma unroll
  for (int db = 0; db < DBLK; ++db) {
#pragma unroll
    for (int jq = 0; jq < 4; ++jq) {
      const float o0 = oacc[db][4 * jq] * sc, o1 = oacc[db][4 * jq + 1] * sc;
      const float o2 = oacc[db][4 * jq + 2] * sc, o3 = oacc[db][4 * jq + 3] * sc;
      u32x2 x;
      if (one_part) {
        x[0] = (uint32_t)f32_to_bf16(o0) | ((uint32_t)f32_to_bf16(o1) << 16);
        x[1] = (uint32_t)f32_to_bf16(o2) | ((uint32_t)f32_to_bf16(o3) << 16);
      } else {
        x[0] = pack_f16x2(o0, o1);
        x[1] = pack_f16x2(o2, o3);
      }
      *(INFLLM_LDS u32x2*)(stage + n_e * kStageRow + (32 * db + 8 * jq + 4 * (lane_e >> 5)) * 2) = x;
    }
  }
  // Values that are not finite must not reach rows that do not see their key: in a masked
  // tile such a value meets P = 0 and leaves a NaN.  A row that came out so is formed again
  // by the wave from the keys it sees, 64 at a time, against its maximum.
  {
    float z4[4] = {};
#pragma unroll
    for (int db = 0; db < DBLK; ++db)
#pragma unroll
      for (int j = 0; j < 16; ++j) z4[j & 3] = __builtin_fmaf(oacc[db][j], 0.f, z4[j & 3]);
    const float z = (z4[0] + z4[1]) + (z4[2] + z4[3]);
    const uint64_t odd = __ballot(row_ok && !(z == 0.f) && l_tot == l_tot);
    uint32_t rows = (uint32_t)odd | (uint32_t)(odd >> 32);
    if (__builtin_expect(rows != 0, 0)) {
      wave_lds_order();
      constexpr int DPL = D / 64;
      for (; rows != 0; rows &= rows - 1) {
        const int r = __builtin_ctz(rows);
        const int i = div_by(row0 + r, d_group), h = g * G + row0 + r - i * G, p_r = w.past + i;
        const float nm = __shfl(neg_m, r), inv_r = __shfl(inv, r), slope_r = __shfl(slope, r);
        float acc[DPL];
        form_row<bf16_t, D>(keys, kbase, vbase, (const bf16_t*)late.q + (int64_t)(w.start + i) * late.q_tok + (int64_t)h * late.q_head,
                            p_r, a.window, a.n_init,
                            [&](float s, int key) { return fast_exp2(score.exponent(score.form(s), score.base(slope_r * (float)(key - p_r))) + nm); }, acc);
        float amax = 0.f;  // (of the finite ones, which keep their precision)
#pragma unroll
        for (int e = 0; e < DPL; ++e) {
          acc[e] *= inv_r;
          const float x = fabsf(acc[e]);
          amax = x < __builtin_inff() ? fmaxf(amax, x) : amax;
        }
        const int ex_r = one_part ? 0 : partial_row_exponent(wave_max(amax));
        if (n_e == r) ex = ex_r;
        const float back = exp2_int(-ex_r);
#pragma unroll
        for (int e = 0; e < DPL; ++e) {
          const uint32_t x = one_part ? f32_to_bf16(acc[e]) : pack_f16x2(acc[e] * back, 0.f) & 0xFFFFu;
          *(INFLLM_LDS uint16_t*)(stage + r * kStageRow + 2 * (DPL * lane + e)) = (uint16_t)x;
        }
      }
    }
  }
  const int64_t prow0 = ((int64_t)blockIdx.x) * late.item_rows;  // of the item's partial rows
  if (row_ok && lane_e < 32) {
    if (!one_part) {
      late.part_lse[prow0 + row_e - tile0] = lse_v;
      late.part_exp[prow0 + row_e - tile0] = ex;
    } else if (late.lse != nullptr) {
      const int i = div_by(row_e, d_group), h = g * G + row_e - i * G;
      late.lse[h * late.lse_stride + w.start + i] = lse_v;
    }
  }
  wave_lds_order();
  {
    constexpr int NS = 32 * CH / 64;  // pieces of a lane
    const int r0 = lane_e / CH, ch = lane_e % CH;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      if (row0 + RPI * k >= R) break;  // (uniform)
      const int r = row0 + RPI * k + r0;
      if (r >= R) continue;
      const u32x4 x = *(const INFLLM_LDS u32x4*)(stage + (RPI * k + r0) * kStageRow + ch * 16);
      if (one_part) {
        const int i = div_by(r, d_group), h = g * G + r - i * G;
        *(u32x4*)((bf16_t*)late.out + (int64_t)(w.start + i) * late.out_tok + (int64_t)h * late.out_head + 8 * ch) = x;
      } else {
        *(u32x4*)((char*)late.part_o + (prow0 + r - tile0) * (D * 2) + 16 * ch) = x;
      }
    }
  }
}

// Float32: NW waves of 32 rows on the float32 matrix cores (v_mfma_f32_32x32x2_f32), key
// tiles of 32 through two LDS buffers, one tile ahead.  S^T = K Q^T takes the dims in the
// order that lets one 16-byte read feed four products; sums of 16 products are joined by
// additions.  O^T += V^T P^T with P^T as it stands; output block db holds dims DBLK*m + db,
// so that one read feeds all blocks.  Rows of an LDS tile are XOR-swizzled by piece, which
// leaves both reads without conflicts.  Bound by the float32 matrix cores where a workgroup
// has its keys (64 dims: a tile's products 1.8 us, its softmax 0.7), and in small batches by
// what stands around them: 637 tokens of five sequences after up to 2,600, 8 query heads of
// 64, 20.9 us and 6.5 for the merge, of which 3.4 are the wait for arguments, table and first
// tile.  Rows of a tile (128, 64, 32) by the longest sequence's: waves without rows would
// only load.
constexpr int kF32Tile = 32;

// e^x for x <= 0 (and NaN): 2^t, t = x log2(e) rounded, which moves e^x by at most 2^-25 of
// the row's largest weight.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269502f); }

template <int D, int NW, int MOD>
__global__ void __launch_bounds__(64 * NW, D == 64 && NW > 1 ? 2 : 1) paged_f32_kernel(PagedArgs a) {
  constexpr int KT = kF32Tile, RW = 32 * NW, QL = D / 2, DBLK = D / 32;
  constexpr int GPR = D / 4, RPI = 64 / GPR, NI = KT / (RPI * NW);
  constexpr uint32_t kTileBytes = KT * D * 4;
  __shared__ __attribute__((aligned(256))) float ks[2][KT * D];
  __shared__ __attribute__((aligned(256))) float vs[2][KT * D];
  __shared__ KeyTable table;
  __shared__ int wave_bad[NW];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, gsel = lane >> 5;
  const int G = (int)a.d_group.d;
  const int item = div_by(blockIdx.x, a.d_kv), g = (int)blockIdx.x - item * (int)a.d_kv.d;
  const PagedWork w = paged_work(a, item);
  const int R = G * w.len, tile0 = w.rt * RW;
  const int i0 = div_by(tile0, a.d_group), i1 = div_by(min(R, tile0 + RW) - 1, a.d_group);
  const PagedRange range = paged_range(a, w.past, i0, i1);
  const int t_begin = w.part * w.part_tiles, t_end = min(t_begin + w.part_tiles, range.n);
  if (t_begin >= t_end) return;
  const bool one_part = range.n <= w.part_tiles;
  const int last = w.past + w.len - 1;
  KeyTiles<KT, 64 * NW, (MOD & kSlopes) != 0> keys{range.sink, range.low - range.sink, t_begin, t_end, last, w.table_row, (a.page_size & 7) == 0 ? 3 : 0, t_begin};

  const int row0 = tile0 + wave * 32, row = row0 + n;
  const bool active = row0 < R, row_ok = row < R;
  const int row_c = min(row, R - 1);
  const int qi = div_by(row_c, a.d_group), qh = g * G + row_c - qi * G;
  const int pos = w.past + qi;
  const char* kbase = (const char*)a.k + g * a.head_stride * 4;
  const char* vbase = (const char*)a.v + g * a.head_stride * 4;
  const float* qp = (const float*)a.q + (int64_t)(w.start + qi) * a.q_tok + (int64_t)qh * a.q_head;
  float qv[QL];
#pragma unroll
  for (int i = 0; i < QL / 4; ++i) {
    const f32x4 x = *(const f32x4*)(qp + 8 * i + 4 * gsel);
#pragma unroll
    for (int e = 0; e < 4; ++e) qv[4 * i + e] = x[e];
  }
  float slope = 0.f;
  if constexpr (MOD & kSlopes) slope = a.slopes[qh];

  {
    const bool any = __ballot(keys.fill_first(table)) != 0;
    if (lane == 0) wave_bad[wave] = any;
  }
  lds_barrier();
  bool has_bad = false;
#pragma unroll
  for (int i = 0; i < NW; ++i) has_bad |= wave_bad[i] != 0;

  const uint32_t lds_k = (uint32_t)(uintptr_t)(INFLLM_LDS float*)ks[0] + NI * wave * 1024;
  const uint32_t lds_v = (uint32_t)(uintptr_t)(INFLLM_LDS float*)vs[0] + NI * wave * 1024;
  const uint32_t gmask = (1u << keys.gshift) - 1u;
  auto load_tile = [&](int t) {
    const uint32_t buf = ((t - t_begin) & 1) * kTileBytes;
    const int in_tile = min(KT - 1, last - keys.key_of(t));
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int lr = (NI * wave + j) * RPI + lane / GPR;
      const uint32_t r = (uint32_t)min(lr, in_tile);
      const uint32_t p = table.place[(t - keys.w0) * keys.tile_groups() + (r >> keys.gshift)] + __umul24(r & gmask, a.token16);
      const uint64_t off = ((uint64_t)p + (uint32_t)((lane % GPR) ^ (lr & 15))) * 16;
      lds_load_lane(lds_k + buf + j * 1024, kbase + off);
      lds_load_lane(lds_v + buf + j * 1024, vbase + off);
    }
  };

  f32x16 o[DBLK];
#pragma unroll
  for (int db = 0; db < DBLK; ++db)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[db][j] = 0.f;
  float m = -__builtin_inff(), l = 0.f;
  auto score_of = [&](float s, int distance) {  // distance: of the key from the query, <= 0
    float z = s * a.sm_scale;
    if constexpr (MOD & kCap) z = a.softcap * tanhf(z / a.softcap);
    if constexpr (MOD & kSlopes) z = __builtin_fmaf(slope, (float)distance, z);
    return z;
  };
  // tiles all of whose keys every row of the wave sees: [plain0, plain1)
  const int w0 = div_by(min(row0, R - 1), a.d_group), w1 = div_by(min(row0 + 31, R - 1), a.d_group);
  int plain0 = a.window > 0 ? (max(0, w.past + w1 - a.window + 1) + KT - 1) / KT : 0;
  int plain1 = has_bad ? 0 : (w.past + w0 + 1) / KT;
  keys.range(&plain0, &plain1);

  load_tile(t_begin);
  for (int t = t_begin; t < t_end; ++t) {
    publish_barrier<0>();  // tile t has landed; the other buffer is free
    asm volatile("" ::: "memory");
    if (t + 1 < t_end) {
      if (t + 1 >= keys.w0 + keys.window()) {
        keys.fill(table, t);  // (tile t's mask may ask it)
        lds_barrier();
      }
      load_tile(t + 1);
    }
    if (!active) continue;
    const float *kt = ks[(t - t_begin) & 1], *vt = vs[(t - t_begin) & 1];
    f32x16 s;
#pragma unroll
    for (int i0 = 0; i0 < QL / 4; i0 += 4) {
      f32x16 s0 = {}, s1 = {};
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) {
        const f32x4 kf = *(const f32x4*)(kt + n * D + 4 * ((2 * i + gsel) ^ (n & 15)));
        s0 = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[0], qv[4 * i], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[1], qv[4 * i + 1], s1, 0, 0, 0);
        s0 = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[2], qv[4 * i + 2], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[3], qv[4 * i + 3], s1, 0, 0, 0);
      }
      s = i0 == 0 ? s0 + s1 : s + (s0 + s1);
    }
    const bool plain = t >= plain0 && t < plain1;
    const int k0 = keys.key_of(t);
    // (without a form a plain tile's scale is part of the exponential's argument)
    const float in_exp = MOD == 0 && plain ? a.sm_scale : 1.f;
    if (MOD != 0 || !plain) {
#pragma unroll
      for (int j = 0; j < 16; ++j) s[j] = score_of(s[j], k0 + 8 * (j >> 2) + 4 * gsel + (j & 3) - pos);
    }
    if (!plain) {
      uint64_t vis = seen_keys(pos, k0, a.window, a.n_init);
      if (has_bad) vis &= keys.there(table, t);
      const uint32_t see = (uint32_t)vis >> (4 * gsel);
#pragma unroll
      for (int j = 0; j < 16; ++j) s[j] = ((see >> (8 * (j >> 2) + (j & 3))) & 1u) != 0 ? s[j] : -__builtin_inff();
    }
    float mx = s[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s[j]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * in_exp;
    if (__ballot(mx > m)) {
      const float m_new = fmaxf(m, mx), corr = m_new == -__builtin_inff() ? 1.f : expf(m - m_new);
      m = m_new;
      l *= corr;
#pragma unroll
      for (int db = 0; db < DBLK; ++db)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[db][j] *= corr;
    }
    const float base = m == -__builtin_inff() ? 0.f : m;
    float ls[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[j] = exp_of(__builtin_fmaf(s[j], in_exp, -base));
      ls[j & 1] += s[j];
    }
    l += ls[0] + ls[1];
    typedef float vfrag_t __attribute__((ext_vector_type(DBLK)));
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int r = 8 * (j >> 2) + 4 * gsel + (j & 3), d0 = DBLK * n;
      const vfrag_t vf = *(const vfrag_t*)(vt + r * D + 4 * ((d0 >> 2) ^ (r & 15)) + (d0 & 3));
#pragma unroll
      for (int db = 0; db < DBLK; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[db], s[j], o[db], 0, 0, 0);
    }
  }
  if (!active) return;

  const auto lw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  const float l_tot = __uint_as_float(lw[0]) + __uint_as_float(lw[1]);
  float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
  float lse_v = l_tot > 0.f ? m + logf(l_tot) : -__builtin_inff();
  if (l_tot != l_tot) {  // a NaN among the row's scores is the row's, through the merge as well
    inv = l_tot;
    lse_v = one_part ? l_tot : __builtin_inff();
  }
  const int64_t prow = (int64_t)blockIdx.x * a.item_rows - tile0;  // plus a row: its partial row
  typedef float orow_t __attribute__((ext_vector_type(DBLK)));
  float z4[4] = {};
#pragma unroll
  for (int db = 0; db < DBLK; ++db)
#pragma unroll
    for (int j = 0; j < 16; ++j) z4[j & 3] = __builtin_fmaf(o[db][j], 0.f, z4[j & 3]);
  const bool odd = row_ok && !((z4[0] + z4[1]) + (z4[2] + z4[3]) == 0.f) && l_tot == l_tot;
  if (row_ok) {
    float* op = one_part ? (float*)a.out + (int64_t)(w.start + qi) * a.out_tok + (int64_t)qh * a.out_head
                         : (float*)a.part_o + (prow + row) * D;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      orow_t x;
#pragma unroll
      for (int db = 0; db < DBLK; ++db) x[db] = o[db][j] * inv;
      if (!odd) *(orow_t*)(op + DBLK * (8 * (j >> 2) + 4 * gsel + (j & 3))) = x;
    }
    if (gsel == 0) {
      if (!one_part) a.part_lse[prow + row] = lse_v;
      else if (a.lse != nullptr) a.lse[qh * a.lse_stride + w.start + qi] = lse_v;
    }
  }
  // Rows that a masked value which is not finite has reached (0 times it) are formed again
  // from the keys that they see.
  const uint64_t odds = __ballot(odd);
  for (uint32_t left = (uint32_t)odds | (uint32_t)(odds >> 32); left != 0; left &= left - 1) {
    const int r = __builtin_ctz(left);
    const int i = div_by(row0 + r, a.d_group), h = g * G + row0 + r - i * G, p_r = w.past + i;
    const float m_r = __shfl(m, r), base_r = m_r == -__builtin_inff() ? 0.f : m_r, inv_r = __shfl(inv, r);
    const float slope_r = __shfl(slope, r);
    float acc[D / 64];
    form_row<float, D>(keys, kbase, vbase, (const float*)a.q + (int64_t)(w.start + i) * a.q_tok + (int64_t)h * a.q_head, p_r, a.window, a.n_init,
                       [&](float x, int key) {
                         float z = x * a.sm_scale;
                         if constexpr (MOD & kCap) z = a.softcap * tanhf(z / a.softcap);
                         return exp_of(__builtin_fmaf(slope_r, (float)(key - p_r), z) - base_r);
                       }, acc);
    float* op = one_part ? (float*)a.out + (int64_t)(w.start + i) * a.out_tok + (int64_t)h * a.out_head
                         : (float*)a.part_o + (prow + row0 + r) * D;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) op[D / 64 * lane + e] = acc[e] * inv_r;
  }
}

template <int D, int MOD>
void launch_form(const PagedArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.items * a.n_kv_heads)), block(2 << a.rows_log2);
  if constexpr ((MOD & kWideCap) == 0) {  // (float32 has one form for every cap)
    if (!a.bf16) {
      if (a.rows_log2 == 7) hipLaunchKernelGGL((paged_f32_kernel<D, 4, MOD>), grid, block, 0, s, a);
      else if (a.rows_log2 == 6) hipLaunchKernelGGL((paged_f32_kernel<D, 2, MOD>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((paged_f32_kernel<D, 1, MOD>), grid, block, 0, s, a);
      return;
    }
  }
  if (a.page_size % 8 == 0) hipLaunchKernelGGL((paged_mfma_kernel<D, MOD, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((paged_mfma_kernel<D, MOD, false>), grid, block, 0, s, a);
}
template <int D>
void launch_d(const PagedArgs& a, hipStream_t s) {
  const int cap = a.softcap == 0.f ? 0 : a.bf16 && a.softcap > kMostFolded ? kWideCap : kCap;
  const int mod = cap | (a.slopes != nullptr ? kSlopes : 0);
  if (mod == 0) launch_form<D, 0>(a, s);
  else if (mod == kCap) launch_form<D, kCap>(a, s);
  else if (mod == kSlopes) launch_form<D, kSlopes>(a, s);
  else if (mod == (kCap | kSlopes)) launch_form<D, kCap | kSlopes>(a, s);
  else if (mod == kWideCap) launch_form<D, kWideCap>(a, s);
  else launch_form<D, kWideCap | kSlopes>(a, s);
}

}  // namespace

hipError_t launch_paged(const PagedArgs& a, hipStream_t s) {
  if (a.head_dim == 128) launch_d<128>(a, s);
  else launch_d<64>(a, s);
  return hipGetLastError();
}

}  // namespace infllm
