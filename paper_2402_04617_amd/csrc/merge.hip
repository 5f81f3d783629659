// Log-sum-exp merge of partial attentions over disjoint key parts:
// LSE = log sum_s exp(lse_s), O = sum_s exp(lse_s - LSE) O_s.  The parts together
// are the single softmax over Concat(C, X) of Section 3.1.
//
// One thread per (row, 16 bytes of partial row): 8 dims of a scaled-fp16 partial
// (bfloat16 inputs; value * 2^exp[row] restores the row) or 4 dims of a float32
// one.  A thread takes all parts, CH at a time (CH = the part count, or 8), every load
// of those issued before the first use.  More than 8 parts of few rows (decoding), at
// least half as many as a workgroup has groups: a workgroup per row, its threads split into groups that take every GR-th part and are
// joined in LDS -- the parts are then the only parallelism (25 parts of 32 rows: 6.8 us
// one thread per piece, 4.3 split; 16 parts of 2,048 rows: 3.7 and 6.5).
#include <type_traits>

#include "paged.h"
#include "shared.h"

namespace infllm {
namespace {

// One piece of one part's row: its values in float, and its lse.
template <bool HALF, typename Args>
__device__ __forceinline__ void load_piece(const Args& a, int64_t pr, int c, float (&o)[HALF ? 8 : 4], float& l) {
  l = a.part_lse[pr];
  if constexpr (HALF) {
    const uint4 w = *(const uint4*)((const uint16_t*)a.part_o + pr * a.head_dim + 8 * c);
    const float sc = exp2_int(a.part_exp[pr]);
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      o[2 * q] = f16_lo(ww[q]) * sc;
      o[2 * q + 1] = f16_hi(ww[q]) * sc;
    }
  } else {
    const float4 w = *(const float4*)((const float*)a.part_o + pr * a.head_dim + 4 * c);
    o[0] = w.x;
    o[1] = w.y;
    o[2] = w.z;
    o[3] = w.w;
  }
}
// Adds the first `n` of CH pieces to a running maximum, weight sum and weighted row.  ANY:
// the pieces may hold values that are not finite, which no weight of 0 may meet: it would
// leave a NaN (the piece of a thread past the last part is that part's again).
template <int DPT, int CH, bool ANY>
__device__ __forceinline__ void add_parts(const float (&l)[CH], const float (&o)[CH][DPT], int n, bool rescale, float& M,
                                          float& tot, float (&acc)[DPT]) {
  float m_new = M;
#pragma unroll
  for (int j = 0; j < CH; ++j)
    if (j < n) m_new = fmaxf(m_new, l[j]);
  if (m_new == -__builtin_inff()) return;  // nothing visible yet
  if (rescale) {
    const float r = M == -__builtin_inff() ? 0.f : expf(M - m_new);
    tot *= r;
#pragma unroll
    for (int e = 0; e < DPT; ++e) acc[e] *= r;
  }
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const bool live = j < n && l[j] != -__builtin_inff();
    const float w = live ? expf(l[j] - m_new) : 0.f;
    tot += w;
#pragma unroll
    for (int e = 0; e < DPT; ++e) acc[e] += w * (!ANY || live ? o[j][e] : 0.f);
  }
  M = m_new;
}
// Joins parts first, first + step, ... (every load of CH of them issued before the
// first use) into a running maximum, weight sum and weighted row.  ONCE: there are at
// most CH of them.
template <bool HALF, int CH, bool ONCE, bool ANY = false>
__device__ __forceinline__ void join_parts(const MergeArgs& a, int row, int c, int first, int step, float& M, float& tot,
                                           float (&acc)[HALF ? 8 : 4]) {
  constexpr int DPT = HALF ? 8 : 4;
  M = -__builtin_inff();
  tot = 0.f;
#pragma unroll
  for (int e = 0; e < DPT; ++e) acc[e] = 0.f;
  for (int p0 = first; p0 < a.parts; p0 += CH * step) {
    float l[CH], o[CH][DPT];
#pragma unroll
    for (int j = 0; j < CH; ++j)
      load_piece<HALF>(a, (int64_t)min(p0 + j * step, a.parts - 1) * a.rows + row, c, o[j], l[j]);
    add_parts<DPT, CH, ANY>(l, o, (a.parts - p0 + step - 1) / step, !ONCE, M, tot, acc);
    if (ONCE) break;
  }
}
template <typename T, int DPT>
__device__ __forceinline__ void store_row_piece(T* op, float* lse, float M, float tot, const float (&acc)[DPT]) {
  const float inv = tot > 0.f ? 1.f / tot : 0.f;
  if constexpr (sizeof(T) == 2) {
    uint32_t w[DPT / 2];
#pragma unroll
    for (int q = 0; q < DPT / 2; ++q)
      w[q] = (uint32_t)f32_to_bf16(acc[2 * q] * inv) | ((uint32_t)f32_to_bf16(acc[2 * q + 1] * inv) << 16);
    if constexpr (DPT == 8) *(uint4*)op = make_uint4(w[0], w[1], w[2], w[3]);
    else *(uint2*)op = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int e = 0; e < DPT; ++e) op[e] = acc[e] * inv;
  }
  // (tot is NaN where a part's scores hold a NaN: such a part comes with lse = +inf)
  if (lse != nullptr) *lse = tot > 0.f ? M + logf(tot) : tot != tot ? tot : -__builtin_inff();
}
template <typename T, int DPT>
__device__ __forceinline__ void store_piece(const MergeArgs& a, int row, int c, float M, float tot, const float (&acc)[DPT]) {
  const int bh = row / a.n_q, i = row - bh * a.n_q;
  store_row_piece<T, DPT>((T*)a.out + (int64_t)bh * a.out_head_stride + (int64_t)i * a.head_dim + DPT * c,
                          a.lse != nullptr && c == 0 ? a.lse + row : nullptr, M, tot, acc);
}

template <typename T, bool HALF, int CH>
__global__ void __launch_bounds__(256) merge_kernel(MergeArgs a) {
  constexpr int DPT = HALF ? 8 : 4;  // dims per thread
  const int tpr = a.head_dim / DPT;
  const int rows_per_wg = 256 / tpr;
  // Workgroups in the attention's XCD order (reversed, consecutive ids on one
  // XCD): where a kv head's parts were written by the workgroups of one XCD, the
  // rows of that kv head are merged on the same XCD and read its L2.
  const int wg = (int)gridDim.x - 1 - xcd_logical_block(blockIdx.x, gridDim.x);
  const int row = wg * rows_per_wg + threadIdx.x / tpr;
  const int c = threadIdx.x % tpr;
  if (row >= a.rows) return;
  float M, tot, acc[DPT];
  join_parts<HALF, CH, (CH < 8)>(a, row, c, 0, 1, M, tot, acc);
  store_piece<T, DPT>(a, row, c, M, tot, acc);
}

// More than 8 parts: one workgroup per row.
template <typename T, bool HALF>
__global__ void __launch_bounds__(256) merge_many_kernel(MergeArgs a) {
  constexpr int DPT = HALF ? 8 : 4, CH = 4;
  const int row = blockIdx.x;
  const int tpr = a.head_dim / DPT, groups = 256 / tpr;  // 8 to 32 groups
  const int c = threadIdx.x % tpr, grp = threadIdx.x / tpr;
  __shared__ float sM[32], sT[32], sO[256 * DPT];
  float M, tot, acc[DPT];
  if (a.parts <= CH * groups) join_parts<HALF, CH, true>(a, row, c, grp, groups, M, tot, acc);
  else join_parts<HALF, CH, false>(a, row, c, grp, groups, M, tot, acc);
  if (c == 0) {
    sM[grp] = M;
    sT[grp] = tot;
  }
#pragma unroll
  for (int e = 0; e < DPT; ++e) sO[threadIdx.x * DPT + e] = acc[e];
  __syncthreads();
  if (grp != 0) return;
  for (int g = 0; g < groups; ++g) M = fmaxf(M, sM[g]);
  tot = 0.f;
#pragma unroll
  for (int e = 0; e < DPT; ++e) acc[e] = 0.f;
  if (M != -__builtin_inff()) {
    for (int g = 0; g < groups; ++g) {
      const float w = sM[g] == -__builtin_inff() ? 0.f : expf(sM[g] - M);
      tot += w * sT[g];
#pragma unroll
      for (int e = 0; e < DPT; ++e) acc[e] += w * sO[(g * tpr + c) * DPT + e];
    }
  }
  store_piece<T, DPT>(a, row, c, M, tot, acc);
}

// The split row tiles of packed prompts: workgroups (row tile, kv head, rows of it); a
// row's parts lie in the items of its row tile.  Bound by the partial rows' bytes and its
// launch: 14 MB of 52,992 float32 rows of 64 dims 7.7 us.
template <typename T, bool HALF, int CH>
__global__ void __launch_bounds__(256) prompt_merge_kernel(PromptArgs a, int rows_log2) {
  constexpr int DPT = HALF ? 8 : 4;
  const int tpr = a.head_dim / DPT, rows_per_wg = 256 / tpr;
  const int per_tile = (1 << rows_log2) / rows_per_wg;  // workgroups of a row tile
  const int tg = (int)blockIdx.x / per_tile, sub = (int)blockIdx.x - tg * per_tile;
  const int t = div_by(tg, a.d_kv), g = tg - t * (int)a.d_kv.d;
  const PromptTile pt = prompt_tile(a, t, rows_log2);
  const int r = sub * rows_per_wg + (int)threadIdx.x / tpr, c = threadIdx.x % tpr;
  const int row = (pt.tile << rows_log2) + r, G = (int)a.d_group.d;
  if (row >= pt.len * G) return;
  int parts = 1;
  for (int p = 1; p < a.parts; ++p) parts += t < prompt_part_count(a, p) ? 1 : 0;
  float l[CH], o[CH][DPT];
  float M = -__builtin_inff(), tot = 0.f, acc[DPT] = {};
  for (int p0 = 0; p0 < parts; p0 += CH) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int64_t pr = (((int64_t)prompt_item_of(a, min(p0 + j, parts - 1), t) * a.n_kv_heads + g) << rows_log2) + r;
      load_piece<HALF>(a, pr, c, o[j], l[j]);
    }
    add_parts<DPT, CH, true>(l, o, parts - p0, p0 > 0, M, tot, acc);
  }
  const int i = div_by(row, a.d_group), h = g * G + row - i * G;
  store_row_piece<T, DPT>((T*)a.out + (pt.start + i) * a.out_tok + h * a.out_head + DPT * c,
                          a.lse != nullptr && c == 0 ? a.lse + h * a.lse_stride + pt.start + i : nullptr, M, tot, acc);
}

// The parts of the prefix attention, and its few current tokens.  A wave per row: its
// 64 / tpr groups of lanes take every GR-th part (the loads of CH of them issued before
// the first use) and every GR-th current token, and are joined by lane exchanges.  A wave
// of a group's first head also writes its token's key and value to the own store: a few
// current tokens cost two 16-byte loads a lane here, and no launch of their own nor a part.
// A row's parts are the only parallelism where rows are few, hence a wave per row.  Bound
// by latency, the pieces' trip to memory and five exchanges: 128 rows of 26 parts and a
// current token 5.7 us; 1,024 rows of 48 parts (13 MB) 8.6.
template <typename T, bool HALF, int D>
__global__ void __launch_bounds__(256) prefix_merge_kernel(PrefixArgs a) {
  constexpr int DPT = HALF ? 8 : 4, TPR = D / DPT, GR = 64 / TPR, CH = 4;
  const int row = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int rows = a.batch * a.n_q_heads * a.n_q;
  if (row >= rows) return;
  const int lane = threadIdx.x & 63, c = lane % TPR, grp = lane / TPR;
  const int bh = div_by(row, a.d_q), i = row - bh * a.n_q;
  const int bg = div_by(bh, a.d_group);  // (sequence, kv head)
  const MergeArgs m = {rows, D, a.parts, a.n_q, a.n_q_heads, a.out_head_stride, a.part_o, a.part_lse, a.part_exp, a.out, a.lse, HALF};
  // the current tokens' rows, requested first
  float q[DPT] = {};
  float xk[CH][DPT], xv[CH][DPT];
  auto load_row = [&](const void* p, int64_t at, float (&x)[DPT]) {
    const T* r = (const T*)p + at + DPT * c;
    if constexpr (HALF) {
      const u32x4 w = *(const u32x4*)r;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
      }
    } else {
      const f32x4 w = *(const f32x4*)r;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = w[j];
    }
  };
  const int64_t x0 = bg * a.x_head_stride;
  if (a.x_k != nullptr) {
    load_row(a.q, bh * a.q_head_stride + (int64_t)i * D, q);
#pragma unroll
    for (int j = 0; j < CH; ++j) {  // (a token past the query's own is not looked at)
      const int64_t at = x0 + (int64_t)min(grp + j * GR, i) * D;
      if (j * GR < a.n_q) {
        load_row(a.x_k, at, xk[j]);
        load_row(a.x_v, at, xv[j]);
      }
    }
  }
  float M, tot, acc[DPT];
  if (a.parts <= CH * GR) join_parts<HALF, CH, true, true>(m, row, c, grp, GR, M, tot, acc);
  else if (a.parts <= 2 * CH * GR) join_parts<HALF, 2 * CH, true, true>(m, row, c, grp, GR, M, tot, acc);
  else join_parts<HALF, 3 * CH, false, true>(m, row, c, grp, GR, M, tot, acc);
  if (a.x_k != nullptr) {
    static_assert(kPrefixMergeTokens <= CH * GR, "every token has a place");
    float z[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      z[j] = -__builtin_inff();
      if (j * GR >= a.n_q) continue;
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < DPT; ++e) s = __builtin_fmaf(q[e], xk[j][e], s);
#pragma unroll
      for (int o = 1; o < TPR; o <<= 1) s += __shfl_xor(s, o);
      s *= a.sm_scale;
      // (a NaN score as the attention's parts give it)
      if (grp + j * GR <= i) z[j] = s == s ? s : __builtin_inff();
    }
    add_parts<DPT, CH, true>(z, xv, CH, true, M, tot, acc);
  }
  // the groups' shares
#pragma unroll
  for (int o = TPR; o < 64; o <<= 1) {
    const float M2 = __shfl_xor(M, o), tot2 = __shfl_xor(tot, o), m_new = fmaxf(M, M2);
    const float w1 = M == -__builtin_inff() ? 0.f : expf(M - m_new), w2 = M2 == -__builtin_inff() ? 0.f : expf(M2 - m_new);
    tot = tot * w1 + tot2 * w2;
#pragma unroll
    for (int e = 0; e < DPT; ++e) {
      const float x2 = __shfl_xor(acc[e], o);
      acc[e] = (M == -__builtin_inff() ? 0.f : acc[e] * w1) + (M2 == -__builtin_inff() ? 0.f : x2 * w2);
    }
    M = m_new;
  }
  if (grp == 0) store_piece<T, DPT>(m, row, c, M, tot, acc);
  if (a.x_k != nullptr && bh == bg * (int)a.d_group.d && grp < 2) {
    const int b = bg / a.n_kv_heads;
    const int64_t to = ((int64_t)bg * a.own_capacity + a.own_len[b] + i) * D + DPT * c;
    const int64_t from = x0 + (int64_t)i * D + DPT * c;
    const void* src = grp == 0 ? a.x_k : a.x_v;
    void* dst = const_cast<void*>(grp == 0 ? a.own_k : a.own_v);
    *(u32x4*)((T*)dst + to) = *(const u32x4*)((const T*)src + from);
  }
}

// Paged attention: the parts of a row tile's rows.  Of a row tile with P parts the
// workgroups of each part's item join a P-th of the rows, so that none is idle.  SPLIT: few
// rows to an item (decoding), a wave per row whose lane groups take every GR-th part; else
// a group of lanes per row.  Bound by its chain of loads (arguments, the parts' rows): 4.5
// to 5 us for one token's parts, 6.5 for 48 sequences', 10.5 where two chunks of 512 and 300
// tokens join some 50,000 partial rows (13.6 MB read, 4.4 written).
//
// TURNS: a workgroup takes its rows in turns of `at_once`.  Where the workgroups do not all fit
// the chip (2,048 of them), half as many are quicker: that batch 10.5 us, not 12.8; where
// they do, a loop costs 0.4 of 6.6.
template <typename T, bool HALF, int D, bool SPLIT, bool TURNS>
__global__ void __launch_bounds__(256) paged_merge_kernel(PagedArgs a, int at_once) {
  constexpr int DPT = HALF ? 8 : 4, TPR = D / DPT, GR = SPLIT ? 64 / TPR : 1;
  const int item = div_by(blockIdx.x, a.d_kv), g = (int)blockIdx.x - item * (int)a.d_kv.d;
  const PagedWork w = paged_work(a, item);
  const int G = (int)a.d_group.d, rows_wg = 1 << a.rows_log2, R = G * w.len, tile0 = w.rt * rows_wg;
  const int i0 = div_by(tile0, a.d_group), i1 = div_by(min(R, tile0 + rows_wg) - 1, a.d_group);
  const int n = paged_range(a, w.past, i0, i1).n;
  const int parts = (n + w.part_tiles - 1) / w.part_tiles;
  if (parts == 1 || w.part >= parts) return;
  const int rows = min(rows_wg, R - tile0), share = (rows + parts - 1) / parts;
  const int r_end = min(rows, (w.part + 1) * share);
  const int r0 = w.part * share + blockIdx.y * (256 / (TPR * GR)) + threadIdx.x / (TPR * GR);
  if (r0 >= r_end) return;
  const int grp = SPLIT ? (threadIdx.x / TPR) % GR : 0, c = threadIdx.x % TPR;
  const int64_t tile_row0 = ((int64_t)(item - w.part) * a.n_kv_heads + g) * a.item_rows, step = (int64_t)a.n_kv_heads * a.item_rows;
  auto row = [&](int r) {
    float M = -__builtin_inff(), tot = 0.f, acc[DPT] = {};
    auto join = [&](auto chunk) {
      constexpr int CH = decltype(chunk)::value;
      for (int p0 = grp; p0 < parts; p0 += CH * GR) {
        float l[CH], o[CH][DPT];
#pragma unroll
        for (int j = 0; j < CH; ++j) load_piece<HALF>(a, tile_row0 + r + min(p0 + j * GR, parts - 1) * step, c, o[j], l[j]);
        add_parts<DPT, CH, true>(l, o, (parts - p0 + GR - 1) / GR, p0 > grp, M, tot, acc);
      }
    };
    if (parts <= 2 * GR) join(std::integral_constant<int, 2>{});
    else if (parts <= 4 * GR) join(std::integral_constant<int, 4>{});
    else join(std::integral_constant<int, 8>{});
    if constexpr (SPLIT) {
#pragma unroll
      for (int o = TPR; o < 64; o <<= 1) {
        const float M2 = __shfl_xor(M, o), tot2 = __shfl_xor(tot, o), m_new = fmaxf(M, M2);
        const float w1 = M == -__builtin_inff() ? 0.f : expf(M - m_new), w2 = M2 == -__builtin_inff() ? 0.f : expf(M2 - m_new);
        tot = tot * w1 + tot2 * w2;
#pragma unroll
        for (int e = 0; e < DPT; ++e) {
          const float x2 = __shfl_xor(acc[e], o);
          acc[e] = (M == -__builtin_inff() ? 0.f : acc[e] * w1) + (M2 == -__builtin_inff() ? 0.f : x2 * w2);
        }
        M = m_new;
      }
      if (grp != 0) return;
    }
    const int i = div_by(tile0 + r, a.d_group), h = g * G + tile0 + r - i * G;
    store_row_piece<T, DPT>((T*)a.out + (int64_t)(w.start + i) * a.out_tok + (int64_t)h * a.out_head + DPT * c,
                            a.lse != nullptr && c == 0 ? a.lse + h * a.lse_stride + w.start + i : nullptr, M, tot, acc);
  };
  if constexpr (TURNS) {
    for (int r = r0; r < r_end; r += at_once) row(r);
  } else {
    row(r0);
  }
}
template <typename T, bool HALF, int D>
void launch_paged_merge_t(const PagedArgs& a, hipStream_t s) {
  constexpr int groups = 256 / (D / (HALF ? 8 : 4));  // of a workgroup
  const bool split = a.item_rows <= 16;
  const int per_wg = split ? 4 : groups, share = (a.item_rows + 1) / 2;  // (of two parts, the most)
  const int wgs = a.items * a.n_kv_heads, turns = (share + per_wg - 1) / per_wg;
  const dim3 block(256);
  if (split) {
    hipLaunchKernelGGL((paged_merge_kernel<T, HALF, D, true, false>), dim3(wgs, turns), block, 0, s, a, 0);
  } else if ((int64_t)wgs * turns <= 2048 || turns < 4) {
    hipLaunchKernelGGL((paged_merge_kernel<T, HALF, D, false, false>), dim3(wgs, turns), block, 0, s, a, 0);
  } else {
    hipLaunchKernelGGL((paged_merge_kernel<T, HALF, D, false, true>), dim3(wgs, turns / 2), block, 0, s, a, turns / 2 * per_wg);
  }
}

constexpr int kManyRows = 1024;  // most rows whose many parts are split over threads

template <typename T, bool HALF>
hipError_t launch_merge_t(const MergeArgs& a, hipStream_t s) {
  constexpr int DPT = HALF ? 8 : 4;
  const int rows_per_wg = 256 / (a.head_dim / DPT);
  const dim3 grid((a.rows + rows_per_wg - 1) / rows_per_wg), block(256);
  // (at least half of a workgroup's groups with a part, or the join of the others' shares
  // shows: 10 parts of 320 rows of 64 dims, 32 groups, 7.6 us split and 5.0 not)
  const int groups = 256 / (a.head_dim / DPT);
  if (a.parts > max(8, groups / 2) && a.rows <= kManyRows) {
    hipLaunchKernelGGL((merge_many_kernel<T, HALF>), dim3(a.rows), block, 0, s, a);
    return hipGetLastError();
  }
  switch (a.parts) {
    case 2: hipLaunchKernelGGL((merge_kernel<T, HALF, 2>), grid, block, 0, s, a); break;
    case 3: hipLaunchKernelGGL((merge_kernel<T, HALF, 3>), grid, block, 0, s, a); break;
    case 4: hipLaunchKernelGGL((merge_kernel<T, HALF, 4>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((merge_kernel<T, HALF, 8>), grid, block, 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_merge(const PromptArgs& a, hipStream_t s) {
  const int rows_wg = 32 * a.row_waves, log2 = __builtin_ctz((unsigned)rows_wg);
  const int rows_per_wg = 256 / (a.head_dim / (a.bf16 ? 8 : 4));
  const dim3 grid(a.split_tiles * a.n_kv_heads * (rows_wg / rows_per_wg)), block(256);
  const bool few = a.parts <= 4;
  if (a.bf16) {
    if (few) hipLaunchKernelGGL((prompt_merge_kernel<bf16_t, true, 4>), grid, block, 0, s, a, log2);
    else hipLaunchKernelGGL((prompt_merge_kernel<bf16_t, true, 8>), grid, block, 0, s, a, log2);
  } else {
    if (few) hipLaunchKernelGGL((prompt_merge_kernel<float, false, 4>), grid, block, 0, s, a, log2);
    else hipLaunchKernelGGL((prompt_merge_kernel<float, false, 8>), grid, block, 0, s, a, log2);
  }
  return hipGetLastError();
}

hipError_t launch_prefix_merge(const PrefixArgs& a, hipStream_t s) {
  const dim3 grid((a.batch * a.n_q_heads * a.n_q + 3) / 4), block(256);
  const bool wide = a.head_dim == 128;
  if (a.bf16 && wide) hipLaunchKernelGGL((prefix_merge_kernel<bf16_t, true, 128>), grid, block, 0, s, a);
  else if (a.bf16) hipLaunchKernelGGL((prefix_merge_kernel<bf16_t, true, 64>), grid, block, 0, s, a);
  else if (wide) hipLaunchKernelGGL((prefix_merge_kernel<float, false, 128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((prefix_merge_kernel<float, false, 64>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_merge(const PagedArgs& a, hipStream_t s) {
  const bool wide = a.head_dim == 128;
  if (a.bf16) wide ? launch_paged_merge_t<bf16_t, true, 128>(a, s) : launch_paged_merge_t<bf16_t, true, 64>(a, s);
  else wide ? launch_paged_merge_t<float, false, 128>(a, s) : launch_paged_merge_t<float, false, 64>(a, s);
  return hipGetLastError();
}

hipError_t launch_merge(const MergeArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return a.bf16 ? launch_merge_t<bf16_t, true>(a, s) : launch_merge_t<float, false>(a, s);
}

}  // namespace infllm
