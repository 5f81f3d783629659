// Causal attention of new tokens over paged keys and values (infllm_paged_attend).
#include "paged.h"

namespace infllm {
namespace {

// One wave per (new token, query head): 64 keys at a time, a key per lane for the scores,
// D / 64 dims per lane for the values.
template <typename T, int D>
__global__ void __launch_bounds__(256) paged_rows_kernel(PagedArgs a) {
  constexpr int DPL = D / 64;
  __shared__ float qs[4][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t first = a.seqs.start[0], tokens = a.seqs.start[a.seqs.n_seqs] - first;
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  const int64_t t = first + item / a.n_q_heads;
  const int h = (int)(item % a.n_q_heads);
  if (t >= first + tokens) return;
  const int s = paged_seq_of(a.seqs, (int)t);
  const int pos = a.seqs.past[s] + ((int)t - a.seqs.start[s]);
  const T* q = (const T*)a.q + t * a.q_tok + h * a.q_head;
  for (int d = lane; d < D; d += 64) qs[wave][d] = Elem<T>::load(q + d);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  const int64_t head = (h / (a.n_q_heads / a.n_kv_heads)) * a.head_stride;
  const float slope = a.slopes != nullptr ? a.slopes[h] : 0.f;
  const int low = a.window > 0 ? max(0, pos - a.window + 1) : 0;  // first key of the window
  float m = -__builtin_inff(), l = 0.f, acc[DPL] = {};
  for (int t0 = 0; t0 <= pos; t0 += 64) {
    if (t0 >= a.n_init && t0 + 64 <= low) {
      t0 = low / 64 * 64 - 64;
      continue;
    }
    const int key = t0 + lane;
    int64_t at = -1;
    float z = -__builtin_inff();
    if (key <= pos && (key >= low || key < a.n_init)) {
      const int x = div_by(key, a.seqs.d_page), page = a.seqs.table[s * a.seqs.table_stride + x];
      if (page >= 0 && page < a.seqs.n_pages) {
        at = page * a.page_stride + (key - x * a.seqs.page_size) * a.token_stride + head;
        float dot = 0.f;
        for (int d = 0; d < D; ++d) dot = __builtin_fmaf(qs[wave][d], Elem<T>::load((const T*)a.k + at + d), dot);
        z = dot * a.sm_scale;
        if (a.softcap > 0.f) z = a.softcap * tanhf(z / a.softcap);
        if (a.slopes != nullptr) z -= slope * (float)(pos - key);
      }
    }
    const float m_new = fmaxf(m, wave_max(z));
    const bool nan = __ballot(z != z) != 0;
    if (m_new == -__builtin_inff() && !nan) continue;
    const float corr = m == -__builtin_inff() ? 0.f : expf(m - m_new);
    const float p = at >= 0 ? expf(z - m_new) : 0.f;
    l = l * corr + wave_sum(p);
    m = m_new;
    for (int e = 0; e < DPL; ++e) acc[e] *= corr;
    for (int j = 0; j < 64; ++j) {
      const int64_t aj = __shfl(at, j);
      const float pj = __shfl(p, j);
      if (aj < 0) continue;
      for (int e = 0; e < DPL; ++e) acc[e] = __builtin_fmaf(pj, Elem<T>::load((const T*)a.v + aj + DPL * lane + e), acc[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = (T*)a.out + t * a.out_tok + h * a.out_head;
  for (int e = 0; e < DPL; ++e) Elem<T>::store(o + DPL * lane + e, acc[e] * inv);
  if (lane == 0 && a.lse != nullptr) a.lse[h * a.lse_stride + t] = l == 0.f ? -__builtin_inff() : m + logf(l);
}

template <typename T>
void launch_t(const PagedArgs& a, hipStream_t s) {
  const int64_t items = (int64_t)(a.seqs.start[a.seqs.n_seqs] - a.seqs.start[0]) * a.n_q_heads;
  const dim3 grid((unsigned)((items + 3) / 4)), block(256);
  if (a.head_dim == 128) hipLaunchKernelGGL((paged_rows_kernel<T, 128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((paged_rows_kernel<T, 64>), grid, block, 0, s, a);
}

}  // namespace

hipError_t launch_paged(const PagedArgs& a, hipStream_t s) {
  if (a.bf16) launch_t<bf16_t>(a, s);
  else launch_t<float>(a, s);
  return hipGetLastError();
}

}  // namespace infllm
