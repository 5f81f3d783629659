// Unit relevance of a shared document (infllm_prefix_score).
#include "qsum.h"
#include "shared.h"

namespace infllm {
namespace {

// Query sums of many query rows, a launch of its own (grid: parts, batch*Hkv).
template <typename T>
__global__ void __launch_bounds__(kQsumThreads) prefix_qsum_kernel(PrefixScoreArgs a, int parts) {
  __shared__ QsumSmem<T> sm;
  qsum_block<T>((const T*)a.q, a.q_head_stride, a.n_q_heads, a.n_kv_heads, a.head_dim, a.n_q, blockIdx.x, parts,
                blockIdx.y, a.qbar_parts, sm);
}

// Relevance of one memory's units to every continuation of it: the product of the
// continuations' query sums [B][D] and the key sums [D][units], float32 on the matrix
// cores (v_mfma_f32_16x16x4_f32), 16 continuations by 16 units at a time.  A wave holds
// the key sums of 32 units, which are so read once whatever the batch: lane (n, kg) the
// cells 4 s + kg of unit n, whose four dims feed four products.  The block's query sums
// go through LDS, row m to the lanes (m, kg); they are formed there from up to
// kPrefixSumRows query rows each, which each block reads again, or from the partial sums
// that a launch before leaves (S = float, n_q = 1, one head).  Bound by the
// memory and one round trip to it: 16 continuations by 8,155 units of 8 heads (33 MB of
// key sums, 4 MB of scores) 9.1 us, 4.1 TB/s; 4 by 217 units 4.4 us.  (With the products
// on the vector ALU and the query sums in a launch before, the calls took 16.4 and 10.5 us;
// now 10.1 and 7.3.)
constexpr int kPrefixSumRows = 16;
template <typename S, int D>
__global__ void __launch_bounds__(256) prefix_score_kernel(const PrefixScoreArgs a, const S* q, int64_t seq_stride, int64_t group_stride,
                                                           int64_t row_stride, int n_q, int rows) {
  constexpr int CELLS = D / 4, STEPS = CELLS / 4, UT = 2, PAIRS = 16 * D / 2 / 256, RB = 4;
  __shared__ __attribute__((aligned(16))) float sums[16][D + 4];
  const int g = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = lane & 15, kg = lane >> 4;
  const int u0 = ((int)blockIdx.x * 4 + wave) * 16 * UT;
  const f32x4* ks = (const f32x4*)a.unit_ksum + (int64_t)g * CELLS * a.max_units;
  f32x4 k4[UT][STEPS];
#pragma unroll
  for (int t = 0; t < UT; ++t)
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      k4[t][s] = ks[(int64_t)(4 * s + kg) * a.max_units + min(u0 + 16 * t + n, a.n_units - 1)];
  for (int b0 = 0; b0 < a.batch; b0 += 16) {
    const int nb = min(16, a.batch - b0);
    float x[PAIRS][2] = {};
    for (int r0 = 0; r0 < rows; r0 += RB) {
      float y[PAIRS][RB][2];
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        const int r = min(r0 + j, rows - 1), h = r / n_q;
        const S* row = q + g * group_stride + h * row_stride + (int64_t)(r - h * n_q) * D;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
          const int at = tid + 256 * i, m = min(at / (D / 2), nb - 1), d = 2 * (at % (D / 2));
          const S* p = row + (b0 + m) * seq_stride + d;
          if constexpr (sizeof(S) == 2) {
            const uint32_t w = *(const uint32_t*)p;
            y[i][j][0] = __uint_as_float(w << 16);
            y[i][j][1] = __uint_as_float(w & 0xFFFF0000u);
          } else {
            const float2 w = *(const float2*)p;
            y[i][j][0] = w.x;
            y[i][j][1] = w.y;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int i = 0; i < PAIRS; ++i)
          if (r0 + j < rows) {
            x[i][0] += y[i][j][0];
            x[i][1] += y[i][j][1];
          }
    }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      const int at = tid + 256 * i;
      *(float2*)&sums[at / (D / 2)][2 * (at % (D / 2))] = make_float2(x[i][0], x[i][1]);
    }
    __syncthreads();
    f32x4 acc[UT] = {};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const f32x4 q4 = *(const f32x4*)&sums[n][16 * s + 4 * kg];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < UT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(q4[e], k4[t][s][e], acc[t], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < UT; ++t) {
      const int u = u0 + 16 * t + n;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * kg + r < nb && u < a.n_units)
          a.scores[((int64_t)(b0 + 4 * kg + r) * a.n_kv_heads + g) * a.n_units + u] = acc[t][r];
    }
    __syncthreads();
  }
}

template <typename T, int D>
void launch_prefix_score_t(const PrefixScoreArgs& a, hipStream_t s) {
  const int G = a.n_q_heads / a.n_kv_heads, rows = G * a.n_q;
  const dim3 grid((a.n_units + 127) / 128, a.n_kv_heads);
  if (rows <= kPrefixSumRows) {
    hipLaunchKernelGGL((prefix_score_kernel<T, D>), grid, dim3(256), 0, s, a, (const T*)a.q, a.n_q_heads * a.q_head_stride,
                       G * a.q_head_stride, a.q_head_stride, a.n_q, rows);
    return;
  }
  const int parts = score_qbar_parts(G, a.n_q);
  hipLaunchKernelGGL((prefix_qsum_kernel<T>), dim3(parts, a.batch * a.n_kv_heads), dim3(kQsumThreads), 0, s, a, parts);
  hipLaunchKernelGGL((prefix_score_kernel<float, D>), grid, dim3(256), 0, s, a, (const float*)a.qbar_parts,
                     (int64_t)a.n_kv_heads * parts * D, (int64_t)parts * D, (int64_t)D, 1, parts);
}

}  // namespace

hipError_t launch_prefix_score(const PrefixScoreArgs& a, hipStream_t s) {
  const bool wide = a.head_dim == 128;
  if (a.bf16) wide ? launch_prefix_score_t<bf16_t, 128>(a, s) : launch_prefix_score_t<bf16_t, 64>(a, s);
  else wide ? launch_prefix_score_t<float, 128>(a, s) : launch_prefix_score_t<float, 64>(a, s);
  return hipGetLastError();
}

}  // namespace infllm
