// Norms and rotation of query and key rows, and the append of keys and values to their
// pages (infllm_rotate, infllm_paged_append).
//
// y = x / sqrt(mean x^2 + eps) * w, then each pair (a, b) of the rotated dims becomes
// m (a cos f - b sin f, a sin f + b cos f) with f = p * theta: 16 bytes of a row per lane,
// D * sizeof(T) / 16 lanes a row, so that a wave has two to eight rows at a time.  A wave
// keeps to one token: each lane forms the sine and cosine of one pair (in float64, reduced
// to half a revolution there; the function's own cost is one lane's), which all rows of
// the token then share.  In float32, rounded once.
#include "paged.h"

namespace infllm {
namespace {

constexpr int kRotWaves = 4;
constexpr int kRotAhead = 4;  // row groups whose loads are in flight

template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  __device__ static void unpack(const u32x4& w, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  __device__ static u32x4 pack(const float (&x)[N]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(x[2 * i]) | ((uint32_t)f32_to_bf16(x[2 * i + 1]) << 16);
    return w;
  }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  __device__ static void unpack(const u32x4& w, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
  __device__ static u32x4 pack(const float (&x)[N]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
    return w;
  }
};

// This wave's LDS writes before it are seen by its reads after it.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

template <typename T, int D, bool PAGED>
__global__ void __launch_bounds__(64 * kRotWaves) rotate_kernel(RotateArgs a) {
  constexpr int N = Piece<T>::N, LPR = D / N, RPP = 64 / LPR;
  __shared__ __attribute__((aligned(16))) float2 trig[kRotWaves][D / 2];
  __shared__ __attribute__((aligned(16))) float rows[kRotWaves][RPP][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x * kRotWaves + wave;
  const int token = div_by(item, a.d_split);
  if (token >= a.n_tokens) return;  // (no barrier of the workgroup follows)
  const int64_t t = (int64_t)a.first_token + token;
  const int r_begin = (item - token * (int)a.d_split.d) * a.rows_wave;
  const int r_end = min(a.n_q + a.n_k + a.n_v, r_begin + a.rows_wave);
  int64_t pos;
  int page = 0, slot = 0;
  if constexpr (PAGED) {
    const int s = paged_seq_of(a.seqs, (int)t);
    const int at = a.seqs.past[s] + ((int)t - a.seqs.start[s]);
    const int x = div_by(at, a.seqs.d_page);
    slot = at - x * a.seqs.page_size;
    page = a.seqs.table[s * a.seqs.table_stride + x];
    pos = at;
  } else {
    pos = a.positions != nullptr ? a.positions[t] : (int64_t)((uint64_t)a.first_position + (uint64_t)t);
  }
  const bool there = !PAGED || (page >= 0 && page < a.seqs.n_pages);

  const int half = a.rotary_dim >> 1;
  if (lane < half) {
    double f = (double)pos * a.rev[lane];
    f -= rint(f);
    double s, c;
    sincospi(2.0 * f, &s, &c);
    trig[wave][lane] = make_float2((float)(c * a.magnitude), (float)(s * a.magnitude));
  }
  wave_lds_order();
  // This lane's elements: the factor of its own value and of its partner's, and where the
  // partner lies.
  const int d0 = (lane % LPR) * N;
  float c[N], s[N];
  int mate[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int d = d0 + e;
    const bool turned = d < a.rotary_dim, first = a.interleaved ? (e & 1) == 0 : d < half;
    const int pair = !turned ? 0 : a.interleaved ? d >> 1 : first ? d : d - half;
    const float2 cs = turned ? trig[wave][pair] : make_float2(1.f, 0.f);
    c[e] = cs.x;
    s[e] = first ? -cs.y : cs.y;
    mate[e] = first ? d + half : d - half;
  }
  const bool whole = a.rotary_dim == D;              // every dim turns
  const bool by_piece = half % N == 0;               // a piece's partners are a piece
  const bool exchange = a.rotary_dim > 0 && !a.interleaved;
  float* const my_row = rows[wave][lane / LPR];

  for (int r0 = r_begin; r0 < r_end; r0 += kRotAhead * RPP) {
    u32x4 raw[kRotAhead];
#pragma unroll
    for (int j = 0; j < kRotAhead; ++j) {
      const int r = r0 + j * RPP + lane / LPR;
      if (r >= r_end) continue;
      const T* from = r < a.n_q             ? (const T*)a.q + t * a.q_tok + r * a.q_head
                      : r < a.n_q + a.n_k ? (const T*)a.k + t * a.kv_tok + (r - a.n_q) * a.kv_head
                                          : (const T*)a.v + t * a.kv_tok + (r - a.n_q - a.n_k) * a.kv_head;
      raw[j] = *(const u32x4*)(from + d0);
    }
#pragma unroll
    for (int j = 0; j < kRotAhead; ++j) {
      if (r0 + j * RPP >= r_end) break;  // (uniform)
      const int r = r0 + j * RPP + lane / LPR;
      const bool is_q = r < a.n_q, is_v = r >= a.n_q + a.n_k;
      float x[N];
      Piece<T>::unpack(raw[j], x);
      if (a.norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor(ss, o);
        const float scale = 1.f / sqrtf(ss * (1.f / D) + a.eps);
        const T* w = (const T*)(is_q ? a.q_weight : a.k_weight);
        float wf[N];
        if (w != nullptr) {
          Piece<T>::unpack(*(const u32x4*)(w + d0), wf);
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = x[e] * scale * wf[e];
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] *= scale;
        }
      }
      float y[N];
      if (exchange) {
        wave_lds_order();  // (the group before has been read)
#pragma unroll
        for (int e = 0; e < N; e += 4) *(f32x4*)(my_row + d0 + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        wave_lds_order();
        float m[N];
        if (by_piece) {
          const int at = d0 < a.rotary_dim ? mate[0] : d0;
#pragma unroll
          for (int e = 0; e < N; e += 4) *(f32x4*)(m + e) = *(const f32x4*)(my_row + at + e);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) m[e] = my_row[d0 + e < a.rotary_dim ? mate[e] : d0 + e];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[e] * c[e] + m[e] * s[e];
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[e] * c[e] + x[e ^ 1] * s[e];
      }
      if (!whole) {  // (an infinity times 0 is not the value as it was)
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = d0 + e < a.rotary_dim ? y[e] : x[e];
      }
      if (r >= r_end || (!is_q && !there)) continue;
      T* to;
      if (is_q) to = (T*)a.q_out + t * a.qo_tok + r * a.qo_head;
      else if constexpr (PAGED)
        to = (T*)(is_v ? a.v_out : a.k_out) + page * a.page_stride + slot * a.ko_tok + (r - a.n_q - (is_v ? a.n_k : 0)) * a.ko_head;
      else to = (T*)a.k_out + t * a.ko_tok + (r - a.n_q) * a.ko_head;
      *(u32x4*)(to + d0) = is_v ? raw[j] : Piece<T>::pack(y);
    }
  }
}

template <typename T, int D>
void launch_d(const RotateArgs& a, int wgs, hipStream_t s) {
  if (a.paged) hipLaunchKernelGGL((rotate_kernel<T, D, true>), dim3(wgs), dim3(64 * kRotWaves), 0, s, a);
  else hipLaunchKernelGGL((rotate_kernel<T, D, false>), dim3(wgs), dim3(64 * kRotWaves), 0, s, a);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& args, hipStream_t s) {
  RotateArgs a = args;
  const int rows = a.n_q + a.n_k + a.n_v, rpp = 64 / (a.head_dim / (a.bf16 ? 8 : 4));
  const int groups = (rows + rpp - 1) / rpp;
  // few tokens: their rows over several waves, until the chip has some 2,048
  const int split = max(1, min(groups, 2048 / max(1, a.n_tokens)));
  const int groups_wave = (groups + split - 1) / split;
  a.rows_wave = groups_wave * rpp;
  const int waves = (groups + groups_wave - 1) / groups_wave;
  a.d_split = fast_div(waves);
  const int wgs = (int)(((int64_t)a.n_tokens * waves + kRotWaves - 1) / kRotWaves);
  if (a.bf16) a.head_dim == 128 ? launch_d<bf16_t, 128>(a, wgs, s) : launch_d<bf16_t, 64>(a, wgs, s);
  else a.head_dim == 128 ? launch_d<float, 128>(a, wgs, s) : launch_d<float, 64>(a, wgs, s);
  return hipGetLastError();
}

}  // namespace infllm
