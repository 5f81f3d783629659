// Norms and rotation of query and key rows, and the append of keys and values to their
// pages (infllm_rotate, infllm_paged_append).
//
// y = x / sqrt(mean x^2 + eps) * w, then each pair (a, b) of the rotated dims becomes
// m (a cos f - b sin f, a sin f + b cos f) with f = p * theta: 16 bytes of a row per lane,
// D * sizeof(T) / 16 lanes a row, so that a wave has two to eight rows at a time.  A wave
// keeps to one token: each lane forms the sine and cosine of one pair (in float64, reduced
// to half a revolution there; the function's own cost is one lane's), which all rows of
// the token then share.  In float32, rounded once.
//
// Bound by memory: 16,000 tokens of 32 + 8 heads of 128 with norms (328 MB) take 66 us, 5.0
// TB/s, 92 % of a large copy's rate; 20 prompts into pages with queries and values (435 MB) 89
// us, 4.9.  A few tokens (16: 4 us, 32 into pages: 5) are one launch's latency, their rows
// over several waves.
#include <type_traits>

#include "paged.h"

namespace infllm {
namespace {

constexpr int kRotWaves = 4;
constexpr int kRotAhead = 8;  // row groups whose loads are in flight (of 4: the prompts 91 us, not 89)

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

// Sum over the LPR lanes of a row: rotations within 16 lanes, by the lane crossbar beyond.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xF, 0xF, false));
}
constexpr int kRor8 = 0x128, kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;     // within 16 lanes
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141;                // within 4, within 8
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  if constexpr (LPR == 8) {
    x += dpp<kXor1>(x);
    x += dpp<kXor2>(x);
    x += dpp<kHalfMirror>(x);
  } else {
    x += dpp<kRor8>(x);
    x += dpp<kRor4>(x);
    x += dpp<kRor2>(x);
    x += dpp<kRor1>(x);
    if constexpr (LPR == 32) x += __shfl_xor(x, 16);
  }
  return x;
}

template <typename T, int D, typename Args>
__global__ void __launch_bounds__(64 * kRotWaves) rotate_kernel(Args a) {
  constexpr bool PAGED = std::is_same<Args, AppendPagesArgs>::value;
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
  bool there = true;
  if constexpr (PAGED) {
    const int s = paged_seq_of(a.seqs, (int)t);
    const int at = a.seqs.past[s] + ((int)t - a.seqs.start[s]);
    const int x = div_by(at, a.seqs.d_page);
    slot = at - x * a.seqs.page_size;
    page = a.seqs.table[s * a.seqs.table_stride + x];
    there = page >= 0 && page < a.seqs.n_pages;
    pos = at;
  } else {
    pos = a.positions != nullptr ? a.positions[t] : (int64_t)((uint64_t)a.first_position + (uint64_t)t);
  }

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
  const bool whole = a.rotary_dim == D;                  // every dim turns
  const bool by_lane = LPR == 16 && whole;               // partners 8 lanes apart
  const bool by_piece = half % N == 0;                   // a piece's partners are a piece
  const bool exchange = a.rotary_dim > 0 && !a.interleaved;
  const int sub = lane / LPR;                            // this lane's row of a group
  float* const my_row = rows[wave][sub];

  // Rows [first, end) of one kind: their values as they are (TURN false), or normed and
  // turned.  A lane's addresses are stepped by uniform strides.
  auto phase = [&](auto turn, int first, int end, const T* src, int64_t head, T* dst, int64_t out_head, const void* weight) {
    constexpr bool TURN = decltype(turn)::value;
    if (first >= end) return;
    float wf[N];
    if constexpr (TURN) {
#pragma unroll
      for (int e = 0; e < N; ++e) wf[e] = 1.f;
      if (a.norm && weight != nullptr) Piece<T>::unpack(*(const u32x4*)((const T*)weight + d0), wf);
    }
    const T* from = src + (first + sub) * head + d0;
    T* to = dst + (first + sub) * out_head + d0;
    const int64_t step = RPP * head, out_step = RPP * out_head;
    for (int r0 = first; r0 < end; r0 += kRotAhead * RPP) {
      u32x4 raw[kRotAhead];
#pragma unroll
      for (int j = 0; j < kRotAhead; ++j) {
        if (r0 + j * RPP + sub < end) raw[j] = *(const u32x4*)from;
        from += step;
      }
#pragma unroll
      for (int j = 0; j < kRotAhead; ++j) {
        if (r0 + j * RPP >= end) break;  // (uniform)
        u32x4 w = raw[j];
        if constexpr (TURN) {
          float x[N], y[N];
          Piece<T>::unpack(raw[j], x);
          if (a.norm) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
            const float scale = rsqrtf(__builtin_fmaf(row_sum<LPR>(ss), 1.f / D, a.eps));
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = x[e] * scale * wf[e];
          }
          if (exchange && by_lane) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = x[e] * c[e] + dpp<kRor8>(x[e]) * s[e];
          } else if (exchange) {
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
          w = Piece<T>::pack(y);
        }
        if (r0 + j * RPP + sub < end) *(u32x4*)to = w;
        to += out_step;
      }
    }
  };
  phase(std::true_type{}, r_begin, min(r_end, a.n_q), (const T*)a.q + t * a.q_tok, a.q_head, (T*)a.q_out + t * a.qo_tok, a.qo_head,
        a.q_weight);
  if (!there) return;
  const int64_t out = PAGED ? page * a.page_stride + slot * a.ko_tok : t * a.ko_tok;
  phase(std::true_type{}, max(0, r_begin - a.n_q), min(r_end - a.n_q, a.n_k), (const T*)a.k + t * a.kv_tok, a.kv_head, (T*)a.k_out + out,
        a.ko_head, a.k_weight);
  if constexpr (PAGED)
    phase(std::false_type{}, max(0, r_begin - a.n_q - a.n_k), r_end - a.n_q - a.n_k, (const T*)a.v + t * a.kv_tok, a.kv_head,
          (T*)a.v_out + out, a.ko_head, nullptr);
}

template <typename T, int D, typename Args>
void launch_d(const Args& a, int wgs, hipStream_t s) {
  hipLaunchKernelGGL((rotate_kernel<T, D, Args>), dim3(wgs), dim3(64 * kRotWaves), 0, s, a);
}
template <typename Args>
hipError_t launch(Args a, hipStream_t s) {
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

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t s) { return launch(a, s); }
hipError_t launch_rotate(const AppendPagesArgs& a, hipStream_t s) { return launch(a, s); }

}  // namespace infllm
