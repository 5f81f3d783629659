// What the kernels on paged caches take, and the arithmetic that their host and device
// sides share.
#pragma once

#include "launch.h"

namespace infllm {

constexpr int kMaxPaged = 256;  // sequences of one launch

// The sequences of a launch, packed one after another.
struct PagedSeqs {
  int n_seqs;
  int n_pages, page_size;
  FastDiv d_page;
  const int32_t* table;  // row of the launch's first sequence
  int64_t table_stride;
  int32_t start[kMaxPaged + 1];  // first new token, in the call's order; the end
  int32_t past[kMaxPaged];       // tokens before it
};

// The sequence of new token t (uniform over the wave): the last one that starts at or
// before it.  Every lane reads its sequences' entries at once.
__device__ __forceinline__ int paged_seq_of(const PagedSeqs& a, int t) {
  constexpr int CH = kMaxPaged / kWave;
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    if (j * kWave >= a.n_seqs) break;
    const int i = j * kWave + lane;
    n += __popcll(__ballot(i < a.n_seqs && a.start[i] <= t));
  }
  return __builtin_amdgcn_readfirstlane(n) - 1;
}

// Norms and rotation (and, with pages, the append).  A token has n_q query rows, n_k key
// rows and n_v value rows, in this order; a wave has `rows_wave` of them.
struct RotateArgs {
  int first_token, n_tokens;  // of this launch
  int n_q, n_k, n_v;
  int rows_wave;
  FastDiv d_split;  // waves of a token
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  void* k_out;
  void* v_out;
  int64_t q_tok, q_head, kv_tok, kv_head, qo_tok, qo_head, ko_tok, ko_head;
  int64_t page_stride;  // (with pages, ko_tok and ko_head are those within a page)
  const int64_t* positions;
  int64_t first_position;
  int rotary_dim, interleaved, norm;
  float magnitude, eps;
  const void* q_weight;
  const void* k_weight;
  int head_dim;
  bool bf16, paged;
  double rev[kMaxPairs];  // revolutions per position of pair i
  PagedSeqs seqs;
};
hipError_t launch_rotate(const RotateArgs& a, hipStream_t s);

// Attention over pages.
struct PagedArgs {
  int n_q_heads, n_kv_heads, head_dim;
  bool bf16;
  float sm_scale, softcap;
  int window, n_init;
  const float* slopes;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  int64_t q_tok, q_head, out_tok, out_head, lse_stride;
  int64_t page_stride, token_stride, head_stride;
  PagedSeqs seqs;
};
hipError_t launch_paged(const PagedArgs& a, hipStream_t s);

}  // namespace infllm
