// Host-side checks and small arithmetic that the entry points of the C ABI share.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <cstring>

#include "../../include/infllm.h"
#include "launch.h"

namespace infllm {

constexpr int kMaxDevices = 64;
inline std::atomic<int> g_device_ok[kMaxDevices];  // 0 unknown, 1 gfx950, 2 unusable

inline infllm_status check_device() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    (void)hipGetLastError();
    return INFLLM_E_DEVICE;
  }
  int st = g_device_ok[dev].load(std::memory_order_relaxed);
  if (st == 0) {
    hipDeviceProp_t prop;
    st = 2;
    if (hipGetDeviceProperties(&prop, dev) == hipSuccess && std::strncmp(prop.gcnArchName, "gfx950", 6) == 0)
      st = 1;
    (void)hipGetLastError();
    g_device_ok[dev].store(st, std::memory_order_relaxed);
  }
  return st == 1 ? INFLLM_OK : INFLLM_E_DEVICE;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int esize(const infllm_params* p) { return p->dtype == INFLLM_BF16 ? 2 : 4; }

inline infllm_status check_params(const infllm_params* p) {
  if (p == nullptr) return INFLLM_E_NULL;
  if (p->n_q_heads <= 0 || p->n_kv_heads <= 0 || p->n_q_heads % p->n_kv_heads != 0) return INFLLM_E_SHAPE;
  if (p->dtype != INFLLM_F32 && p->dtype != INFLLM_BF16) return INFLLM_E_SHAPE;
  if (p->head_dim <= 0) return INFLLM_E_SHAPE;
  if (p->head_dim != 64 && p->head_dim != 128) return INFLLM_E_UNSUPPORTED;
  if (p->n_init < 0 || p->n_local < 1 || p->block_size < 1 || p->topk < 0) return INFLLM_E_SHAPE;
  if (p->block_size > 256) return INFLLM_E_UNSUPPORTED;
  if (p->n_repr < 1 || p->n_repr > p->block_size) return INFLLM_E_SHAPE;
  if (!std::isfinite(p->sm_scale) || !(p->sm_scale > 0.f)) return INFLLM_E_SHAPE;
  if (p->repr_mode != INFLLM_REPR_TOKENS && p->repr_mode != INFLLM_REPR_MEAN) return INFLLM_E_SHAPE;
  if (p->rope_inv_freq != nullptr) {
    for (int i = 0; i < p->head_dim / 2; ++i)
      if (!std::isfinite(p->rope_inv_freq[i]) || p->rope_inv_freq[i] < 0.0) return INFLLM_E_SHAPE;
  }
  return INFLLM_OK;
}

inline bool remap(const infllm_params* p) { return p->rope_inv_freq != nullptr; }
// Units scored by their mean key: no representative scores, so no query ring.
inline bool mean_repr(const infllm_params* p) { return p->repr_mode == INFLLM_REPR_MEAN; }

inline infllm_status check_store(const infllm_params* p, const infllm_memory* m) {
  if (m == nullptr || m->k == nullptr || m->v == nullptr) return INFLLM_E_NULL;
  if (m->batch < 1 || m->capacity < 1) return INFLLM_E_SHAPE;
  if (!aligned16(m->k) || !aligned16(m->v)) return INFLLM_E_SHAPE;
  if (remap(p)) {
    if (m->k_rot == nullptr) return INFLLM_E_NULL;
    if (!aligned16(m->k_rot)) return INFLLM_E_SHAPE;
  }
  return INFLLM_OK;
}

inline infllm_status check_units(const infllm_params* p, const infllm_memory* m) {
  if ((m->repr_idx == nullptr && !mean_repr(p)) || m->unit_ksum == nullptr) return INFLLM_E_NULL;
  if (m->max_units < 0) return INFLLM_E_SHAPE;
  if (!aligned16(m->unit_ksum)) return INFLLM_E_SHAPE;
  return INFLLM_OK;
}

// Rows of `n_q` tokens per head with stride `head_stride` elements, read as 16-byte vectors.
inline infllm_status check_rows(const infllm_params* p, const void* ptr, int64_t head_stride, int32_t n_q) {
  if (ptr == nullptr) return INFLLM_E_NULL;
  if (head_stride < (int64_t)n_q * p->head_dim) return INFLLM_E_SHAPE;
  if (((head_stride * esize(p)) & 15) != 0 || !aligned16(ptr)) return INFLLM_E_SHAPE;
  return INFLLM_OK;
}

struct Part {
  int64_t n_init, local_begin;
  int32_t n_units;
};
inline Part partition(const infllm_params* p, int64_t past_len) {
  Part r;
  r.n_init = past_len < p->n_init ? past_len : p->n_init;
  const int64_t evicted = past_len - p->n_init - p->n_local;
  const int64_t nu = evicted > 0 ? evicted / p->block_size : 0;
  r.n_units = (int32_t)(nu > INT32_MAX ? INT32_MAX : nu);
  r.local_begin = r.n_init + nu * p->block_size;
  return r;
}

// Workspace bytes of one part's partial row: fp16 values, lse and exponent for
// bf16 inputs; float32 values and lse for float32 inputs.
inline size_t part_row_bytes(const infllm_params* p) {
  return p->dtype == INFLLM_BF16 ? (size_t)p->head_dim * 2u + 8u : (size_t)(p->head_dim + 1) * 4u;
}

inline size_t attend_ws_bytes(const infllm_params* p, int32_t batch, int32_t n_q, int parts) {
  const int64_t rows = (int64_t)batch * p->n_q_heads * n_q;
  return (size_t)parts * (size_t)rows * part_row_bytes(p);
}

// Partial arrays inside the workspace: [parts][rows][D] values, then [parts][rows]
// lse, then (bf16) [parts][rows] exponents.
inline void partial_layout(const infllm_params* p, void* workspace, int parts, int64_t rows, void** o, float** lse,
                    int32_t** ex) {
  const size_t vbytes = (size_t)parts * (size_t)rows * (size_t)p->head_dim * (p->dtype == INFLLM_BF16 ? 2u : 4u);
  char* w = (char*)workspace;
  *o = w;
  *lse = w ? (float*)(w + vbytes) : nullptr;
  *ex = (w && p->dtype == INFLLM_BF16) ? (int32_t*)(w + vbytes + (size_t)parts * (size_t)rows * 4u) : nullptr;
}

inline size_t qbar_ws_bytes(const infllm_params* p, int32_t batch, int32_t n_q) {
  const int G = p->n_q_heads / p->n_kv_heads;
  return (size_t)batch * p->n_kv_heads * score_qbar_parts(G, n_q) * p->head_dim * 4u;
}

inline infllm_status launch_status(hipError_t e) {
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return INFLLM_E_LAUNCH;
  }
  return INFLLM_OK;
}

inline MergeArgs merge_args(const infllm_params* p, int32_t batch, int32_t n_q, int32_t n_parts, const void* workspace,
                     void* out, int64_t out_head_stride, float* lse) {
  MergeArgs ma;
  const int64_t rows = (int64_t)batch * p->n_q_heads * n_q;
  ma.rows = (int)rows;
  ma.head_dim = p->head_dim;
  ma.parts = n_parts;
  ma.n_q = n_q;
  ma.n_q_heads = p->n_q_heads;
  ma.out_head_stride = out_head_stride;
  void* po;
  float* pl;
  int32_t* pe;
  partial_layout(p, const_cast<void*>(workspace), n_parts, rows, &po, &pl, &pe);
  ma.part_o = po;
  ma.part_lse = pl;
  ma.part_exp = pe;
  ma.out = out;
  ma.lse = lse;
  ma.bf16 = p->dtype == INFLLM_BF16;
  return ma;
}

}  // namespace infllm
