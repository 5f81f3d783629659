// Copies of whole sequences between memories of a layer (forking a document's memory to
// several batch slots, closing up a batch from which sequences have finished).
//
// Nothing is computed: the floor is each source byte read once and each copy's bytes
// written once, and the memory's rate bounds it.  The pairs come sorted by source; a
// workgroup takes 32 KB of one source (2,048 pieces of 16 bytes, eight loads per thread in
// flight), and stores them to every copy of it.  One launch for all arrays and pairs: the
// blocks of a source run through its K, V (and rotated K) rows, then its rings, key sums
// and representatives.  Four copies of a memory of 131,072 tokens (2.95 GB read and
// written): 565 us, 5.22 TB/s, a large copy's rate; three sequences of 1,500 to 9,001
// tokens (0.32 GB) 63 us.
#include "shared.h"

namespace infllm {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                        // pieces per thread
constexpr int kPieces = kThreads * kPer;       // pieces per workgroup

// Blocks of the roles of a source.
struct Roles {
  int stores, per_row, store, qprefix, rpart, ksum, repr;
};
__host__ __device__ inline int blocks_of(int64_t pieces) { return (int)((pieces + kPieces - 1) / kPieces); }
__host__ __device__ inline Roles roles(const SeqCopyArgs& a, int64_t len, int built, int held) {
  Roles r;
  r.stores = a.src_rot != nullptr ? 3 : 2;
  r.per_row = blocks_of(len * (a.row_bytes / 16));
  r.store = r.stores * a.n_kv_heads * r.per_row;
  r.qprefix = a.ring_rows > 0 ? blocks_of((int64_t)a.n_kv_heads * held * (a.cells * 2)) : 0;
  r.rpart = a.ring_rows > 0 ? blocks_of((int64_t)a.n_kv_heads * a.ring_rows * held) : 0;
  r.ksum = blocks_of((int64_t)a.n_kv_heads * a.cells * built);
  r.repr = a.repr_bytes > 0 ? blocks_of((int64_t)a.n_kv_heads * built * (a.repr_bytes / 4)) : 0;
  return r;
}
// Ring slots that a copy of `len` positions carries: its last ones.
__host__ __device__ inline int held_slots(const SeqCopyArgs& a, int64_t len) {
  const int ring = a.src_ring < a.dst_ring ? a.src_ring : a.dst_ring;
  return len < ring ? (int)len : ring;
}

// `rows` rows of `per_row` elements of type V, element (row, col) at base(row) + col; the
// pair's own length of a row is limit(pair).
template <typename V, typename Src, typename Dst, typename Limit>
__device__ __forceinline__ void copy_rows(int64_t first, int64_t total, int per_row, int p0, int p1, Src src, Dst dst,
                                          Limit limit) {
  V x[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int64_t e = first + j * kThreads;
    const uint32_t c = (uint32_t)min(e, total - 1), row = c / (uint32_t)per_row;
    x[j] = *src((int)row, (int)(c - row * (uint32_t)per_row));
  }
  for (int p = p0; p < p1; ++p) {
    const int lim = limit(p);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int64_t e = first + j * kThreads;
      const uint32_t c = (uint32_t)min(e, total - 1), row = c / (uint32_t)per_row, col = c - row * (uint32_t)per_row;
      if (e < total && (int)col < lim) *dst(p, (int)row, (int)col) = x[j];
    }
  }
}

__global__ void __launch_bounds__(kThreads) copy_sequences_kernel(SeqCopyArgs a) {
  // the source this block belongs to
  int s;
  {
    const int lane = threadIdx.x & 63;
    s = __popcll(__ballot(lane < a.n_sources && a.block_begin[lane] <= (int)blockIdx.x)) - 1;
    s = __builtin_amdgcn_readfirstlane(s);
  }
  int blk = (int)blockIdx.x - a.block_begin[s];
  const int p0 = a.pair_begin[s], p1 = a.pair_begin[s + 1];
  int64_t len = 0;
  int built = 0;
  for (int p = p0; p < p1; ++p) {
    len = max(len, a.len[p]);
    built = max(built, a.built[p]);
  }
  const int held = held_slots(a, len), H = a.n_kv_heads, from = a.src_seq[s];
  const Roles r = roles(a, len, built, held);
  const int tid = threadIdx.x;
  if (blk < r.store) {
    const int row = blk / r.per_row, chunk = blk - row * r.per_row;
    const int which = row / H, h = row - which * H;
    const char* src = which == 0 ? a.src_k : which == 1 ? a.src_v : a.src_rot;
    char* dst = which == 0 ? a.dst_k : which == 1 ? a.dst_v : a.dst_rot;
    src += ((int64_t)from * H + h) * a.src_capacity * a.row_bytes;
    const int64_t first = (int64_t)chunk * kPieces + tid, total = len * (a.row_bytes / 16);
    u32x4 x[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = *(const u32x4*)(src + 16 * min(first + j * kThreads, total - 1));
    for (int p = p0; p < p1; ++p) {
      char* to = dst + ((int64_t)a.dst_seq[p] * H + h) * a.dst_capacity * a.row_bytes;
      const int64_t end = a.len[p] * (a.row_bytes / 16);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (first + j * kThreads < end) *(u32x4*)(to + 16 * (first + j * kThreads)) = x[j];
    }
    return;
  }
  blk -= r.store;
  if (blk < r.qprefix + r.rpart) {
    // Ring slots by position: the last `held` positions of each copy, slot position mod
    // ring on either side.  Copies of one length share the loads.
    const bool prefix = blk < r.qprefix;
    const int64_t first = (int64_t)(blk - (prefix ? 0 : r.qprefix)) * kPieces + tid;
    for (int q = p0; q < p1;) {
      int q1 = q + 1;
      while (q1 < p1 && a.len[q1] == a.len[q]) ++q1;
      const int n = held_slots(a, a.len[q]);
      const int s0 = (int)((a.len[q] - n) % a.src_ring), d0 = (int)((a.len[q] - n) % a.dst_ring);
      auto wrap = [](int slot, int ring) { return slot >= ring ? slot - ring : slot; };
      if (n > 0 && prefix) {
        const int pp = a.cells * 2;  // 16-byte pieces of a slot
        copy_rows<u32x4>(
            first, (int64_t)H * n * pp, n * pp, q, q1,
            [&](int row, int col) {
              const int j = col / pp;
              return (const u32x4*)a.src_qprefix + (((int64_t)from * H + row) * a.src_ring + wrap(s0 + j, a.src_ring)) * pp + (col - j * pp);
            },
            [&](int p, int row, int col) {
              const int j = col / pp;
              return (u32x4*)a.dst_qprefix + (((int64_t)a.dst_seq[p] * H + row) * a.dst_ring + wrap(d0 + j, a.dst_ring)) * pp + (col - j * pp);
            },
            [&](int) { return n * pp; });
      } else if (n > 0) {
        const int rows = H * a.ring_rows;
        copy_rows<uint64_t>(
            first, (int64_t)rows * n, n, q, q1,
            [&](int row, int col) {
              return (const uint64_t*)a.src_rpart + ((int64_t)from * rows + row) * a.src_ring + wrap(s0 + col, a.src_ring);
            },
            [&](int p, int row, int col) {
              return (uint64_t*)a.dst_rpart + ((int64_t)a.dst_seq[p] * rows + row) * a.dst_ring + wrap(d0 + col, a.dst_ring);
            },
            [&](int) { return n; });
      }
      q = q1;
    }
    return;
  }
  blk -= r.qprefix + r.rpart;
  if (blk < r.ksum) {
    const int rows = H * a.cells;
    copy_rows<u32x4>(
        (int64_t)blk * kPieces + tid, (int64_t)rows * built, built, p0, p1,
        [&](int row, int col) { return (const u32x4*)a.src_ksum + ((int64_t)from * rows + row) * a.src_units + col; },
        [&](int p, int row, int col) { return (u32x4*)a.dst_ksum + ((int64_t)a.dst_seq[p] * rows + row) * a.dst_units + col; },
        [&](int p) { return a.built[p]; });
    return;
  }
  blk -= r.ksum;
  const int words = a.repr_bytes / 4;
  copy_rows<uint32_t>(
      (int64_t)blk * kPieces + tid, (int64_t)H * built * words, built * words, p0, p1,
      [&](int row, int col) { return (const uint32_t*)a.src_repr + ((int64_t)from * H + row) * a.src_units * words + col; },
      [&](int p, int row, int col) { return (uint32_t*)a.dst_repr + ((int64_t)a.dst_seq[p] * H + row) * a.dst_units * words + col; },
      [&](int p) { return a.built[p] * words; });
}

}  // namespace

hipError_t launch_copy_sequences(const SeqCopyArgs& args, hipStream_t s) {
  SeqCopyArgs a = args;
  int blocks = 0;
  for (int i = 0; i < a.n_sources; ++i) {
    a.block_begin[i] = blocks;
    int64_t len = 0;
    int built = 0;
    for (int p = a.pair_begin[i]; p < a.pair_begin[i + 1]; ++p) {
      len = a.len[p] > len ? a.len[p] : len;
      built = a.built[p] > built ? a.built[p] : built;
    }
    const Roles r = roles(a, len, built, held_slots(a, len));
    blocks += r.store + r.qprefix + r.rpart + r.ksum + r.repr;
  }
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(copy_sequences_kernel, dim3(blocks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace infllm
