// The position table of the attention kernel with four waves a workgroup: a window of
// tiles of a part [t_begin, t_end), which moves along where the part is longer.
#pragma once
#include <hip/hip_runtime.h>

namespace infllm {

// The tile whose load offsets step t forms: three ahead, so that its loads can be issued
// two steps before its use.  What runs ahead of the part's end takes its last tile again:
// its keys come from the cache and are not used (parts of four tiles would otherwise read
// three from memory that they do not need).
constexpr int kRowsAhead = 3;
__host__ __device__ inline int offsets_tile(int tile, int t_end) { return tile < t_end ? tile : t_end - 1; }
// Whether step t needs the window moved, to begin at tile t + kRowsAhead, given the one of
// `window` tiles from w0 on.  Not where that tile is past the part's end: the table holds
// the last tile then, as it did for the step before.
__host__ __device__ inline bool window_moves(int t, int t_end, int w0, int window) {
  return t + kRowsAhead >= w0 + window && t + kRowsAhead < t_end;
}

}  // namespace infllm
