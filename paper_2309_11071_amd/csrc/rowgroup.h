// Rows that a group of lanes holds in registers (layer norm and root-mean-square norm): where a lane's vectors stand in a row, and
// sums and maxima over the group.
#pragma once
#include "head.h"

namespace ink {

constexpr int kWideThreads = 1024;         // rows that a wave does not hold: one workgroup a row

template <int L> constexpr int norm_threads() { return L > kWave ? L : kHeadThreads; }

// This lane's place in a row: vector i starts at element `at`, its first `skip` elements belong to the vector before.
template <int L, int V, bool FULL> struct NormPlace {
  int q, cols;
  __device__ __forceinline__ NormPlace(int cols_) : q(threadIdx.x % L), cols(cols_) {}
  __device__ __forceinline__ int first(int i) const { return (i * L + q) * V; }
  __device__ __forceinline__ int at(int i) const { return FULL ? first(i) : min(first(i), cols - V); }
  __device__ __forceinline__ bool live(int i, int j) const { return FULL || at(i) + j >= first(i); }
  __device__ __forceinline__ bool any(int i) const { return FULL || first(i) < cols; }
};

template <int L> __device__ __forceinline__ float row_sum(float x, float *s) {
  if constexpr (L > kWave) return block_sum<L>(x, s);
  else return group_sum<L>(x);
}

// Partial rows [n_part][stride] to a sum of `cols` columns: 32 columns a workgroup, 32 threads a column, in the partial rows' order.
__device__ __forceinline__ void sum_partial_rows(const float *part, int n_part, int64_t stride, int cols, int type, void *out) {
  __shared__ float s[32][33];
  const int x = threadIdx.x % 32, y = threadIdx.x / 32, c = blockIdx.x * 32 + x;
  float t = 0.f;
  if (c < cols)
#pragma unroll 8
    for (int i = y; i < n_part; i += 32) t += part[i * stride + c];
  s[y][x] = t;
  __syncthreads();
  if (y) return;
  t = 0.f;
#pragma unroll
  for (int i = 0; i < 32; i++) t += s[i][x];
  if (c < cols) store_any(out, c, type, t);
}

}  // namespace ink
