// eql_colsum.h -- sums over the rows of a table of partial sums, in a fixed order, for the gradients of
// per-channel parameters.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace eqk {

// A workgroup of kColsumThreads takes up to 64 columns of one kind of rows [rows][.. K ..], `step` apart, whole channels of T
// columns each; its waves add every sixteenth row, four at a time (64 of these, then the sums of so many: thousands of rows
// one after the other would lose digits), then a thread a channel adds the waves and the channel's columns.  f(channel, sum) for each.
constexpr int kColsumWidth = 64, kColsumWaves = 16, kColsumThreads = 64 * kColsumWaves;
inline int colsum_channels(int T) { return kColsumWidth / T; }  // (T <= 16)
inline int colsum_blocks(int C, int T) { return (C + colsum_channels(T) - 1) / colsum_channels(T); }

template <typename F>
__device__ __forceinline__ void column_sums(const float* part, int64_t rows, int64_t step, int C, int T, int block, F&& f) {
  __shared__ float red[kColsumWaves][kColsumWidth];
  const int per = kColsumWidth / T, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c0 = block * per, n = min(per, C - c0) * T;
  float v = 0.0f;
  if (lane < n) {
    const float* p = part + c0 * T + lane;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    int64_t r = wave;
    while (r + 3 * kColsumWaves < rows) {
      float u[4] = {0.f, 0.f, 0.f, 0.f};
      for (int i = 0; i < 64 && r + 3 * kColsumWaves < rows; ++i, r += 4 * kColsumWaves) {
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] += p[(r + kColsumWaves * k) * step];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] += u[k];
    }
    for (; r < rows; r += kColsumWaves) w[0] += p[r * step];
    v = (w[0] + w[1]) + (w[2] + w[3]);
  }
  red[wave][lane] = v;
  __syncthreads();
  if ((int)threadIdx.x < n / T) {
    float s = 0.0f;
    for (int t = 0; t < T; ++t) {
#pragma unroll
      for (int k = 0; k < kColsumWaves; ++k) s += red[k][threadIdx.x * T + t];
    }
    f(c0 + (int)threadIdx.x, s);
  }
}

}  // namespace eqk
