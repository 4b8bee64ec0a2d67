// What the LayerNorm kernels share: the team of threads that holds a row.
#pragma once
#include "rowvec.h"

namespace layup {

// A team of TPR threads takes a row, thread t its groups t, t + TPR, ... of
// eight columns, all of them in registers (at most NV).
//
// Sums over the team: inside a wave by exchanges, across waves through LDS;
// every thread of the team gets the same value.
template <int TPR>
__device__ __forceinline__ void team_sum2(float& a, float& b, float* red /* 2 * TPR / 64 floats */) {
  a = lanes_sum<(TPR < 64 ? TPR : 64)>(a);
  b = lanes_sum<(TPR < 64 ? TPR : 64)>(b);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      red[w] = a;
      red[W + w] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      a += red[i];
      b += red[W + i];
    }
  }
}

constexpr int threads_of(int tpr) { return tpr > 256 ? tpr : 256; }

// Threads of a team: as few as hold the row in four groups each (in one from
// 1024 columns on: 64 threads and four groups took 5.1 us for one row of 1237
// and 15.1 for 4096, 256 threads 3.5 and 15.5), and the next larger team where
// rows are few, which shortens what a thread does one after another (768
// columns: 1 row 3.8 -> 3.0 us, 512 rows 4.3 -> 4.0, 1003 rows 4.6 -> 4.8).
inline int team_of(int64_t rows, int d) {
  if (d <= 1024) return d > 256 && rows <= 768 ? 256 : 32;
  if (d <= 2048) return 256;
  if (d <= 8192) return rows <= 128 ? 1024 : 256;
  return 1024;
}

}  // namespace layup
