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

// Threads of a team and groups of each for rows of d: as few threads as hold
// the row in four groups each.
inline int team_of(int d) { return d <= 1024 ? 32 : d <= 2048 ? 64 : d <= 8192 ? 256 : 1024; }

}  // namespace layup
