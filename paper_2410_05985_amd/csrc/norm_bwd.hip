// Backward of LayerNorm with its residual add and dropout, with the reduction of
// the weights' gradients, for any width and row distance.  Bound by HBM; every
// reduction has a fixed order.
#include "norm.h"

namespace layup {

struct BwdArgs {
  const void *dy, *s, *dsum;
  void *dres, *dx;
  const float *mean, *rstd, *gamma;
  float* part;  // partial rows of dgamma and dbeta (nullable)
  int64_t lddy, lds, lddsum, lddres, lddx, rows;
  int32_t d;
  Mask K;
};

// With h = (s - mean) rstd and g = dy gamma: ds = rstd (g - mean(g) - h
// mean(g h)) + dsum; dres = ds, dx = m scale ds.  A row stays in registers
// between its two sums and its results.  A block goes through rows at the
// grid's distance and keeps its share of dgamma and dbeta in registers; one row
// of partial sums a block goes to memory, which norm_sum_kernel adds (atomics
// would add them in another order each time).  Bound by HBM: 8192 x 8192, five
// bfloat16 streams, 132 us (5.1 TB/s) and the sums 8; 8192 x 768 with a float32
// residual stream 22 us (4.6 TB/s) and the sums 4.  The next row's loads before
// this row's sums were measured: 1237 columns 41.3 -> 37.7 us, 8192 columns 141
// -> 140, a float32 stream of 2048 columns 55 -> 56, 768 columns 22 -> 24; not kept.
// Above 8192 columns 1024 threads leave a thread 128 registers, and 20 to 47 of
// what it keeps between rows are spilled: 4096 x 12288 bfloat16 103 us without the
// sums (4.9 TB/s), 130 with them, whose partial rows are 50 MB.
// WHOLE: d is a multiple of 8.
template <class TY, class TS, class TX, int TPR, int NV, bool WHOLE>
__global__ __launch_bounds__(threads_of(TPR)) void norm_bwd_kernel(const BwdArgs P) {
  constexpr int RPB = threads_of(TPR) / TPR, WAVES = threads_of(TPR) / 64;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  const int t = threadIdx.x % TPR;
  const int d = P.d;
  const float inv_d = 1.0f / (float)d;
  const uint64_t offset = mask_offset(P.K);
  float g[NV][8], ag[NV][8], ab[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 8 * (t + TPR * j);
    Raw8<float> rg;
    if (P.gamma) load_group<WHOLE>(rg, P.gamma, c, d);
    if (P.gamma) finish_group<WHOLE>(rg, P.gamma, c, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      g[j][e] = P.gamma ? rg.get(e) : 1.f;
      ag[j][e] = ab[j][e] = 0.f;
    }
  }
  for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < P.rows; row += (int64_t)gridDim.x * RPB) {
    Raw8<TY> ry[NV];
    Raw8<TS> rs[NV], rd[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = 8 * (t + TPR * j);
      load_group<WHOLE>(ry[j], (const TY*)P.dy + row * P.lddy, c, d);
      load_group<WHOLE>(rs[j], (const TS*)P.s + row * P.lds, c, d);
      if (P.dsum) load_group<WHOLE>(rd[j], (const TS*)P.dsum + row * P.lddsum, c, d);
    }
    const float mu = P.mean[row], r = P.rstd[row];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = 8 * (t + TPR * j);
      finish_group<WHOLE>(ry[j], (const TY*)P.dy + row * P.lddy, c, d);
      finish_group<WHOLE>(rs[j], (const TS*)P.s + row * P.lds, c, d);
      if (P.dsum) finish_group<WHOLE>(rd[j], (const TS*)P.dsum + row * P.lddsum, c, d);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // behind the row's end dy is 0, so every sum takes 0
        const float y = ry[j].get(e), xh = (rs[j].get(e) - mu) * r, a = y * g[j][e];
        s1 += a;
        s2 = fmaf(a, xh, s2);
        ag[j][e] = fmaf(y, xh, ag[j][e]);
        ab[j][e] += y;
      }
    team_sum2<TPR>(s1, s2, red);
    s1 *= inv_d;
    s2 *= inv_d;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = 8 * (t + TPR * j);
      if (c >= d) continue;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = (rs[j].get(e) - mu) * r;
        o[e] = r * (ry[j].get(e) * g[j][e] - s1 - xh * s2);
        if (P.dsum) o[e] += rd[j].get(e);
      }
      if (P.dres) store_group<WHOLE>((TS*)P.dres + row * P.lddres + c, o, d - c);
      if (P.dx) {
        if (P.K.thr) drop_group(o, c >> 3, (uint32_t)row, P.K, offset);
        store_group<WHOLE>((TX*)P.dx + row * P.lddx + c, o, d - c);
      }
    }
  }
  if (!P.part) return;
  // partial row of this block: the teams of a wave, then the waves in order
  float* part = P.part + (int64_t)blockIdx.x * 2 * d;
  if constexpr (TPR < 64) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ag[j][e] += __shfl_xor(ag[j][e], 32, 64);
        ab[j][e] += __shfl_xor(ab[j][e], 32, 64);
      }
  }
  if constexpr (TPR <= 64) {
    __shared__ float acc[2][8 * TPR * NV];
    const int w = threadIdx.x >> 6;
    const bool on = (int)(threadIdx.x & 63) < TPR;
    for (int k = 0; k < WAVES; ++k) {
      if (k == w && on) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int c = 8 * (t + TPR * j) + e;
            acc[0][c] = k == 0 ? ag[j][e] : acc[0][c] + ag[j][e];
            acc[1][c] = k == 0 ? ab[j][e] : acc[1][c] + ab[j][e];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * d; c += 256) part[c] = c < d ? acc[0][c] : acc[1][c - d];
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = 8 * (t + TPR * j);
      if (c >= d) continue;
      store_group<WHOLE>(part + c, ag[j], d - c);
      store_group<WHOLE>(part + d + c, ab[j], d - c);
    }
  }
}

// dgamma and dbeta from the partial rows: a block takes 32 columns with 32 row
// lanes; lane l adds rows l, l + 32, ... in order, sixteen of them in flight,
// then the lanes are added in a fixed tree.
constexpr int SUM_COLS = 32, SUM_LANES = 32;
__global__ __launch_bounds__(SUM_COLS * SUM_LANES) void norm_sum_kernel(const float* part, int nb, int d, float* dgamma,
                                                                        float* dbeta) {
  __shared__ float red[SUM_LANES][SUM_COLS + 1];
  const int x = threadIdx.x % SUM_COLS, l = threadIdx.x / SUM_COLS, c = blockIdx.x * SUM_COLS + x;
  const int64_t ld = 2 * (int64_t)d;
  float s = 0.f;
  if (c < ld) {
    for (int r0 = l; r0 < nb; r0 += 16 * SUM_LANES) {
      float v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int r = r0 + k * SUM_LANES;
        v[k] = r < nb ? part[r * ld + c] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) s += v[k];
    }
  }
  red[l][x] = s;
  __syncthreads();
#pragma unroll
  for (int h = SUM_LANES / 2; h > 0; h >>= 1) {
    if (l < h) red[l][x] += red[l + h][x];
    __syncthreads();
  }
  if (l > 0 || c >= ld) return;
  if (c < d) {
    if (dgamma) dgamma[c] = red[0][x];
  } else {
    if (dbeta) dbeta[c - d] = red[0][x];
  }
}

// Blocks of the backward (and partial rows): two a CU.
constexpr int64_t MAX_PARTS = 512;
int64_t norm_partial_rows(int64_t rows, int d) {
  const int tpr = team_of(rows, d), rpb = threads_of(tpr) / tpr;
  return std::min<int64_t>(cdiv(rows, rpb), MAX_PARTS);
}
// Room for them, whatever the team: more rows never need less.
int64_t norm_partial_floats(int64_t rows, int d) { return std::min(rows, MAX_PARTS) * 2 * (int64_t)d; }

template <class TY, class TS, class TX, int TPR, int NV, bool WHOLE>
static hipError_t bwd_launch(const BwdArgs& P, hipStream_t s) {
  norm_bwd_kernel<TY, TS, TX, TPR, NV, WHOLE><<<(unsigned)norm_partial_rows(P.rows, P.d), threads_of(TPR), 0, s>>>(P);
  return hipGetLastError();
}
template <class TY, class TS, class TX>
static hipError_t bwd_width(const BwdArgs& P, hipStream_t s) {
  const int team = team_of(P.rows, P.d), nv = (int)cdiv(cdiv(P.d, 8), team);
  if (P.d % 8) {  // fewer forms for widths off the groups
    switch (team) {
      case 32:
        return nv <= 1 ? bwd_launch<TY, TS, TX, 32, 1, false>(P, s)
                       : nv == 2 ? bwd_launch<TY, TS, TX, 32, 2, false>(P, s) : bwd_launch<TY, TS, TX, 32, 4, false>(P, s);
      case 256:
        return nv <= 1 ? bwd_launch<TY, TS, TX, 256, 1, false>(P, s)
                       : nv == 2 ? bwd_launch<TY, TS, TX, 256, 2, false>(P, s) : bwd_launch<TY, TS, TX, 256, 4, false>(P, s);
      default: return nv <= 1 ? bwd_launch<TY, TS, TX, 1024, 1, false>(P, s) : bwd_launch<TY, TS, TX, 1024, 2, false>(P, s);
    }
  }
  switch (team) {
    case 32:
      switch (nv) {
        case 1: return bwd_launch<TY, TS, TX, 32, 1, true>(P, s);
        case 2: return bwd_launch<TY, TS, TX, 32, 2, true>(P, s);
        case 3: return bwd_launch<TY, TS, TX, 32, 3, true>(P, s);
        default: return bwd_launch<TY, TS, TX, 32, 4, true>(P, s);
      }
    case 256:
      switch (nv) {
        case 1: return bwd_launch<TY, TS, TX, 256, 1, true>(P, s);
        case 2: return bwd_launch<TY, TS, TX, 256, 2, true>(P, s);
        case 3: return bwd_launch<TY, TS, TX, 256, 3, true>(P, s);
        default: return bwd_launch<TY, TS, TX, 256, 4, true>(P, s);
      }
    default: return nv <= 1 ? bwd_launch<TY, TS, TX, 1024, 1, true>(P, s) : bwd_launch<TY, TS, TX, 1024, 2, true>(P, s);
  }
}
template <class TY, class TS>
static hipError_t bwd_type(const BwdArgs& P, bool xf, hipStream_t s) {
  return xf ? bwd_width<TY, TS, float>(P, s) : bwd_width<TY, TS, bf16_t>(P, s);
}

hipError_t launch_norm_bwd_rows(const layup_layernorm_grad_desc& d, const Mask& k, float* part, hipStream_t s) {
  const BwdArgs P{d.dy,   d.s,   d.dsum,   d.dres,   d.dx,   d.mean, d.rstd, d.gamma, part,
                  d.lddy, d.lds, d.lddsum, d.lddres, d.lddx, d.rows, d.d,    k};
  const bool yf = d.dy_dtype == LAYUP_F32, sf = d.s_dtype == LAYUP_F32, xf = d.dx_dtype == LAYUP_F32;
  if (yf) return sf ? bwd_type<float, float>(P, xf, s) : bwd_type<float, bf16_t>(P, xf, s);
  return sf ? bwd_type<bf16_t, float>(P, xf, s) : bwd_type<bf16_t, bf16_t>(P, xf, s);
}

hipError_t launch_norm_bwd(const layup_layernorm_grad_desc& d, const Mask& k, hipStream_t s) {
  const bool sums = d.dgamma || d.dbeta;
  if (d.rows > 0) {
    const hipError_t e = launch_norm_bwd_rows(d, k, sums ? (float*)d.workspace : nullptr, s);
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  norm_sum_kernel<<<(unsigned)cdiv(2 * d.d, SUM_COLS), SUM_COLS * SUM_LANES, 0, s>>>(
      (const float*)d.workspace, (int)norm_partial_rows(d.rows, d.d), d.d, d.dgamma, d.dbeta);
  return hipGetLastError();
}

}  // namespace layup
