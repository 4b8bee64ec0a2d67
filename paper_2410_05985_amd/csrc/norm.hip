// Dropout from a counter-based generator and LayerNorm with its residual add,
// forward and backward, for any width and row distance.  All are bound by HBM;
// every reduction has a fixed order.
#include "rowvec.h"

namespace layup {

Mask make_mask(const layup_dropout_mask& d) {
  const double t = floor((double)d.p * 65536.0 + 0.5);
  const uint32_t T = t > 65535.0 ? 65535u : (uint32_t)t;
  Mask k;
  k.k0 = (uint32_t)d.seed;
  k.k1 = (uint32_t)(d.seed >> 32);
  k.thr = T << 16;
  k.scale = (float)(65536.0 / (65536.0 - T));
  k.offset = d.offset;
  k.offset_dev = d.offset_dev;
  return k;
}

// ---------------------------------------------------------------- dropout
template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, int64_t ldx, T* y, int64_t ldy, uint32_t row0,
                                                      uint32_t groups, int64_t total, int64_t cols, Mask K) {
  const uint64_t offset = mask_offset(K);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const uint32_t row = (uint32_t)i / groups, g = (uint32_t)i - row * groups;
  const int64_t c = (int64_t)g * 8, n = cols - c;
  Raw8<T> r;
  load_group(r, x + (int64_t)row * ldx + c, n);
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = r.get(e);
  if (K.thr) drop_group(f, g, row0 + row, K, offset);
  store_group(y + (int64_t)row * ldy + c, f, n);
}

template <class T>
static hipError_t dropout_rows(const layup_dropout_desc& d, const Mask& k, hipStream_t s) {
  // launches of fewer than 2^31 groups, so that 32 bits number them
  const int64_t groups = cdiv(d.cols, 8), most = std::max<int64_t>(1, ((1ll << 31) - 1) / groups);
  for (int64_t r = 0; r < d.rows; r += most) {
    const int64_t rows = std::min(most, d.rows - r), total = rows * groups;
    dropout_kernel<T><<<(unsigned)cdiv(total, 256), 256, 0, s>>>((const T*)d.x + r * d.ldx, d.ldx, (T*)d.y + r * d.ldy,
                                                                 d.ldy, (uint32_t)r, (uint32_t)groups, total, d.cols, k);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_dropout(const layup_dropout_desc& d, const Mask& k, hipStream_t s) {
  return d.dtype == LAYUP_F32 ? dropout_rows<float>(d, k, s) : dropout_rows<bf16_t>(d, k, s);
}

// -------------------------------------------------------------- LayerNorm
// A team of TPR threads takes a row, thread t its groups t, t + TPR, ... of
// eight columns, all of them in registers (at most NV).
//
// Sums over the team: inside a wave by exchanges, across waves through LDS;
// every thread of the team gets the same value.
template <int TPR>
__device__ __forceinline__ void team_sum2(float& a, float& b, float* red /* 2 * TPR / 64 floats */) {
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o > 0; o >>= 1) {
    a += __shfl_xor(a, o, 64);
    b += __shfl_xor(b, o, 64);
  }
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

struct FwdArgs {
  const void *x, *res;
  void *sum, *y;
  const float *gamma, *beta;
  float *mean, *rstd;
  uint8_t* yscale;
  int64_t ldx, ldr, lds, ldy, ldsc, rows;
  int32_t d;
  float eps;
  Mask K;
};

constexpr int threads_of(int tpr) { return tpr > 256 ? tpr : 256; }

// YD: layup_dtype of y.
template <class TX, class TS, int YD, int TPR, int NV>
__global__ __launch_bounds__(threads_of(TPR)) void norm_fwd_kernel(const FwdArgs P) {
  constexpr int RPB = threads_of(TPR) / TPR;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  const int t = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (row >= P.rows) return;  // whole teams; a team of several waves is the whole block
  const int d = P.d;
  const TX* x = (const TX*)P.x + row * P.ldx;
  const TS* res = (const TS*)P.res + row * P.ldr;
  Raw8<TX> rx[NV];
  Raw8<TS> rr[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 8 * (t + TPR * j);
    load_group(rx[j], x + c, d - c);
    if (P.res) load_group(rr[j], res + c, d - c);
  }
  const uint64_t offset = mask_offset(P.K);
  float v[NV][8];
  float s = 0.f, ss = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 8 * (t + TPR * j);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[j][e] = rx[j].get(e);
    if (P.K.thr && c < d) drop_group(v[j], c >> 3, (uint32_t)row, P.K, offset);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (P.res) v[j][e] += rr[j].get(e);
      v[j][e] = Raw8<TS>::round(v[j][e]);
      s += v[j][e];  // 0 behind the row's end
    }
    if (P.sum && c < d) store_group((TS*)P.sum + row * P.lds + c, v[j], d - c);
  }
  team_sum2<TPR>(s, ss, red);
  const float mu = s / d;
  float dummy = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float c = 8 * (t + TPR * j) + e < d ? v[j][e] - mu : 0.f;
      ss = fmaf(c, c, ss);
    }
  team_sum2<TPR>(ss, dummy, red);
  const float r = 1.0f / sqrtf(ss / d + P.eps);
  if (t == 0) {
    if (P.mean) P.mean[row] = mu;
    if (P.rstd) P.rstd[row] = r;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 8 * (t + TPR * j);
    Raw8<float> g, b;
    if (P.gamma) load_group(g, P.gamma + c, d - c);
    if (P.beta) load_group(b, P.beta + c, d - c);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = (v[j][e] - mu) * r;
      if (P.gamma) y[e] *= g.get(e);
      if (P.beta) y[e] += b.get(e);
    }
    if constexpr (YD == LAYUP_F32 || YD == LAYUP_BF16) {
      typedef typename std::conditional<YD == LAYUP_F32, float, bf16_t>::type TY;
      if (c < d) store_group((TY*)P.y + row * P.ldy + c, y, d - c);
    } else {
      // sixteen threads hold a block of 128 columns
      constexpr int TOP = YD == LAYUP_E4M3 ? 8 : 15;
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c + e >= d) y[e] = 0.f;
        m = max(m, finite_bits(y[e]));
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
      const uint32_t byte = scale_byte<TOP>(m);
      if (c < (d + 127) / 128 * 128) {
        *reinterpret_cast<u32x2*>((uint8_t*)P.y + row * P.ldy + c) = to_fp8<TOP>(y, inverse_scale(byte));
        if ((t & 15) == 0) P.yscale[row * P.ldsc + (c >> 7)] = (uint8_t)byte;
      }
    }
  }
}

struct BwdArgs {
  const void *dy, *s, *dsum;
  void *dres, *dx;
  const float *mean, *rstd, *gamma;
  float* part;  // partial rows of dgamma and dbeta (nullable)
  int64_t lddy, lds, lddsum, lddres, lddx, rows;
  int32_t d;
  Mask K;
};

template <class TY, class TS, class TX, int TPR, int NV>
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
    if (P.gamma) load_group(rg, P.gamma + c, d - c);
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
      load_group(ry[j], (const TY*)P.dy + row * P.lddy + c, d - c);
      load_group(rs[j], (const TS*)P.s + row * P.lds + c, d - c);
      if (P.dsum) load_group(rd[j], (const TS*)P.dsum + row * P.lddsum + c, d - c);
    }
    const float mu = P.mean[row], r = P.rstd[row];
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
      if (P.dres) store_group((TS*)P.dres + row * P.lddres + c, o, d - c);
      if (P.dx) {
        if (P.K.thr) drop_group(o, c >> 3, (uint32_t)row, P.K, offset);
        store_group((TX*)P.dx + row * P.lddx + c, o, d - c);
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
      store_group(part + c, ag[j], d - c);
      store_group(part + d + c, ab[j], d - c);
    }
  }
}

// dgamma and dbeta from the partial rows: 16 columns a block, 16 row lanes
// each taking every 16th row, then a fixed tree.
__global__ __launch_bounds__(256) void norm_sum_kernel(const float* part, int64_t nb, int d, float* dgamma, float* dbeta) {
  __shared__ float red[16][17];
  const int c = blockIdx.x * 16 + threadIdx.x % 16, l = threadIdx.x / 16;
  float s = 0.f;
  if (c < 2 * d)
    for (int64_t r = l; r < nb; r += 16) s += part[r * 2 * d + c];
  red[l][threadIdx.x % 16] = s;
  __syncthreads();
  if (l > 0 || c >= 2 * d) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) s += red[k][threadIdx.x];
  if (c < d) {
    if (dgamma) dgamma[c] = s;
  } else {
    if (dbeta) dbeta[c - d] = s;
  }
}

// Threads of a team and groups of each for rows of d: as few threads as hold
// the row in four groups each.
static int team_of(int d) { return d <= 1024 ? 32 : d <= 2048 ? 64 : d <= 8192 ? 256 : 1024; }

// Blocks of the backward (and partial rows).
static int64_t bwd_blocks(int64_t rows, int d) {
  const int tpr = team_of(d), rpb = threads_of(tpr) / tpr;
  return std::min<int64_t>(cdiv(rows, rpb), 512);
}

int64_t norm_partial_floats(int64_t rows, int d) { return bwd_blocks(rows, d) * 2 * (int64_t)d; }

template <class TX, class TS, int YD, int TPR, int NV>
static hipError_t fwd_launch(const FwdArgs& P, hipStream_t s) {
  norm_fwd_kernel<TX, TS, YD, TPR, NV><<<(unsigned)cdiv(P.rows, threads_of(TPR) / TPR), threads_of(TPR), 0, s>>>(P);
  return hipGetLastError();
}
template <class TX, class TS, int YD>
static hipError_t fwd_width(const FwdArgs& P, hipStream_t s) {
  const int nv = (int)cdiv(cdiv(P.d, 8), team_of(P.d));
  switch (team_of(P.d)) {
    case 32:
      switch (nv) {
        case 1: return fwd_launch<TX, TS, YD, 32, 1>(P, s);
        case 2: return fwd_launch<TX, TS, YD, 32, 2>(P, s);
        case 3: return fwd_launch<TX, TS, YD, 32, 3>(P, s);
        default: return fwd_launch<TX, TS, YD, 32, 4>(P, s);
      }
    case 64: return fwd_launch<TX, TS, YD, 64, 4>(P, s);
    case 256: return nv <= 2 ? fwd_launch<TX, TS, YD, 256, 2>(P, s) : fwd_launch<TX, TS, YD, 256, 4>(P, s);
    default: return fwd_launch<TX, TS, YD, 1024, 2>(P, s);
  }
}
template <class TX, class TS>
static hipError_t fwd_type(const FwdArgs& P, int yd, hipStream_t s) {
  switch (yd) {
    case LAYUP_F32: return fwd_width<TX, TS, LAYUP_F32>(P, s);
    case LAYUP_BF16: return fwd_width<TX, TS, LAYUP_BF16>(P, s);
    case LAYUP_E4M3: return fwd_width<TX, TS, LAYUP_E4M3>(P, s);
    default: return fwd_width<TX, TS, LAYUP_E5M2>(P, s);
  }
}

hipError_t launch_norm_fwd(const layup_layernorm_desc& d, const Mask& k, hipStream_t s) {
  const FwdArgs P{d.x,   d.residual, d.sum, d.y,   d.gamma,    d.beta, d.mean, d.rstd, d.y_scale,
                  d.ldx, d.ldr,      d.lds, d.ldy, d.ld_scale, d.rows, d.d,    d.eps,  k};
  const bool xf = d.x_dtype == LAYUP_F32, sf = d.s_dtype == LAYUP_F32;
  if (xf) return sf ? fwd_type<float, float>(P, d.y_dtype, s) : fwd_type<float, bf16_t>(P, d.y_dtype, s);
  return sf ? fwd_type<bf16_t, float>(P, d.y_dtype, s) : fwd_type<bf16_t, bf16_t>(P, d.y_dtype, s);
}

template <class TY, class TS, class TX, int TPR, int NV>
static hipError_t bwd_launch(const BwdArgs& P, hipStream_t s) {
  norm_bwd_kernel<TY, TS, TX, TPR, NV><<<(unsigned)bwd_blocks(P.rows, P.d), threads_of(TPR), 0, s>>>(P);
  return hipGetLastError();
}
template <class TY, class TS, class TX>
static hipError_t bwd_width(const BwdArgs& P, hipStream_t s) {
  const int nv = (int)cdiv(cdiv(P.d, 8), team_of(P.d));
  switch (team_of(P.d)) {
    case 32:
      switch (nv) {
        case 1: return bwd_launch<TY, TS, TX, 32, 1>(P, s);
        case 2: return bwd_launch<TY, TS, TX, 32, 2>(P, s);
        case 3: return bwd_launch<TY, TS, TX, 32, 3>(P, s);
        default: return bwd_launch<TY, TS, TX, 32, 4>(P, s);
      }
    case 64: return bwd_launch<TY, TS, TX, 64, 4>(P, s);
    case 256: return nv <= 2 ? bwd_launch<TY, TS, TX, 256, 2>(P, s) : bwd_launch<TY, TS, TX, 256, 4>(P, s);
    default: return bwd_launch<TY, TS, TX, 1024, 2>(P, s);
  }
}
template <class TY, class TS>
static hipError_t bwd_type(const BwdArgs& P, bool xf, hipStream_t s) {
  return xf ? bwd_width<TY, TS, float>(P, s) : bwd_width<TY, TS, bf16_t>(P, s);
}

hipError_t launch_norm_bwd(const layup_layernorm_grad_desc& d, const Mask& k, hipStream_t s) {
  const bool sums = d.dgamma || d.dbeta;
  const int64_t nb = bwd_blocks(d.rows, d.d);
  if (d.rows > 0) {
    const BwdArgs P{d.dy,   d.s,   d.dsum,   d.dres,   d.dx,   d.mean, d.rstd, d.gamma, sums ? (float*)d.workspace : nullptr,
                    d.lddy, d.lds, d.lddsum, d.lddres, d.lddx, d.rows, d.d,    k};
    const bool yf = d.dy_dtype == LAYUP_F32, sf = d.s_dtype == LAYUP_F32, xf = d.dx_dtype == LAYUP_F32;
    hipError_t e;
    if (yf) e = sf ? bwd_type<float, float>(P, xf, s) : bwd_type<float, bf16_t>(P, xf, s);
    else e = sf ? bwd_type<bf16_t, float>(P, xf, s) : bwd_type<bf16_t, bf16_t>(P, xf, s);
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  norm_sum_kernel<<<(unsigned)cdiv(2 * d.d, 16), 256, 0, s>>>((const float*)d.workspace, nb, d.d, d.dgamma, d.dbeta);
  return hipGetLastError();
}

}  // namespace layup
