// Dropout from a counter-based generator, and the forward of LayerNorm with its
// residual add, for any width and row distance.  Bound by HBM.
#include "norm.h"

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
// y = m scale x, where m(r, c) is 1 if the 16 bits that the generator draws for
// (r, c) are at least the threshold: computed here and again by whoever needs it
// later, never stored.  A thread takes eight neighbouring columns, which one
// call of the generator serves and one 128-bit access moves in bfloat16.  Bound
// by HBM: 8192 x 8192 bfloat16 45 us (5.9 TB/s; a copy of that size 5.4), 16 x
// 2048 3.5 us, a launch's latency.
template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, int64_t ldx, T* y, int64_t ldy, uint32_t row0,
                                                      uint32_t groups, int64_t total, int64_t cols, Mask K) {
  const uint64_t offset = mask_offset(K);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const uint32_t row = (uint32_t)i / groups, g = (uint32_t)i - row * groups;
  const int64_t c = (int64_t)g * 8, n = cols - c;
  Raw8<T> r;
  load_group(r, x + (int64_t)row * ldx, c, cols);
  finish_group(r, x + (int64_t)row * ldx, c, cols);
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
struct FwdArgs {
  const void *x, *res;
  void *sum, *y;
  const float *gamma, *beta;
  float *mean, *rstd;
  uint8_t* yscale;
  int64_t ldx, ldr, lds, ldy, ldsc, rows, row0;  // row0: the launch's first row
  int32_t d;
  float eps;
  Mask K;
};

// s = res + m scale x, rounded to its type; y = (s - mean) rstd gamma + beta of
// the rounded s, which the backward reads too.  The row is read once and stays
// in registers: mean, then the sum of the squared differences from it (no
// difference of large sums), then the result.  Bound by HBM where rows are
// many: 8192 x 8192, four bfloat16 streams, 104 us (5.2 TB/s); 8192 x 768 with
// a float32 residual stream 18 us (4.2 TB/s).
// Below about 1000 rows the two reductions and the loads' round trip are all
// there is: 2.7 us for 1 x 768.
// YD: layup_dtype of y.
// WHOLE: d is a multiple of 8.
template <class TX, class TS, int YD, int TPR, int NV, bool WHOLE>
__global__ __launch_bounds__(threads_of(TPR)) void norm_fwd_kernel(const FwdArgs P) {
  constexpr int RPB = threads_of(TPR) / TPR;
  constexpr bool EARLY = TPR <= 64;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  const int t = threadIdx.x % TPR;
  const int64_t row = P.row0 + (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (row >= P.rows) return;  // whole teams; a team of several waves is the whole block
  const int d = P.d;
  const TX* x = (const TX*)P.x + row * P.ldx;
  const TS* res = (const TS*)P.res + row * P.ldr;
  Raw8<TX> rx[NV];
  Raw8<TS> rr[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 8 * (t + TPR * j);
    load_group<WHOLE>(rx[j], x, c, d);
    if (P.res) load_group<WHOLE>(rr[j], res, c, d);
  }
  // gain and bias too are requested before the first reduction where they fit
  Raw8<float> rg[NV], rb[NV];
  if constexpr (EARLY) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = 8 * (t + TPR * j);
      if (P.gamma) load_group<WHOLE>(rg[j], P.gamma, c, d);
      if (P.beta) load_group<WHOLE>(rb[j], P.beta, c, d);
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = 8 * (t + TPR * j);
    finish_group<WHOLE>(rx[j], x, c, d);
    if (P.res) finish_group<WHOLE>(rr[j], res, c, d);
    if constexpr (EARLY) {
      if (P.gamma) finish_group<WHOLE>(rg[j], P.gamma, c, d);
      if (P.beta) finish_group<WHOLE>(rb[j], P.beta, c, d);
    }
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
    if (P.sum && c < d) store_group<WHOLE>((TS*)P.sum + row * P.lds + c, v[j], d - c);
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
    if constexpr (!EARLY) {
      if (P.gamma) load_group<WHOLE>(rg[j], P.gamma, c, d);
      if (P.beta) load_group<WHOLE>(rb[j], P.beta, c, d);
      if (P.gamma) finish_group<WHOLE>(rg[j], P.gamma, c, d);
      if (P.beta) finish_group<WHOLE>(rb[j], P.beta, c, d);
    }
    const Raw8<float>&g = rg[j], &b = rb[j];
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = (v[j][e] - mu) * r;
      if (P.gamma) y[e] *= g.get(e);
      if (P.beta) y[e] += b.get(e);
    }
    if constexpr (YD == LAYUP_F32 || YD == LAYUP_BF16) {
      typedef typename std::conditional<YD == LAYUP_F32, float, bf16_t>::type TY;
      if (c < d) store_group<WHOLE>((TY*)P.y + row * P.ldy + c, y, d - c);
    } else {
      // sixteen threads hold a block of 128 columns
      constexpr int TOP = YD == LAYUP_E4M3 ? 8 : 15;
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c + e >= d) y[e] = 0.f;
        m = max(m, finite_bits(y[e]));
      }
      m = lanes16_max(m);
      const uint32_t byte = scale_byte<TOP>(m);
      if (c < (d + 127) / 128 * 128) {
        *reinterpret_cast<u32x2*>((uint8_t*)P.y + row * P.ldy + c) = to_fp8<TOP>(y, inverse_scale(byte));
        if ((t & 15) == 0) P.yscale[row * P.ldsc + (c >> 7)] = (uint8_t)byte;
      }
    }
  }
}

template <class TX, class TS, int YD, int TPR, int NV, bool WHOLE>
static hipError_t fwd_launch(FwdArgs P, hipStream_t s) {
  constexpr int NT = threads_of(TPR), RPB = NT / TPR;
  constexpr int64_t most = MAX_LAUNCH_THREADS / NT * RPB;
  for (; P.row0 < P.rows; P.row0 += most) {
    norm_fwd_kernel<TX, TS, YD, TPR, NV, WHOLE><<<(unsigned)cdiv(std::min(most, P.rows - P.row0), RPB), NT, 0, s>>>(P);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <class TX, class TS, int YD>
static hipError_t fwd_width(const FwdArgs& P, hipStream_t s) {
  const int team = team_of(P.rows, P.d), nv = (int)cdiv(cdiv(P.d, 8), team);
  if (P.d % 8) {  // fewer forms for widths off the groups
    switch (team) {
      case 32:
        return nv <= 1 ? fwd_launch<TX, TS, YD, 32, 1, false>(P, s)
                       : nv == 2 ? fwd_launch<TX, TS, YD, 32, 2, false>(P, s) : fwd_launch<TX, TS, YD, 32, 4, false>(P, s);
      case 256:
        return nv <= 1 ? fwd_launch<TX, TS, YD, 256, 1, false>(P, s)
                       : nv == 2 ? fwd_launch<TX, TS, YD, 256, 2, false>(P, s) : fwd_launch<TX, TS, YD, 256, 4, false>(P, s);
      default: return nv <= 1 ? fwd_launch<TX, TS, YD, 1024, 1, false>(P, s) : fwd_launch<TX, TS, YD, 1024, 2, false>(P, s);
    }
  }
  switch (team) {
    case 32:
      switch (nv) {
        case 1: return fwd_launch<TX, TS, YD, 32, 1, true>(P, s);
        case 2: return fwd_launch<TX, TS, YD, 32, 2, true>(P, s);
        case 3: return fwd_launch<TX, TS, YD, 32, 3, true>(P, s);
        default: return fwd_launch<TX, TS, YD, 32, 4, true>(P, s);
      }
    case 256:
      switch (nv) {
        case 1: return fwd_launch<TX, TS, YD, 256, 1, true>(P, s);
        case 2: return fwd_launch<TX, TS, YD, 256, 2, true>(P, s);
        case 3: return fwd_launch<TX, TS, YD, 256, 3, true>(P, s);
        default: return fwd_launch<TX, TS, YD, 256, 4, true>(P, s);
      }
    default: return nv <= 1 ? fwd_launch<TX, TS, YD, 1024, 1, true>(P, s) : fwd_launch<TX, TS, YD, 1024, 2, true>(P, s);
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
                  d.ldx, d.ldr,      d.lds, d.ldy, d.ld_scale, d.rows, 0,      d.d,    d.eps, k};
  const bool xf = d.x_dtype == LAYUP_F32, sf = d.s_dtype == LAYUP_F32;
  if (xf) return sf ? fwd_type<float, float>(P, d.y_dtype, s) : fwd_type<float, bf16_t>(P, d.y_dtype, s);
  return sf ? fwd_type<bf16_t, float>(P, d.y_dtype, s) : fwd_type<bf16_t, bf16_t>(P, d.y_dtype, s);
}

}  // namespace layup
