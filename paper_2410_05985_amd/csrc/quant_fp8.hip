// Matrices in 8-bit floats with a power-of-two scale for each block of 128
// along a row (or 128 x 128), as they are and transposed.  Bound by HBM.
#include "rowvec.h"

namespace layup {

namespace {

// One block takes a tile of 128 x 128, thread t the columns 8 (t % 16) .. of
// the rows 8 (t / 16) .. + 7: an 8 x 8 patch, so that both q and qt leave the
// registers in 8-byte pieces.
struct QuantArgs {
  const void* x;
  uint8_t *q, *scale, *qt, *scale_t;
  int64_t rows, cols, ldx, ldq, ldsc, ldqt, ldsct;
};

template <class T, int TOP, bool BLOCK>
__global__ __launch_bounds__(256) void quant_kernel(const QuantArgs P) {
  __shared__ uint32_t red[4][128];
  __shared__ uint8_t tile[128][136];
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, w = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)blockIdx.y * 128 + 8 * rg, c0 = (int64_t)blockIdx.x * 128 + 8 * cg;
  Raw8<T> raw[8];
  const int64_t n = P.cols - c0;
  if (r0 + 8 <= P.rows && n >= 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i].load((const T*)P.x + (r0 + i) * P.ldx + c0);
  } else if (r0 < P.rows && n > 0) {
    // the edge: rows past the last are loaded from it and zeroed
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T* row = (const T*)P.x + min(r0 + i, P.rows - 1) * P.ldx;
      load_group(raw[i], row, c0, P.cols);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r0 + i >= P.rows) raw[i].zero();
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i].zero();
  }
  uint32_t rmax[8], cmax[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rmax[i] = cmax[i] = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t a = finite_bits(raw[i].get(e));
      rmax[i] = max(rmax[i], a);
      cmax[e] = max(cmax[e], a);
    }
  if constexpr (BLOCK) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, rmax[i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if ((threadIdx.x & 63) == 0) red[w][0] = m;
    __syncthreads();
    m = max(max(red[0][0], red[1][0]), max(red[2][0], red[3][0]));
#pragma unroll
    for (int i = 0; i < 8; ++i) rmax[i] = cmax[i] = m;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      rmax[i] = lanes16_max(rmax[i]);
#pragma unroll
      for (int o = 32; o > 8; o >>= 1) cmax[i] = max(cmax[i], (uint32_t)__shfl_xor((int)cmax[i], o, 64));
    }
    if ((threadIdx.x & 63) < 16) {
#pragma unroll
      for (int e = 0; e < 8; ++e) red[w][8 * cg + e] = cmax[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e)
      cmax[e] = max(max(red[0][8 * cg + e], red[1][8 * cg + e]), max(red[2][8 * cg + e], red[3][8 * cg + e]));
  }
  if (P.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (r0 + i >= P.rows) break;
      const uint32_t byte = scale_byte<TOP>(rmax[i]);
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = raw[i].get(e);
      *reinterpret_cast<u32x2*>(P.q + (r0 + i) * P.ldq + c0) = to_fp8<TOP>(f, inverse_scale(byte));
      if (cg == 0 && !BLOCK) P.scale[(r0 + i) * P.ldsc + blockIdx.x] = (uint8_t)byte;
    }
    if (BLOCK && threadIdx.x == 0) P.scale[blockIdx.y * P.ldsc + blockIdx.x] = (uint8_t)scale_byte<TOP>(rmax[0]);
  }
  if (P.qt) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t byte = scale_byte<TOP>(cmax[e]);
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = raw[i].get(e);
      *reinterpret_cast<u32x2*>(&tile[8 * cg + e][8 * rg]) = to_fp8<TOP>(f, inverse_scale(byte));
      if (!BLOCK && rg == 0 && c0 + e < P.cols) P.scale_t[(c0 + e) * P.ldsct + blockIdx.y] = (uint8_t)byte;
    }
    if (BLOCK && threadIdx.x == 0) P.scale_t[blockIdx.x * P.ldsct + blockIdx.y] = (uint8_t)scale_byte<TOP>(cmax[0]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {  // 8 bytes of 16 rows of qt at a time
      const int c = 16 * k + (threadIdx.x >> 4);
      if ((int64_t)blockIdx.x * 128 + c < P.cols)
        *reinterpret_cast<u32x2*>(P.qt + ((int64_t)blockIdx.x * 128 + c) * P.ldqt + (int64_t)blockIdx.y * 128 + 8 * cg) =
            *reinterpret_cast<const u32x2*>(&tile[c][8 * cg]);
    }
  }
}

template <class T, int TOP>
hipError_t quant_launch(const QuantArgs& P, int block_rows, hipStream_t s) {
  // at most 65535 tile rows a launch: more go in slices of whole tiles
  const int64_t most = 65535ll * 128;
  for (int64_t r = 0; r < P.rows; r += most) {
    QuantArgs Q = P;
    Q.rows = std::min(most, P.rows - r);
    Q.x = (const T*)P.x + r * P.ldx;
    if (P.q) Q.q = P.q + r * P.ldq;
    if (P.q) Q.scale = P.scale + r / block_rows * P.ldsc;
    if (P.qt) Q.qt = P.qt + r;
    if (P.qt) Q.scale_t = P.scale_t + r / 128;
    const dim3 grid((unsigned)cdiv(P.cols, 128), (unsigned)cdiv(Q.rows, 128));
    if (block_rows == 128) quant_kernel<T, TOP, true><<<grid, 256, 0, s>>>(Q);
    else quant_kernel<T, TOP, false><<<grid, 256, 0, s>>>(Q);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_quant_fp8(const layup_quant_desc& d, hipStream_t s) {
  const QuantArgs P{d.x,    (uint8_t*)d.q, d.scale, (uint8_t*)d.qt, d.scale_t, d.rows,
                    d.cols, d.ldx,         d.ldq,   d.ld_scale,     d.ldqt,    d.ld_scale_t};
  const bool f32 = d.x_dtype == LAYUP_F32, e4 = d.q_dtype == LAYUP_E4M3;
  if (f32) return e4 ? quant_launch<float, 8>(P, d.block_rows, s) : quant_launch<float, 15>(P, d.block_rows, s);
  return e4 ? quant_launch<bf16_t, 8>(P, d.block_rows, s) : quant_launch<bf16_t, 15>(P, d.block_rows, s);
}

}  // namespace layup
