// Matrices in 8-bit floats with a power-of-two scale for each block of 128
// along a row (or 128 x 128), as they are and transposed.  Bound by HBM.
#include "rowvec.h"

namespace layup {

namespace {

// One block takes a tile of 128 x 128, thread t the columns 8 (t % 16) .. + 7 of
// R rows from R (t / 16) on.  R = 8 (256 threads): an 8 x 8 patch, so that both
// q and qt leave the registers in 8-byte pieces.  R = 2 (1024 threads) where
// there are few tiles, which then wait for their slowest thread.
struct QuantArgs {
  const void* x;
  uint8_t *q, *scale, *qt, *scale_t;
  int64_t rows, cols, ldx, ldq, ldsc, ldqt, ldsct;
};

template <class T, int TOP, bool BLOCK, int R>
__global__ __launch_bounds__(2048 / R) void quant_kernel(const QuantArgs P) {
  constexpr int WAVES = 32 / R;
  __shared__ uint32_t red[WAVES][128];
  __shared__ __attribute__((aligned(8))) uint8_t tile[128][136];
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, w = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)blockIdx.y * 128 + R * rg, c0 = (int64_t)blockIdx.x * 128 + 8 * cg;
  Raw8<T> raw[R];
#pragma unroll
  for (int i = 0; i < R; ++i)  // rows past the last: that again, zeroed below
    load_group(raw[i], (const T*)P.x + min(r0 + i, P.rows - 1) * P.ldx, c0, P.cols);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    finish_group(raw[i], (const T*)P.x + min(r0 + i, P.rows - 1) * P.ldx, c0, P.cols);
    if (r0 + i >= P.rows) raw[i].zero();
  }
  uint32_t rmax[R], cmax[8];
#pragma unroll
  for (int i = 0; i < R; ++i) rmax[i] = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) cmax[e] = 0;
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t a = finite_bits(raw[i].get(e));
      rmax[i] = max(rmax[i], a);
      cmax[e] = max(cmax[e], a);
    }
  if constexpr (BLOCK) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) m = max(m, rmax[i]);
    m = lanes16_max(m);
    if (cg == 0) red[0][rg] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int i = 0; i < 128 / R; ++i) m = max(m, red[0][i]);
#pragma unroll
    for (int i = 0; i < R; ++i) rmax[i] = m;
#pragma unroll
    for (int e = 0; e < 8; ++e) cmax[e] = m;
  } else {
#pragma unroll
    for (int i = 0; i < R; ++i) rmax[i] = lanes16_max(rmax[i]);
    if (P.qt) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        cmax[e] = max(cmax[e], (uint32_t)__shfl_xor((int)cmax[e], 16, 64));
        cmax[e] = max(cmax[e], (uint32_t)__shfl_xor((int)cmax[e], 32, 64));
      }
      if ((threadIdx.x & 63) < 16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) red[w][8 * cg + e] = cmax[e];
      }
      __syncthreads();
      if (threadIdx.x < 128) {  // a column each, over the waves
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) m = max(m, red[k][threadIdx.x]);
        red[0][threadIdx.x] = m;
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) cmax[e] = red[0][8 * cg + e];
    }
  }
  if (P.q) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
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
      for (int i = 0; i < 8; ++i) f[i] = i < R ? raw[i < R ? i : 0].get(e) : 0.f;
      const u32x2 o = to_fp8<TOP>(f, inverse_scale(byte));
      if constexpr (R == 8) *reinterpret_cast<u32x2*>(&tile[8 * cg + e][8 * rg]) = o;
      else *reinterpret_cast<uint16_t*>(&tile[8 * cg + e][R * rg]) = (uint16_t)o[0];
      if (!BLOCK && rg == 0 && c0 + e < P.cols) P.scale_t[(c0 + e) * P.ldsct + blockIdx.y] = (uint8_t)byte;
    }
    if (BLOCK && threadIdx.x == 0) P.scale_t[blockIdx.x * P.ldsct + blockIdx.y] = (uint8_t)scale_byte<TOP>(cmax[0]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < R; ++k) {  // 8 bytes of 128 / R rows of qt at a time
      const int c = 128 / R * k + rg;
      if ((int64_t)blockIdx.x * 128 + c < P.cols)
        *reinterpret_cast<u32x2*>(P.qt + ((int64_t)blockIdx.x * 128 + c) * P.ldqt + (int64_t)blockIdx.y * 128 + 8 * cg) =
            *reinterpret_cast<const u32x2*>(&tile[c][8 * cg]);
    }
  }
}

template <class T, int TOP, bool BLOCK>
void quant_tiles(const QuantArgs& P, dim3 grid, hipStream_t s) {
  // 256 against 1024 threads: 1101 x 523 (45 tiles) 10.4 us against 5.6, 4096 x
  // 2048 (512 tiles) 11.6 against 15.0
  if ((int64_t)grid.x * grid.y <= 256) quant_kernel<T, TOP, BLOCK, 2><<<grid, 1024, 0, s>>>(P);
  else quant_kernel<T, TOP, BLOCK, 8><<<grid, 256, 0, s>>>(P);
}

template <class T, int TOP>
hipError_t quant_launch(const QuantArgs& P, int block_rows, hipStream_t s) {
  // at most 65535 tile rows a launch, and columns for which its threads (256 a
  // tile) suffice: more go in slices of whole tiles
  constexpr int64_t most_r = 65535ll * 128, most_c = MAX_LAUNCH_THREADS / 256 * 128;
  for (int64_t r = 0; r < P.rows; r += most_r)
    for (int64_t c = 0; c < P.cols; c += most_c) {
      QuantArgs Q = P;
      Q.rows = std::min(most_r, P.rows - r);
      Q.cols = std::min(most_c, P.cols - c);
      Q.x = (const T*)P.x + r * P.ldx + c;
      if (P.q) Q.q = P.q + r * P.ldq + c;
      if (P.q) Q.scale = P.scale + r / block_rows * P.ldsc + c / 128;
      if (P.qt) Q.qt = P.qt + c * P.ldqt + r;
      if (P.qt) Q.scale_t = P.scale_t + c / block_rows * P.ldsct + r / 128;
      const dim3 grid((unsigned)cdiv(Q.cols, 128), (unsigned)cdiv(Q.rows, 128));
      if (block_rows == 128) quant_tiles<T, TOP, true>(Q, grid, s);
      else quant_tiles<T, TOP, false>(Q, grid, s);
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
