// Matrices in 8-bit floats with a power-of-two scale for each block of 128,
// and their product on the CDNA4 matrix cores: v_mfma_scale_f32_32x32x64_f8f6f4
// takes both scales as exponent bytes, so a scaled product costs no more than
// a plain one.
#include "rowvec.h"

namespace layup {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// -------------------------------------------------------------- quantiser
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
#pragma unroll
  for (int i = 0; i < 8; ++i) load_group(raw[i], (const T*)P.x + (r0 + i) * P.ldx + c0, r0 + i < P.rows ? P.cols - c0 : 0);
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
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) rmax[i] = max(rmax[i], (uint32_t)__shfl_xor((int)rmax[i], o, 64));
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

// ---------------------------------------------------------------- product
struct Fp8Args {
  const uint8_t *A, *B, *sa, *sb;
  void* C;
  const float* bias;
  int64_t M, N, lda, ldb, ldc, ldsa, ldsb;
  int32_t kb;      // blocks of 128 k
  int32_t fa, fb;  // log2 of the rows that share a scale
  int32_t c_f32;
};

// Eight 8-bit values, times a power of two, in bfloat16: exact.
template <int F>
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale) {
  bf16x2 p[4];
  if constexpr (F == 0) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
  }
  return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

// 2^(byte - 127)
__device__ __forceinline__ float scale_of(int byte) { return __builtin_bit_cast(float, byte << 23); }

__device__ __forceinline__ i32x8 frag(const uint8_t* p) {
  const u32x4 lo = *reinterpret_cast<const u32x4*>(p), hi = *reinterpret_cast<const u32x4*>(p + 16);
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// One wave, one 32 x 32 tile of C.  Operand fragment of the 32x32x64 product:
// lane l holds 32 k of row l % 32; which 32 does not matter as long as A and B
// agree, since all 64 share a scale.  Rows past the end repeat the last one.
//
// The 8-bit matrix instructions align eight products at a time and drop what
// lies 2^-13 below the largest (measured: a product of 2^(16-g) beside one of
// 2^16 is kept up to g = 13 within a group of eight, up to g = 23 outside it;
// the scaled and the plain instruction give the same bits).  The result is off
// by 1.3e-5 of itself for normal operands whatever K: nothing next to the
// rounding of a bfloat16 result (1.7e-3), but fifty times a float32 sum's
// error.  So a float32 result (EXACT) is computed from the operands widened to
// bfloat16, which holds them exactly, scale included.
template <int FA, int FB, bool EXACT>
__global__ __launch_bounds__(64) void gemm_fp8_kernel(const Fp8Args P) {
  const int lane = threadIdx.x;
  const int64_t m = (int64_t)blockIdx.x * 32, n = (int64_t)blockIdx.y * 32;
  const int64_t ra = min(m + (lane & 31), P.M - 1), rb = min(n + (lane & 31), P.N - 1);
  const uint8_t *a = P.A + ra * P.lda + 32 * (lane >> 5), *b = P.B + rb * P.ldb + 32 * (lane >> 5);
  const uint8_t *sa = P.sa + (ra >> P.fa) * P.ldsa, *sb = P.sb + (rb >> P.fb) * P.ldsb;
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  for (int k = 0; k < P.kb; ++k) {
    const int ea = sa[k], eb = sb[k];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const i32x8 fa = frag(a + k * 128 + 64 * h), fb = frag(b + k * 128 + 64 * h);
      if constexpr (EXACT) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen<FA>(fa[2 * i], fa[2 * i + 1], scale_of(ea)),
                                                        widen<FB>(fb[2 * i], fb[2 * i + 1], scale_of(eb)), acc, 0, 0, 0);
      } else {
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa, fb, acc, FA, FB, 0, ea, 0, eb);
      }
    }
  }
  const int64_t c = n + (lane & 31);
  if (c >= P.N) return;
  const float bias = P.bias ? P.bias[c] : 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int64_t row = m + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3);
    if (row >= P.M) continue;
    if (EXACT) ((float*)P.C)[row * P.ldc + c] = acc[r] + bias;
    else ((bf16_t*)P.C)[row * P.ldc + c] = f2bf(acc[r] + bias);
  }
}

template <int FA, int FB>
hipError_t gemm_launch(const Fp8Args& P, hipStream_t s) {
  const dim3 grid((unsigned)cdiv(P.M, 32), (unsigned)cdiv(P.N, 32));
  if (P.c_f32) gemm_fp8_kernel<FA, FB, true><<<grid, 64, 0, s>>>(P);
  else gemm_fp8_kernel<FA, FB, false><<<grid, 64, 0, s>>>(P);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quant_fp8(const layup_quant_desc& d, hipStream_t s) {
  const QuantArgs P{d.x,    (uint8_t*)d.q, d.scale, (uint8_t*)d.qt, d.scale_t, d.rows,
                    d.cols, d.ldx,         d.ldq,   d.ld_scale,     d.ldqt,    d.ld_scale_t};
  const bool f32 = d.x_dtype == LAYUP_F32, e4 = d.q_dtype == LAYUP_E4M3;
  if (f32) return e4 ? quant_launch<float, 8>(P, d.block_rows, s) : quant_launch<float, 15>(P, d.block_rows, s);
  return e4 ? quant_launch<bf16_t, 8>(P, d.block_rows, s) : quant_launch<bf16_t, 15>(P, d.block_rows, s);
}

hipError_t launch_gemm_fp8(const layup_gemm_fp8_desc& d, hipStream_t s) {
  const Fp8Args P{(const uint8_t*)d.A, (const uint8_t*)d.B, d.a_scale, d.b_scale, d.C, d.bias, d.M, d.N, d.lda, d.ldb,
                  d.ldc, d.ld_a_scale, d.ld_b_scale, (int32_t)cdiv(d.K, 128), d.a_block == 128 ? 7 : 0,
                  d.b_block == 128 ? 7 : 0, d.c_f32};
  const bool a4 = d.a_dtype == LAYUP_E4M3, b4 = d.b_dtype == LAYUP_E4M3;
  if (a4) return b4 ? gemm_launch<0, 0>(P, s) : gemm_launch<0, 1>(P, s);
  return b4 ? gemm_launch<1, 0>(P, s) : gemm_launch<1, 1>(P, s);
}

}  // namespace layup
