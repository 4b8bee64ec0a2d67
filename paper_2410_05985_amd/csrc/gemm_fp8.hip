// Product of two matrices in 8-bit floats with a power-of-two scale for each
// block of 128 k on the CDNA4 matrix cores.  v_mfma_scale_f32_32x32x64_f8f6f4
// takes both scales as exponent bytes, so a scaled product costs no more than
// a plain one and the accumulators run through all of K.
//
// The 8-bit matrix instructions align eight products at a time and drop what
// lies 2^-13 below the largest (measured: a product of 2^(16-g) beside one of
// 2^16 is kept up to g = 13 within a group of eight, up to g = 23 outside it;
// the scaled and the plain instruction give the same bits).  A result is off
// by 1.3e-5 of itself for normal operands whatever K: nothing next to the
// rounding of a bfloat16 result (1.7e-3), but fifty times a float32 sum's
// error.  So a float32 result (EXACT) is computed from the operands widened in
// registers to bfloat16, which holds them exactly, scale included, at the
// bfloat16 instructions' half rate.
#include "lds_pipe.h"

namespace layup {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp8Args {
  const uint8_t *A, *B, *sa, *sb;
  void* C;
  const float* bias;
  float* partial;  // split-K: float32 partial results, one M x N after another
  int64_t M, N, lda, ldb, ldc, ldsa, ldsb;
  int32_t fa, fb;  // log2 of the rows that share a scale
  int32_t kb;      // K in blocks of 128
  int32_t c_f32, splits, kb_split;  // blocks of a split: a multiple of 4
  int32_t tiles_m, tiles_n;
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

// 2^(byte - 127) of the low byte
__device__ __forceinline__ float scale_of(uint32_t s) { return __builtin_bit_cast(float, (s & 255u) << 23); }

// 64 k of a fragment: two 16-byte chunks of one row a lane, which 32 k of the
// row they are does not matter as long as A and B agree (all share a scale).
struct Frag {
  u32x4 lo, hi;
};

// acc += A B^T over the 64 k of two fragments; the scales are the low bytes.
template <int FA, int FB, bool EXACT>
__device__ __forceinline__ void product64(const Frag& a, const Frag& b, uint32_t sa, uint32_t sb, f32x16& acc) {
  const i32x8 x{(int)a.lo[0], (int)a.lo[1], (int)a.lo[2], (int)a.lo[3], (int)a.hi[0], (int)a.hi[1], (int)a.hi[2], (int)a.hi[3]};
  const i32x8 y{(int)b.lo[0], (int)b.lo[1], (int)b.lo[2], (int)b.lo[3], (int)b.hi[0], (int)b.hi[1], (int)b.hi[2], (int)b.hi[3]};
  acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc, FA, FB, 0, (int)sa, 0, (int)sb);
}

// ------------------------------------------------------------------ tiles
// A BM x BN tile by WGM x WGN waves, each (BM/WGM) x (BN/WGN) in 32 x 32
// blocks.  K advances by one scale block (128 bytes of a row) through a ring
// of STAGES LDS stages filled by direct-to-LDS copies; rows are clamped into
// the operand, K needs no care since rows are zero up to a multiple of 128.
//
// LDS: row r of a tile = 128 B = eight 16-byte chunks, chunk c at
// r*128 + 16*(c ^ ((r >> 1) & 7)): sixteen lanes reading one chunk of sixteen
// consecutive rows cover all banks.
//
// A step's products go in clusters of CA blocks of rows by all TN of columns
// and 64 k, whose fragments are read while the cluster before is multiplied.
// A step starts with the last cluster of the step before, already in
// registers: its products cover the barrier's and the new stage's first
// fragment reads' latency and carry the copies of a later step.
__device__ __forceinline__ int chunk_off(int r, int c) { return r * 128 + 16 * (c ^ ((r >> 1) & 7)); }

template <int BM, int BN, int WGM, int WGN, int S, int FA, int FB, bool EXACT>
__device__ __forceinline__ void tile_item(const Fp8Args& P, int lid) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
  constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
  constexpr int LOADS_A = BM / 8 / NW, LOADS_B = BN / 8 / NW, NPIECE = LOADS_A + LOADS_B;
  static_assert(BM / 8 % NW == 0 && BN / 8 % NW == 0, "copies must split evenly over the waves");
  constexpr int CA = TM >= 2 ? 2 : 1, NC = TM / CA;  // clusters of 64 k
  static_assert(TM % CA == 0, "whole clusters");
  __shared__ __attribute__((aligned(1024))) char smem[S * (A_BYTES + B_BYTES)];

  // tiles go in groups of 8 tile-rows for L2 reuse of B
  const int n_tiles = P.tiles_m * P.tiles_n;
  const int split = lid / n_tiles, id = lid % n_tiles;
  constexpr int GROUP = 8;
  const int width = GROUP * P.tiles_n;
  const int first_m = id / width * GROUP, gsz = min(P.tiles_m - first_m, GROUP);
  const int tm = first_m + (id % width) % gsz, tn = (id % width) / gsz;
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int kb0 = split * P.kb_split, nk = min(P.kb, kb0 + P.kb_split) - kb0;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WGN, wn = wave % WGN;

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // copies: block b of a wave's share is 8 rows, a lane 16 bytes of one.  The
  // tile's first row and the step are scalar, a lane's offset has 32 bits
  // (leading dimensions are at most 2^24).
  char* const smem_b = smem + S * A_BYTES;
  uint32_t off_a[LOADS_A], off_b[LOADS_B];
#pragma unroll
  for (int i = 0; i < LOADS_A; ++i) {
    const int r = (wave * LOADS_A + i) * 8 + (lane >> 3);
    off_a[i] = (uint32_t)min((int64_t)r, P.M - 1 - m0) * (uint32_t)P.lda + 16 * ((lane & 7) ^ ((r >> 1) & 7));
  }
#pragma unroll
  for (int i = 0; i < LOADS_B; ++i) {
    const int r = (wave * LOADS_B + i) * 8 + (lane >> 3);
    off_b[i] = (uint32_t)min((int64_t)r, P.N - 1 - n0) * (uint32_t)P.ldb + 16 * ((lane & 7) ^ ((r >> 1) & 7));
  }
  const char* base_a = (const char*)P.A + m0 * P.lda + (int64_t)kb0 * 128;
  const char* base_b = (const char*)P.B + n0 * P.ldb + (int64_t)kb0 * 128;
  auto issue = [&](int slot, int p) {  // copy p of the next step into a stage
    if (p < LOADS_A) copy_block<0>(base_a + off_a[p], smem + slot * A_BYTES + (wave * LOADS_A + p) * 1024);
    else copy_block<0>(base_b + off_b[p - LOADS_A], smem_b + slot * B_BYTES + (wave * LOADS_B + p - LOADS_A) * 1024);
    if (p == LOADS_A - 1) base_a += 128;
    if (p == NPIECE - 1) base_b += 128;
  };

  // scale bytes, four steps to a word: sa, sb the words in use (the low byte
  // is the step's), na, nb the next ones
  uint32_t sa[TM], sb[TN], na[TM], nb[TN], wa[TM], wb[TN];
  const int64_t ma = m0 >> P.fa, mb = n0 >> P.fb;
  const uint32_t* base_sa = reinterpret_cast<const uint32_t*>(P.sa + ma * P.ldsa + kb0);
  const uint32_t* base_sb = reinterpret_cast<const uint32_t*>(P.sb + mb * P.ldsb + kb0);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t r = min(m0 + wm * WM + 32 * i + (lane & 31), P.M - 1);
    wa[i] = (uint32_t)((r >> P.fa) - ma) * ((uint32_t)P.ldsa >> 2);
    na[i] = base_sa[wa[i]];
    sa[i] = 127;
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t r = min(n0 + wn * WN + 32 * j + (lane & 31), P.N - 1);
    wb[j] = (uint32_t)((r >> P.fb) - mb) * ((uint32_t)P.ldsb >> 2);
    nb[j] = base_sb[wb[j]];
    sb[j] = 127;
  }

  // fragments: rows 32 i + lane % 32, chunks 2 ks + lane / 32; the swizzle
  // leaves whole blocks of 32 rows alone
  uint32_t a_off[4], b_off[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    a_off[ks] = chunk_off(wm * WM + (lane & 31), 2 * ks + (lane >> 5));
    b_off[ks] = chunk_off(wn * WN + (lane & 31), 2 * ks + (lane >> 5));
  }
  const uint32_t lds0 = lds_addr(smem);
  Frag af[2][CA], bf[2][TN];
#pragma unroll
  for (int i = 0; i < CA; ++i) af[1][i].lo = af[1][i].hi = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < TN; ++j) bf[1][j].lo = bf[1][j].hi = u32x4{0, 0, 0, 0};

  // cluster q of a step: 64 k number q / NC, row blocks CA (q % NC) ..
  auto read_cluster = [&](auto Q, int slot) {
    constexpr int q = decltype(Q)::value, h = q / NC, i0 = CA * (q % NC);
    const uint32_t ab = lds0 + (uint32_t)(slot * A_BYTES), bb = lds0 + (uint32_t)(S * A_BYTES + slot * B_BYTES);
    if constexpr (q % NC == 0)
      static_for<0, TN>([&](auto J) {
        constexpr int j = decltype(J)::value;
        bf[h & 1][j].lo = lds_read_b128<j * 4096>(bb + b_off[2 * h]);
        bf[h & 1][j].hi = lds_read_b128<j * 4096>(bb + b_off[2 * h + 1]);
      });
    static_for<0, CA>([&](auto I) {
      constexpr int i = decltype(I)::value;
      af[q & 1][i].lo = lds_read_b128<(i0 + i) * 4096>(ab + a_off[2 * h]);
      af[q & 1][i].hi = lds_read_b128<(i0 + i) * 4096>(ab + a_off[2 * h + 1]);
    });
  };
  auto landed = [&](auto Q) {  // the cluster's reads have been waited for
    constexpr int q = decltype(Q)::value, h = q / NC;
    if constexpr (q % NC == 0)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        after_wait(bf[h & 1][j].lo);
        after_wait(bf[h & 1][j].hi);
      }
#pragma unroll
    for (int i = 0; i < CA; ++i) {
      after_wait(af[q & 1][i].lo);
      after_wait(af[q & 1][i].hi);
    }
  };
  // COPY: with the copies of a later step into stage `slot` between them
  auto multiply = [&](auto Q, auto COPY, int slot) {
    constexpr int q = decltype(Q)::value, h = q / NC, i0 = CA * (q % NC);
    constexpr bool copy = decltype(COPY)::value != 0;
    constexpr int PER = (NPIECE + CA * TN - 1) / (CA * TN);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (EXACT) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // 16 k
        bf16x8 xb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const u32x4& v = x < 2 ? bf[h & 1][j].lo : bf[h & 1][j].hi;
          xb[j] = widen<FB>(v[2 * (x & 1)], v[2 * (x & 1) + 1], scale_of(sb[j]));
        }
#pragma unroll
        for (int i = 0; i < CA; ++i) {
          const u32x4& v = x < 2 ? af[q & 1][i].lo : af[q & 1][i].hi;
          const bf16x8 xa = widen<FA>(v[2 * (x & 1)], v[2 * (x & 1) + 1], scale_of(sa[i0 + i]));
#pragma unroll
          for (int j = 0; j < TN; ++j)
            acc[i0 + i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xa, xb[j], acc[i0 + i][j], 0, 0, 0);
        }
        if constexpr (copy) {
#pragma unroll
          for (int p = x * ((NPIECE + 3) / 4); p < (x + 1) * ((NPIECE + 3) / 4); ++p)
            if (p < NPIECE) issue(slot, p);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < CA; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          product64<FA, FB, EXACT>(af[q & 1][i], bf[h & 1][j], sa[i0 + i], sb[j], acc[i0 + i][j]);
          if constexpr (copy) {
#pragma unroll
            for (int p = (i * TN + j) * PER; p < (i * TN + j + 1) * PER; ++p)
              if (p < NPIECE) issue(slot, p);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto advance = [&](int kt) {  // the scales of step kt
    if ((kt & 3) == 0) {
      const int g = min(kt + 4, (nk - 1) & ~3) >> 2;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        sa[i] = na[i];
        na[i] = base_sa[g + wa[i]];
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        sb[j] = nb[j];
        nb[j] = base_sb[g + wb[j]];
      }
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] >>= 8;
#pragma unroll
      for (int j = 0; j < TN; ++j) sb[j] >>= 8;
    }
  };
  constexpr int LAST = 2 * NC - 1;
  // reads outstanding that belong to the younger cluster
  auto reads_of = [](int q) constexpr { return 2 * CA + (q % NC == 0 ? 2 * TN : 0); };
  // MAIN: step kt + S - 1 exists.  No branch between LDS reads and their wait.
  auto k_step = [&](auto MAIN, int kt, int slot) {
    constexpr bool main = decltype(MAIN)::value != 0;
    const int pslot = slot == 0 ? S - 1 : slot - 1;  // of steps kt - 1 and kt + S - 1
    if constexpr (main) {
      WAIT_VMCNT((S - 2) * NPIECE);  // loads complete in order: step kt has landed
    } else {
      const int left = min(S - 2, nk - 1 - kt);  // younger steps still in flight
      static_for<0, S - 1>([&](auto D) {
        constexpr int d = decltype(D)::value;
        if (left == d) WAIT_VMCNT(d * NPIECE);
      });
    }
    barrier_only();
    read_cluster(IntC<0>{}, slot);
    multiply(IntC<LAST>{}, IntC<main ? 1 : 0>{}, pslot);
    lgkm_wait<0>();
    landed(IntC<0>{});
    advance(kt);
    static_for<0, LAST>([&](auto Q) {
      constexpr int q = decltype(Q)::value;
      read_cluster(IntC<q + 1>{}, slot);
      multiply(Q, IntC<0>{}, 0);
      lgkm_wait<0>();
      landed(IntC<q + 1>{});
    });
  };
  for (int t = 0; t < S - 1; ++t)
    if (t < nk)
#pragma unroll
      for (int p = 0; p < NPIECE; ++p) issue(t, p);
  int kt = 0, slot = 0;
  for (; kt + S - 1 < nk; ++kt) {
    k_step(IntC<1>{}, kt, slot);
    slot = slot + 1 == S ? 0 : slot + 1;
  }
  for (; kt < nk; ++kt) {
    k_step(IntC<0>{}, kt, slot);
    slot = slot + 1 == S ? 0 : slot + 1;
  }
  multiply(IntC<LAST>{}, IntC<0>{}, 0);

  // ---- epilogue.  32x32 accumulator layout: lane l, register r holds row
  // (r/4)*8 + (l/32)*4 + r%4, column l%32.  Each block passes through a
  // wave-private LDS buffer, after which a lane owns eight consecutive columns
  // of one row (LDS requests of one wave are served in order).
  constexpr int LDW = 40;  // floats per staged row: rows r and r + 4 sit 32 banks apart
  static_assert(NW * 32 * LDW * 4 <= S * (A_BYTES + B_BYTES), "staging fits in the stages");
  __syncthreads();  // every wave has finished reading the stages
  float* const stg = reinterpret_cast<float*>(smem) + wave * 32 * LDW;
  const bool part = P.splits > 1;
  const bool wide = part || EXACT;  // float32 stores
  float* const cf = part ? P.partial + (int64_t)split * P.M * P.N : (float*)P.C;
  const int64_t ldc = part ? P.N : P.ldc;
  const float* const bias = part ? nullptr : P.bias;
  const bool vec = ((part ? (uintptr_t)P.partial : (uintptr_t)P.C) & 15) == 0 && (ldc & 7) == 0 && (P.N & 7) == 0 &&
                   ((uintptr_t)bias & 15) == 0;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
      for (int r = 0; r < 16; ++r) stg[((r >> 2) * 8 + (lane >> 5) * 4 + (r & 3)) * LDW + (lane & 31)] = acc[i][j][r];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int it = 0; it < 2; ++it) {
        const int rr = (lane + 64 * it) >> 2, cc = ((lane + 64 * it) & 3) * 8;
        const int64_t m = m0 + wm * WM + i * 32 + rr, n = n0 + wn * WN + j * 32 + cc;
        f32x4 v0 = *reinterpret_cast<const f32x4*>(stg + rr * LDW + cc), v1 = *reinterpret_cast<const f32x4*>(stg + rr * LDW + cc + 4);
        if (m >= P.M || n >= P.N) continue;
        if (vec) {
          if (bias) {
            v0 += *reinterpret_cast<const f32x4*>(bias + n);
            v1 += *reinterpret_cast<const f32x4*>(bias + n + 4);
          }
          if (wide) {
            *reinterpret_cast<f32x4*>(cf + m * ldc + n) = v0;
            *reinterpret_cast<f32x4*>(cf + m * ldc + n + 4) = v1;
          } else {
            *reinterpret_cast<u32x4*>((bf16_t*)P.C + m * ldc + n) =
                u32x4{pack_bf2(v0[0], v0[1]), pack_bf2(v0[2], v0[3]), pack_bf2(v1[0], v1[1]), pack_bf2(v1[2], v1[3])};
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (n + e >= P.N) continue;
            const float x = (e < 4 ? v0[e & 3] : v1[e & 3]) + (bias ? bias[n + e] : 0.f);
            if (wide) cf[m * ldc + n + e] = x;
            else ((bf16_t*)P.C)[m * ldc + n + e] = f2bf(x);
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// OCC: workgroups per CU.
template <int BM, int BN, int WGM, int WGN, int S, int OCC, int FA, int FB, bool EXACT>
__global__ __launch_bounds__(64 * WGM * WGN, OCC * WGM * WGN / 4) void gemm_fp8_kernel(const Fp8Args P) {
  const int n = P.tiles_m * P.tiles_n * P.splits;
  const int lid = work_item(n, blockIdx.x);
  if (lid >= n) return;
  tile_item<BM, BN, WGM, WGN, S, FA, FB, EXACT>(P, lid);
}

// Sum of the split-K partials in split order, bias, rounding: four columns of
// a row a thread.
__global__ __launch_bounds__(256) void fp8_reduce_kernel(const Fp8Args P) {
  const int64_t nq = (P.N + 3) / 4, idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= P.M * nq) return;
  const int64_t m = idx / nq, n = (idx - m * nq) * 4, total = P.M * P.N;
  const float* src = P.partial + m * P.N + n;
  const int ne = (int)min(P.N - n, (int64_t)4);
  f32x4 v{0.f, 0.f, 0.f, 0.f};
  if ((P.N & 3) == 0) {
    for (int s = 0; s < P.splits; ++s) v += *reinterpret_cast<const f32x4*>(src + s * total);
  } else {
    for (int s = 0; s < P.splits; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < ne) v[e] += src[s * total + e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (e >= ne) break;
    const float x = v[e] + (P.bias ? P.bias[n + e] : 0.f);
    if (P.c_f32) ((float*)P.C)[m * P.ldc + n + e] = x;
    else ((bf16_t*)P.C)[m * P.ldc + n + e] = f2bf(x);
  }
}

template <int BM, int BN, int WGM, int WGN, int S, int OCC, int FA, int FB>
hipError_t launch_tiles(const Fp8Args& P, hipStream_t s) {
  const int64_t n = (int64_t)P.tiles_m * P.tiles_n * P.splits;
  if (n >= (1ll << 31) - 8) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)((n + 7) / 8 * 8);
  constexpr int NT = 64 * WGM * WGN;
  if (P.c_f32) gemm_fp8_kernel<BM, BN, WGM, WGN, S, OCC, FA, FB, true><<<grid, NT, 0, s>>>(P);
  else gemm_fp8_kernel<BM, BN, WGM, WGN, S, OCC, FA, FB, false><<<grid, NT, 0, s>>>(P);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || P.splits == 1) return e;
  const int64_t groups = P.M * cdiv(P.N, 4);
  if (groups >= (1ll << 31) * 256ll) return hipErrorInvalidValue;
  fp8_reduce_kernel<<<(unsigned)cdiv(groups, 256), 256, 0, s>>>(P);
  return hipGetLastError();
}

struct TileCfg {
  int bm, bn;
};
enum TileId { T256x256 = 0, T256x128, T128x128, T64x64, kNumCfg };
const TileCfg kCfgs[kNumCfg] = {{256, 256}, {256, 128}, {128, 128}, {64, 64}};

template <int FA, int FB>
hipError_t launch_cfg(const Fp8Args& P, int cfg, hipStream_t s) {
  switch (cfg) {
    case T256x256: return launch_tiles<256, 256, 2, 4, 2, 1, FA, FB>(P, s);
    case T256x128: return launch_tiles<256, 128, 4, 2, 3, 1, FA, FB>(P, s);
    case T128x128: return launch_tiles<128, 128, 2, 2, 2, 2, FA, FB>(P, s);
    default: return launch_tiles<64, 64, 2, 2, 2, 4, FA, FB>(P, s);
  }
}

// Columns of C without a product: the bias, or zero.
__global__ __launch_bounds__(256) void fp8_bias_kernel(const Fp8Args P) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= P.M * P.N) return;
  const int64_t m = idx / P.N, n = idx - m * P.N;
  const float x = P.bias ? P.bias[n] : 0.f;
  if (P.c_f32) ((float*)P.C)[m * P.ldc + n] = x;
  else ((bf16_t*)P.C)[m * P.ldc + n] = f2bf(x);
}

}  // namespace

hipError_t launch_gemm_fp8_cfg(const layup_gemm_fp8_desc& d, int cfg, int splits, hipStream_t s) {
  Fp8Args P{};
  P.A = (const uint8_t*)d.A;
  P.B = (const uint8_t*)d.B;
  P.sa = d.a_scale;
  P.sb = d.b_scale;
  P.C = d.C;
  P.bias = d.bias;
  P.partial = (float*)d.workspace;
  P.M = d.M;
  P.N = d.N;
  P.lda = d.lda;
  P.ldb = d.ldb;
  P.ldc = d.ldc;
  P.ldsa = d.ld_a_scale;
  P.ldsb = d.ld_b_scale;
  P.fa = d.a_block == 128 ? 7 : 0;
  P.fb = d.b_block == 128 ? 7 : 0;
  P.kb = (int32_t)cdiv(d.K, 128);
  P.c_f32 = d.c_f32 != 0;
  if (P.kb == 0) {
    if (P.M * P.N >= (1ll << 31) * 256ll) return hipErrorInvalidValue;
    fp8_bias_kernel<<<(unsigned)cdiv(P.M * P.N, 256), 256, 0, s>>>(P);
    return hipGetLastError();
  }
  if (cfg < 0 || cfg >= kNumCfg) return hipErrorInvalidValue;
  P.kb_split = (int32_t)(cdiv(cdiv(P.kb, std::max(1, splits)), 4) * 4);
  P.splits = (int32_t)cdiv(P.kb, P.kb_split);
  if (P.splits > 1 && (!d.workspace || d.workspace_bytes < (size_t)P.splits * P.M * P.N * 4)) return hipErrorInvalidValue;
  P.tiles_m = (int32_t)cdiv(P.M, kCfgs[cfg].bm);
  P.tiles_n = (int32_t)cdiv(P.N, kCfgs[cfg].bn);
  const bool a4 = d.a_dtype == LAYUP_E4M3, b4 = d.b_dtype == LAYUP_E4M3;
  if (a4) return b4 ? launch_cfg<0, 0>(P, cfg, s) : launch_cfg<0, 1>(P, cfg, s);
  return b4 ? launch_cfg<1, 0>(P, cfg, s) : launch_cfg<1, 1>(P, cfg, s);
}

hipError_t launch_gemm_fp8(const layup_gemm_fp8_desc& d, hipStream_t s) {
  const int64_t t256 = cdiv(d.M, 256) * cdiv(d.N, 256), t128 = cdiv(d.M, 128) * cdiv(d.N, 128);
  const int cfg = t256 >= 200 ? T256x256 : t128 >= 200 ? T128x128 : T64x64;
  return launch_gemm_fp8_cfg(d, cfg, 1, s);
}

}  // namespace layup
