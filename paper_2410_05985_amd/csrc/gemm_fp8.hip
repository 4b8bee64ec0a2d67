// Product of two matrices in 8-bit floats with a power-of-two scale for each
// block of 128 k on the CDNA4 matrix cores.  v_mfma_scale_f32_32x32x64_f8f6f4
// takes both scales as exponent bytes, so a scaled product costs no more than
// a plain one and the accumulators run through all of K.
//
// The 8-bit matrix instructions align eight products at a time and drop what
// lies 2^-13 below the largest (measured: a product of 2^(16-g) beside one of
// 2^16 is kept up to g = 13 within a group of eight, up to g = 23 outside it;
// the scaled and the plain instruction give the same bits).  For operands of
// random signs a sum is off by 1.2e-5 to 1.5e-5 of the results' size whatever K
// (2e-5 to 3e-5 where some k are much louder), for positive ones by 1.5e-6 to
// 2.9e-6, always too small; never by more than 1.7e-5 of the products' added
// magnitudes.  That changes one or two in a hundred bfloat16 results, by a step
// of theirs, and leaves their distance from the exact product at that of the
// rounding, 1.66e-3; but it is fifty times a float32 sum's error, and where a sum
// cancels not small next to the result.
//
// So a float32 result (EXACT) is computed from the operands widened in registers
// to bfloat16, which holds them exactly, scale included, at the bfloat16
// instructions' half rate.  Its range ends before the least values times the
// least scales and the largest times the largest: a wave that meets such a scale
// byte computes its results again from the values alone (plain_sum; 4096 x 1024 x
// 8192 with one in every row 6.7 ms, else 66 us.  Watching for them costs up to
// 4 %: 1 x 2048 x 8192 7.4 -> 7.7 us, 2048 x 2048 x 2048 21.7 -> 22.5, 4000 x
// 4000 x 16384 398 -> 402).
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
__device__ __forceinline__ uint32_t scale_bits(uint32_t s) { return (s & 255u) << 23; }
__device__ __forceinline__ float scale_of(uint32_t s) { return __builtin_bit_cast(float, scale_bits(s)); }

// bfloat16 holds every value of either format (E4M3 2^-9 to 1.75 2^8, E5M2
// 2^-16 to 1.75 2^15) times the scales of bytes 10 to 239: from 2^-133, its
// least subnormal, which conversion and matrix instructions keep, to 1.75 2^127.
constexpr uint32_t WIDEN_LO = 10, WIDEN_HI = 239;
__device__ __forceinline__ bool too_wide(uint32_t s) { return (s & 255u) - WIDEN_LO > WIDEN_HI - WIDEN_LO; }

// Two values of the format in float32; H: the upper half of the word.
template <int F, bool H>
__device__ __forceinline__ auto values2(uint32_t w) {
  if constexpr (F == 0) return __builtin_amdgcn_cvt_pk_f32_fp8((int)w, H);
  else return __builtin_amdgcn_cvt_pk_f32_bf8((int)w, H);
}

// Blocks k0 .. k0 + nk - 1 of an element of C, for scales that bfloat16 cannot
// carry: a block's sum without its scales, then times both at once.
template <int FA, int FB>
__device__ float plain_sum(const Fp8Args& P, int64_t m, int64_t n, int k0, int nk) {
  const uint8_t *a = P.A + m * P.lda + (int64_t)k0 * 128, *b = P.B + n * P.ldb + (int64_t)k0 * 128;
  const uint8_t *sa = P.sa + (m >> P.fa) * P.ldsa + k0, *sb = P.sb + (n >> P.fb) * P.ldsb + k0;
  float sum = 0.f;
#pragma unroll 1
  for (int k = 0; k < nk; ++k, a += 128, b += 128) {
    float s = 0.f;
#pragma unroll 1
    for (int c = 0; c < 128; c += 16) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(a + c), y = *reinterpret_cast<const u32x4*>(b + c);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const auto x0 = values2<FA, false>(x[w]), x1 = values2<FA, true>(x[w]);
        const auto y0 = values2<FB, false>(y[w]), y1 = values2<FB, true>(y[w]);
        s = fmaf(x1[1], y1[1], fmaf(x1[0], y1[0], fmaf(x0[1], y0[1], fmaf(x0[0], y0[0], s))));
      }
    }
    sum += ldexpf(s, (int)sa[k] + (int)sb[k] - 254);
  }
  return sum;
}

// 64 k of a fragment: two 16-byte chunks of one row a lane, which 32 k of the
// row they are does not matter as long as A and B agree (all share a scale).
struct Frag {
  u32x4 lo, hi;
};

__device__ __forceinline__ i32x8 words(const Frag& f) {
  return i32x8{(int)f.lo[0], (int)f.lo[1], (int)f.lo[2], (int)f.lo[3], (int)f.hi[0], (int)f.hi[1], (int)f.hi[2], (int)f.hi[3]};
}

// acc += (A B^T)^T over the 64 k of two fragments; the scales are the low
// bytes.  The accumulator holds the transposed block: lane l, register r is
// column (r/4)*8 + (l/32)*4 + r%4 of row l%32 of C, so a lane has four
// neighbouring columns in a row.
template <int FA, int FB>
__device__ __forceinline__ void product64(const Frag& a, const Frag& b, uint32_t sa, uint32_t sb, f32x16& acc) {
  acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(words(b), words(a), acc, FB, FA, 0, (int)sb, 0, (int)sa);
}

// Moves the odd 16-lane (32-lane) groups of a with the even ones of b.
__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
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
// Scale bytes: those of the tile's rows for SCN steps are copied to LDS before
// the first one, as words of four steps; every step reads its words.  Row r has
// SCN / 4 words, word w at place w ^ sc_swz(r), so that 32 consecutive rows'
// words of a step lie in different banks.  (Fetched by the step, a word for
// each row is a cache line for each row, as many requests as the operands
// themselves: the copies alone took 446 us of 8192 x 8192 x 8192, then 399.
// Kept in registers and loaded every fourth step, they brought a branch into
// the step, over which the compiler moved the products it was to overlap, and
// a wait for every copy in flight.)  A longer K drains the pipeline every SCN
// steps.
//
// A step's products go in clusters of CA blocks of rows by all TN of columns
// and 64 k, whose fragments are read while the cluster before is multiplied.
// A step starts with the last cluster of the step before, already in
// registers: its products cover the barrier's and the new stage's first
// fragment reads' latency and carry the copies of a later step.
//
// Two stages leave a copy one step to arrive.  The 256 x 256 tile (MID) has room
// for no third one, but its first two clusters read all of B and half of A: a
// second barrier behind them gives those three quarters of the stage to the
// step after next, so every copy has a step and a half (8192 x 8192 x 8192 475
// -> 447 us, of it the copies alone 399 -> 300).  Where a wave's rows are
// one cluster (EARLY), it reads both halves of k before it multiplies the first,
// and the barrier behind them gives the whole stage away: two steps for a copy,
// at the price of a wait for a cluster's reads (700 x 1000 x 4300 on 64 x 64 19.6 ->
// 14.0 us; where the chip is full 8192 x 8192 x 2048 on 128 x 128 150 -> 148).
// Widening makes the products so long that copies arrive anyway: 128 x 128 with
// float32 results lost (4096 x 1024 x 8192 62.5 -> 68.5 us) and keeps one
// barrier, 64 x 64 gained (700 x 1000 x 4300 20.3 -> 17.5).
//
// What bounds it: at 8192 x 8192 x 8192 (450 us, 2.44 PFLOP/s; the card reaches
// 2.8 in a large library product) the products need 220 us at full clock, the
// copies and fragment reads alone 300; zeros for operands, which draw less
// power, take 370.  Float32 results: 8192 x 2048 x 8192 211 us, 1.30 PFLOP/s of
// the 1.4 of a large bfloat16 product.  With a short K the stores weigh more:
// 8192 x 8192 x 2048 138 us.  Measured and not kept: K steps of 64 in rings of
// four and five stages (600 us: half a cache line a row), four waves of 128 x
// 128 (a third fewer LDS reads: 444 at that size, but 111 against 106 at 8192 x
// 2048 x 8192), workgroups that start the next tile before their stores.
__device__ __forceinline__ int chunk_off(int r, int c) { return r * 128 + 16 * (c ^ ((r >> 1) & 7)); }

// W words a row: 64 / W rows fill the banks once
template <int W>
__device__ __forceinline__ int sc_swz(int r) { return (r & 31) / (64 / W); }

// What a workgroup computes.  Tiles go in groups of 8 tile-rows for L2 reuse of B.
struct Place {
  int64_t m0, n0;
  int split, kb0, nk;
};
template <int BM, int BN>
__device__ __forceinline__ Place place(const Fp8Args& P, int lid) {
  const int n_tiles = P.tiles_m * P.tiles_n;
  const int split = lid / n_tiles, id = lid % n_tiles;
  constexpr int GROUP = 8;
  const int width = GROUP * P.tiles_n;
  const int first_m = id / width * GROUP, gsz = min(P.tiles_m - first_m, GROUP);
  const int tm = first_m + (id % width) % gsz, tn = (id % width) / gsz;
  const int kb0 = split * P.kb_split;
  return {(int64_t)tm * BM, (int64_t)tn * BN, split, kb0, min(P.kb, kb0 + P.kb_split) - kb0};
}

// A wave's part of a tile by plain_sum.
template <int BM, int BN, int WGM, int WGN, int FA, int FB>
__device__ __forceinline__ void plain_tile() {
  // the arguments and the place anew, so that the main loop keeps nothing for this
  const Fp8Args* args = (const Fp8Args*)__builtin_amdgcn_kernarg_segment_ptr();
  int block = blockIdx.x, thread = threadIdx.x;
  asm volatile("" : "+s"(args), "+s"(block), "+v"(thread));
  const Fp8Args& P = *args;
  const Place at = place<BM, BN>(P, work_item(P.tiles_m * P.tiles_n * P.splits, block));
  constexpr int WM = BM / WGM, WN = BN / WGN;
  const int wave = thread >> 6;
#pragma unroll 1
  for (int t = thread & 63; t < WM * WN; t += 64) {
    const int64_t m = at.m0 + wave / WGN * WM + t / WN, n = at.n0 + wave % WGN * WN + t % WN;
    if (m >= P.M || n >= P.N) continue;
    const float v = plain_sum<FA, FB>(P, m, n, at.kb0, at.nk);
    if (P.splits > 1) P.partial[((int64_t)at.split * P.M + m) * P.N + n] = v;
    else ((float*)P.C)[m * P.ldc + n] = v + (P.bias ? P.bias[n] : 0.f);
  }
}

template <int BM, int BN, int WGM, int WGN, int S, int FA, int FB, bool EXACT>
__device__ __forceinline__ void tile_item(const Fp8Args& P, int lid) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
  constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
  constexpr int LOADS_A = BM / 8 / NW, LOADS_B = BN / 8 / NW, NPIECE = LOADS_A + LOADS_B;
  constexpr int SCN = 32, W = SCN / 4, ROWS = BM + BN, LOADS_S = ROWS * W / 64 / NW;  // scale words a row, copies a wave
  static_assert(ROWS * W % (64 * NW) == 0, "copies of scales split evenly over the waves");
  static_assert(BM / 8 % NW == 0 && BN / 8 % NW == 0, "copies must split evenly over the waves");
  constexpr int CA = TM >= 2 ? 2 : 1, NC = TM / CA;  // clusters of 64 k
  static_assert(TM % CA == 0, "whole clusters");
  // MID, EARLY: a second barrier in a step
  constexpr bool MID = NC == 2, EARLY = NC == 1 && S == 2 && (!EXACT || TM * TN == 1), TWO = MID || EARLY;
  static_assert(MID ? S == 2 && LOADS_A % 2 == 0 : NC == 1, "a stage in two parts, or in one");
  constexpr int PIECE_E = MID ? LOADS_A / 2 : 0, PIECE_M = NPIECE - PIECE_E;  // copies of the second part, of the first
  __shared__ __attribute__((aligned(1024))) char smem[S * (A_BYTES + B_BYTES) + ROWS * SCN];

  const Place at = place<BM, BN>(P, lid);
  const int64_t m0 = at.m0, n0 = at.n0;
  const int split = at.split, kb0 = at.kb0, nk = at.nk;
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
  auto a_block = [&](int i) {  // 8 rows of A; with MID a wave's first copies are of the first part
    if constexpr (!MID) return wave * LOADS_A + i;
    constexpr int HALF = CA * 4;  // blocks of a part of a wave's rows
    const int t = wave * PIECE_E + i % std::max(1, PIECE_E);
    return t / HALF * 2 * HALF + t % HALF + (i < PIECE_E ? 0 : HALF);
  };
  uint32_t off_a[LOADS_A], off_b[LOADS_B];
#pragma unroll
  for (int i = 0; i < LOADS_A; ++i) {
    const int r = a_block(i) * 8 + (lane >> 3);
    off_a[i] = (uint32_t)min((int64_t)r, P.M - 1 - m0) * (uint32_t)P.lda + 16 * ((lane & 7) ^ ((r >> 1) & 7));
  }
#pragma unroll
  for (int i = 0; i < LOADS_B; ++i) {
    const int r = (wave * LOADS_B + i) * 8 + (lane >> 3);
    off_b[i] = (uint32_t)min((int64_t)r, P.N - 1 - n0) * (uint32_t)P.ldb + 16 * ((lane & 7) ^ ((r >> 1) & 7));
  }
  const char* base_a = (const char*)P.A + m0 * P.lda + (int64_t)kb0 * 128;
  const char* base_b = (const char*)P.B + n0 * P.ldb + (int64_t)kb0 * 128;
  const char* base_e = base_a;
  // a scalar base and the lane's offset, not a pointer for each copy: sixteen
  // registers, with which the 256 x 256 tile's scales and offsets spilled
  auto copy = [&](const char* base, uint32_t off, char* lds) {
    asm volatile("" : "+v"(off));
    copy_block<0>(base + off, lds);
  };
  auto copy_a = [&](const char* base, int slot, int i) {
    copy(base, off_a[i], smem + slot * A_BYTES + a_block(i) * 1024);
  };
  auto issue = [&](int slot, int p) {  // copy p of the next step's first part into a stage
    if (p < LOADS_B) copy(base_b, off_b[p], smem_b + slot * B_BYTES + (wave * LOADS_B + p) * 1024);
    else copy_a(base_a, slot, p - LOADS_B);
    if (p == PIECE_M - 1) {
      base_a += 128;
      base_b += 128;
    }
  };
  auto issue_e = [&](int slot, int p) {  // of the second
    copy_a(base_e, slot, LOADS_A - PIECE_E + p);
    if (p == PIECE_E - 1) base_e += 128;
  };
  // the scale words of steps k0 .. k0 + SCN - 1; past the last one, that again
  char* const smem_s = smem + S * (A_BYTES + B_BYTES);
  auto copy_scales = [&](int k0) {
    int ln = lane;
    asm volatile("" : "+v"(ln));  // no addresses kept in registers for a next round
    const int last = (min(nk - k0, SCN) - 1) >> 2;
    const int in_a = (int)(m0 & ((1 << P.fa) - 1)), in_b = (int)(n0 & ((1 << P.fb) - 1));  // rows into the first block
    const char* sa0 = (const char*)P.sa + (m0 >> P.fa) * P.ldsa + kb0 + k0;
    const char* sb0 = (const char*)P.sb + (n0 >> P.fb) * P.ldsb + kb0 + k0;
    const int max_a = (int)min(P.M - 1 - m0, (int64_t)BM), max_b = (int)min(P.N - 1 - n0, (int64_t)BN);
#pragma unroll
    for (int i = 0; i < LOADS_S; ++i) {
      const int t = (wave * LOADS_S + i) * 64, r0 = t / W, r = r0 + ln / W;
      const int w = min((ln % W) ^ sc_swz<W>(r), last);
      if (r0 < BM)  // uniform: a copy's rows are of one operand
        copy_words<0>(sa0 + ((uint32_t)((min(r, max_a) + in_a) >> P.fa) * (uint32_t)P.ldsa + 4 * w), smem_s + t * 4);
      else
        copy_words<0>(sb0 + ((uint32_t)((min(r - BM, max_b) + in_b) >> P.fb) * (uint32_t)P.ldsb + 4 * w), smem_s + t * 4);
    }
  };

  // fragments: rows 32 i + lane % 32, chunks 2 ks + lane / 32; the swizzle
  // leaves whole blocks of 32 rows alone, and a chunk's number meets it in bits
  // that the stages' and blocks' offsets leave zero
  const uint32_t lds0 = lds_addr(smem);
  const uint32_t frag = chunk_off(lane & 31, lane >> 5);
  const uint32_t frag_a = lds0 + wm * WM * 128, frag_b = lds0 + S * A_BYTES + wn * WN * 128;
  const uint32_t sc = lds0 + S * (A_BYTES + B_BYTES) + 4 * W * (lane & 31);
  uint32_t sa[TM], sb[TN], wa[TM], wb[TN];  // scales in use (EXACT: as floats, else the low byte counts); the words of the step that begins
#pragma unroll
  for (int i = 0; i < TM; ++i) sa[i] = EXACT ? scale_bits(127) : 127;
#pragma unroll
  for (int j = 0; j < TN; ++j) sb[j] = EXACT ? scale_bits(127) : 127;
  Frag af[2][CA], bf[2][TN];
#pragma unroll
  for (int i = 0; i < CA; ++i) af[1][i].lo = af[1][i].hi = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < TN; ++j) bf[1][j].lo = bf[1][j].hi = u32x4{0, 0, 0, 0};

  // cluster q of a step: 64 k number q % 2, row blocks CA (q / 2) ..
  auto read_cluster = [&](auto Q, int kt, int slot) {
    constexpr int q = decltype(Q)::value, h = q & 1, i0 = CA * (q / 2);
    const uint32_t ab = (frag_a + (uint32_t)(slot * A_BYTES) + frag) ^ (64 * h), bb = (frag_b + (uint32_t)(slot * B_BYTES) + frag) ^ (64 * h);
    if constexpr (q == 0) {
      const uint32_t w = 4 * ((kt >> 2) ^ sc_swz<W>(lane));
      static_for<0, TM>([&](auto I) { wa[decltype(I)::value] = lds_read_b32<decltype(I)::value * 128 * W>(sc + w + 4 * W * wm * WM); });
      static_for<0, TN>([&](auto J) { wb[decltype(J)::value] = lds_read_b32<decltype(J)::value * 128 * W>(sc + w + 4 * W * (BM + wn * WN)); });
    }
    if constexpr (q < 2)
      static_for<0, TN>([&](auto J) {
        constexpr int j = decltype(J)::value;
        bf[h][j].lo = lds_read_b128<j * 4096>(bb);
        bf[h][j].hi = lds_read_b128<j * 4096>(bb ^ 32);
      });
    static_for<0, CA>([&](auto I) {
      constexpr int i = decltype(I)::value;
      af[h][i].lo = lds_read_b128<(i0 + i) * 4096>(ab);
      af[h][i].hi = lds_read_b128<(i0 + i) * 4096>(ab ^ 32);
    });
  };
  auto landed = [&](auto Q) {  // the cluster's reads have been waited for
    constexpr int q = decltype(Q)::value, h = q & 1;
    if constexpr (q == 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) after_wait(wa[i]);
#pragma unroll
      for (int j = 0; j < TN; ++j) after_wait(wb[j]);
    }
    if constexpr (q < 2)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        after_wait(bf[h][j].lo);
        after_wait(bf[h][j].hi);
      }
#pragma unroll
    for (int i = 0; i < CA; ++i) {
      after_wait(af[h][i].lo);
      after_wait(af[h][i].hi);
    }
  };
  // COPY 1 (2): with the copies of a later step's first (second) part into stage
  // `slot` between them
  auto multiply = [&](auto Q, auto COPY, int slot) {
    constexpr int q = decltype(Q)::value, h = q & 1, i0 = CA * (q / 2);
    constexpr int which = decltype(COPY)::value, pieces = which == 0 ? 0 : which == 1 ? PIECE_M : PIECE_E;
    // copies between product x of n and the next
    auto copies = [&](int x, int n) {
      const int per = (pieces + n - 1) / n;
#pragma unroll
      for (int p = x * per; p < (x + 1) * per; ++p)
        if (p < pieces) which == 1 ? issue(slot, p) : issue_e(slot, p);
    };
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (EXACT) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // 16 k
        bf16x8 xb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const u32x4& v = x < 2 ? bf[h][j].lo : bf[h][j].hi;
          xb[j] = widen<FB>(v[2 * (x & 1)], v[2 * (x & 1) + 1], __builtin_bit_cast(float, sb[j]));
        }
#pragma unroll
        for (int i = 0; i < CA; ++i) {
          const u32x4& v = x < 2 ? af[h][i].lo : af[h][i].hi;
          const bf16x8 xa = widen<FA>(v[2 * (x & 1)], v[2 * (x & 1) + 1], __builtin_bit_cast(float, sa[i0 + i]));
#pragma unroll
          for (int j = 0; j < TN; ++j)
            acc[i0 + i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[j], xa, acc[i0 + i][j], 0, 0, 0);
        }
        copies(x, 4);
      }
    } else {
#pragma unroll
      for (int i = 0; i < CA; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          product64<FA, FB>(af[h][i], bf[h][j], sa[i0 + i], sb[j], acc[i0 + i][j]);
          if constexpr (pieces > 0) {
            copies(i * TN + j, CA * TN);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  uint64_t wide_at = 0;  // lanes with a scale that bfloat16 cannot carry
  auto advance = [&](int kt) {  // the scales of step kt
    const int sh = 8 * (kt & 3);
    if constexpr (EXACT) {
#pragma unroll
      for (int i = 0; i < TM; ++i) wide_at |= __ballot(too_wide(wa[i] >> sh));
#pragma unroll
      for (int j = 0; j < TN; ++j) wide_at |= __ballot(too_wide(wb[j] >> sh));
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = EXACT ? scale_bits(wa[i] >> sh) : wa[i] >> sh;
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = EXACT ? scale_bits(wb[j] >> sh) : wb[j] >> sh;
  };
  constexpr int LAST = 2 * NC - 1;
  // Step kt of ns.  Copies complete in order, and a step waits for its own alone.
  // TWO: MORE (0 to 2) steps follow at least.  Parts are asked for in the order
  // first, second, first, ..: the first part of step kt + 2 at kt's second
  // barrier, into the stage that kt has read (MID: half read), its second part
  // at kt + 1's first.  Else MORE: step kt + S - 1 exists, and is asked for.
  // No branch between LDS reads and their wait.
  auto k_step = [&](auto MORE, int kt, int ns, int slot) {
    constexpr int more = decltype(MORE)::value;
    const int pslot = slot == 0 ? S - 1 : slot - 1;  // of steps kt - 1 and kt + S - 1
    if constexpr (TWO) {
      WAIT_VMCNT(more ? NPIECE : PIECE_E);
    } else if constexpr (more) {
      WAIT_VMCNT((S - 2) * NPIECE);
    } else {
      const int left = min(S - 2, ns - 1 - kt);  // younger steps still in flight
      static_for<0, S - 1>([&](auto D) {
        constexpr int d = decltype(D)::value;
        if (left == d) WAIT_VMCNT(d * NPIECE);
      });
    }
    barrier_only();
    read_cluster(IntC<0>{}, kt, slot);
    multiply(IntC<LAST>{}, IntC<more == 0 ? 0 : TWO ? 2 : 1>{}, pslot);
    lgkm_wait<0>();
    landed(IntC<0>{});
    advance(kt);
    static_for<0, LAST>([&](auto Q) {
      constexpr int q = decltype(Q)::value;
      if constexpr (MID && q == 1) {
        WAIT_VMCNT(more ? NPIECE : 0);
        barrier_only();
      }
      read_cluster(IntC<q + 1>{}, kt, slot);
      if constexpr (EARLY) {
        lgkm_wait<0>();
        landed(IntC<q + 1>{});
        barrier_only();
        multiply(Q, IntC<more == 2 ? 1 : 0>{}, slot);
      } else {
        multiply(Q, IntC<MID && q == 1 && more == 2 ? 1 : 0>{}, slot);
        lgkm_wait<0>();
        landed(IntC<q + 1>{});
      }
    });
  };
  auto all = [&](int slot) {
#pragma unroll
    for (int p = 0; p < PIECE_M; ++p) issue(slot, p);
  };
  for (int k0 = 0; k0 < nk; k0 += SCN) {
    const int ns = min(nk - k0, SCN);
    if (k0 > 0) barrier_only();  // every wave has read the last stage
    // the first copies before the scales, which the first step waits for too
    int kt = 0, slot = 0;
    if constexpr (TWO) {
      all(0);
      copy_scales(k0);
#pragma unroll
      for (int p = 0; p < PIECE_E; ++p) issue_e(0, p);
      if (ns > 1) all(1);
      for (; kt + 2 < ns; ++kt, slot ^= 1) k_step(IntC<2>{}, kt, ns, slot);
      if (kt + 1 < ns) k_step(IntC<1>{}, kt++, ns, slot), slot ^= 1;
      k_step(IntC<0>{}, kt, ns, slot);
    } else {
#pragma unroll
      for (int t = 0; t < S - 1; ++t) {
        if (t < ns) all(t);
        if (t == 0) copy_scales(k0);
      }
      for (; kt + S - 1 < ns; ++kt) {
        k_step(IntC<1>{}, kt, ns, slot);
        slot = slot + 1 == S ? 0 : slot + 1;
      }
      for (; kt < ns; ++kt) {
        k_step(IntC<0>{}, kt, ns, slot);
        slot = slot + 1 == S ? 0 : slot + 1;
      }
    }
  }
  multiply(IntC<LAST>{}, IntC<0>{}, 0);
  if constexpr (EXACT) {
    if (wide_at) {
      plain_tile<BM, BN, WGM, WGN, FA, FB>();
      return;
    }
  }

  // ---- epilogue, from the registers.  A lane has columns 8 q + 4 (l/32) ..+3
  // of row l%32 for q = 0..3; exchanges between lane groups gather 16 bytes of
  // a row in a lane and 64 bytes of it in four lanes, so a store covers sixteen
  // rows' 64-byte pieces.  The pieces carry the alignment of one element (element
  // by element 8192 x 2303 x 768 took 66 us, now 39; 2304 columns 24); what the
  // last column cuts goes by the element.
  //
  // Stores around the caches are not used: alone the product mostly gains (4096 x
  // 14592 x 512 67 -> 59 us, 8192 x 8512 x 1536 140 -> 123), but whoever reads the
  // result next pays more (with a quantiser behind it 102 -> 112 and 182 -> 183; 40
  // to 256 MB of results at three K: up to 16 % lost, at most 3 % won).  Up to 20 MB
  // of whole 64-byte pieces product and reader win 1 % on average, and off those
  // lose up to 19 % (8192 x 1000 x 600 20.8 -> 24.7).
  const bool part = P.splits > 1;
  const bool wide = part || EXACT;  // float32 stores
  float* const cf = part ? P.partial + (int64_t)split * P.M * P.N : (float*)P.C;
  const int64_t ldc = part ? P.N : P.ldc;
  const float* const bias = part ? nullptr : P.bias;
  const int hf = lane >> 5, l16 = (lane >> 4) & 1, l4 = lane & 15;
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t nb = n0 + wn * WN + j * 32;
    if (bias) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int64_t n = nb + 8 * q + 4 * hf + t;
          const float x = n < P.N ? bias[n] : 0.f;
#pragma unroll
          for (int i = 0; i < TM; ++i) acc[i][j][4 * q + t] += x;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t mb = m0 + wm * WM + i * 32;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int64_t nb = n0 + wn * WN + j * 32;
      if (wide) {
        // q pairs: columns 16 p .. + 15
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uint32_t x[4], y[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const float u = acc[i][j][8 * p + t], v = acc[i][j][8 * p + 4 + t];
            x[t] = __builtin_bit_cast(uint32_t, u);
            y[t] = __builtin_bit_cast(uint32_t, v);
            swap16(x[t], y[t]);  // x: rows 0..15, y: rows 16..31; odd lane groups: columns 8 ..
          }
          const int64_t n = nb + 16 * p + 8 * l16 + 4 * hf;
          typedef u32x4 V __attribute__((aligned(4)));
          uint32_t* const to = reinterpret_cast<uint32_t*>(cf + (mb + l4) * ldc + n);
          uint32_t* const to2 = to + 16 * ldc;
          if (n + 4 <= P.N) {
            if (mb + l4 < P.M) *reinterpret_cast<V*>(to) = u32x4{x[0], x[1], x[2], x[3]};
            if (mb + 16 + l4 < P.M) *reinterpret_cast<V*>(to2) = u32x4{y[0], y[1], y[2], y[3]};
          } else if (n < P.N) {
#pragma unroll
            for (int t = 0; t < 3; ++t) {
              if (n + t < P.N && mb + l4 < P.M) to[t] = x[t];
              if (n + t < P.N && mb + 16 + l4 < P.M) to2[t] = y[t];
            }
          }
        }
      } else {
        uint32_t w[2][4];  // columns 16 p + 8 (l/32) .. + 7 of row l%32
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const f32x16& v = acc[i][j];
          w[p][0] = pack_bf2(v[8 * p], v[8 * p + 1]);
          w[p][1] = pack_bf2(v[8 * p + 2], v[8 * p + 3]);
          w[p][2] = pack_bf2(v[8 * p + 4], v[8 * p + 5]);
          w[p][3] = pack_bf2(v[8 * p + 6], v[8 * p + 7]);
          swap32(w[p][0], w[p][2]);
          swap32(w[p][1], w[p][3]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) swap16(w[0][t], w[1][t]);  // w[y]: row 16 y + l%16, columns 16 (l/16 odd) + 8 (l/32)
        const int64_t n = nb + 16 * l16 + 8 * hf;
        typedef u32x4 V __attribute__((aligned(2)));
        bf16_t* const to[2] = {(bf16_t*)P.C + (mb + l4) * ldc + n, (bf16_t*)P.C + (mb + 16 + l4) * ldc + n};
        if (n + 8 <= P.N) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            if (mb + 16 * y + l4 < P.M) *reinterpret_cast<V*>(to[y]) = u32x4{w[y][0], w[y][1], w[y][2], w[y][3]};
          }
        } else if (n < P.N) {
#pragma unroll
          for (int y = 0; y < 2; ++y)
            if (mb + 16 * y + l4 < P.M)
#pragma unroll
              for (int t = 0; t < 7; ++t)
                if (n + t < P.N) to[y][t] = (bf16_t)(w[y][t >> 1] >> (16 * (t & 1)));
        }
      }
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

// -------------------------------------------------------- few rows of A
// M <= 32 (serving): bound by the stream of B, which goes from memory to the
// matrix cores without LDS.  A workgroup takes 16 columns (16x16x128 products),
// its waves share K in groups of four blocks (512 k, one word of scales a row),
// a group's loads all in flight at once.  Of a block a lane takes the 16-byte
// chunks l/16 and 4 + l/16 of row l%16, so a load covers 64 neighbouring bytes
// of sixteen rows (with 32 columns and 32x32x64 products, 32 bytes of 32 rows:
// 1 x 2048 x 8192 took 11.8 us).  The waves' sums meet in LDS and are added in
// wave order.
template <int TM, int FA, int FB, bool EXACT>
__global__ __launch_bounds__(1024) void gemm_fp8_rows_kernel(const Fp8Args P) {
  __shared__ float sums[16][TM * 4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int64_t rb = min(n0 + (lane & 15), P.N - 1);
  const uint8_t* b = P.B + rb * P.ldb + 16 * (lane >> 4);
  const uint32_t* sb = reinterpret_cast<const uint32_t*>(P.sb + (rb >> P.fb) * P.ldsb);
  const uint8_t* a[TM];
  const uint32_t* sa[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t ra = min((int64_t)16 * i + (lane & 15), P.M - 1);
    a[i] = P.A + ra * P.lda + 16 * (lane >> 4);
    sa[i] = reinterpret_cast<const uint32_t*>(P.sa + (ra >> P.fa) * P.ldsa);
  }
  f32x4 acc[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto load = [](const uint8_t* p, int block) {
    p += (int64_t)block * 128;
    return Frag{*reinterpret_cast<const u32x4*>(p), *reinterpret_cast<const u32x4*>(p + 64)};
  };
  // a block's 128 k: lane l has column l%16 and rows 4 (l/16) .. + 3 of the sum
  auto block = [&](const Frag& x, const Frag& y, uint32_t ea, uint32_t eb, f32x4& c) {
    if constexpr (EXACT) {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const u32x4 &xv = h < 2 ? x.lo : x.hi, &yv = h < 2 ? y.lo : y.hi;
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FA>(xv[2 * (h & 1)], xv[2 * (h & 1) + 1], scale_of(ea)),
                                                    widen<FB>(yv[2 * (h & 1)], yv[2 * (h & 1) + 1], scale_of(eb)), c, 0, 0, 0);
      }
    } else {
      c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(words(x), words(y), c, FA, FB, 0, (int)ea, 0, (int)eb);
    }
  };
  bool wide = false;
  for (int g = wave; 4 * g < P.kb; g += nw) {
    uint32_t wa[TM];
    const uint32_t wb = sb[g];
#pragma unroll
    for (int i = 0; i < TM; ++i) wa[i] = sa[i][g];
    if constexpr (EXACT) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (4 * g + k >= P.kb) break;
        wide |= too_wide(wb >> (8 * k));
#pragma unroll
        for (int i = 0; i < TM; ++i) wide |= too_wide(wa[i] >> (8 * k));
      }
    }
    if (4 * g + 4 <= P.kb) {
      Frag y[4], x[TM][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        y[k] = load(b, 4 * g + k);
#pragma unroll
        for (int i = 0; i < TM; ++i) x[i][k] = load(a[i], 4 * g + k);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < TM; ++i) block(x[i][k], y[k], wa[i] >> (8 * k), wb >> (8 * k), acc[i]);
    } else {
      for (int k = 0; 4 * g + k < P.kb; ++k) {
        const Frag y = load(b, 4 * g + k);
#pragma unroll
        for (int i = 0; i < TM; ++i) block(load(a[i], 4 * g + k), y, wa[i] >> (8 * k), wb >> (8 * k), acc[i]);
      }
    }
  }
  if constexpr (EXACT) {
    if (__any(wide)) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t m = min((int64_t)16 * i + 4 * (lane >> 4) + r, P.M - 1);
          float v = 0.f;
#pragma unroll 1
          for (int g = wave; 4 * g < P.kb; g += nw) v += plain_sum<FA, FB>(P, m, rb, 4 * g, min(4, P.kb - 4 * g));
          acc[i][r] = v;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][4 * i + r][lane] = acc[i][r];
  __syncthreads();
  for (int t = threadIdx.x; t < TM * 256; t += blockDim.x) {
    const int i = t >> 8, r = (t >> 6) & 3, l = t & 63;
    const int64_t m = 16 * i + 4 * (l >> 4) + r, n = n0 + (l & 15);
    if (m >= P.M || n >= P.N) continue;
    float v = 0.f;
    for (int w = 0; w < nw; ++w) v += sums[w][4 * i + r][l];
    if (P.bias) v += P.bias[n];
    if (EXACT) ((float*)P.C)[m * P.ldc + n] = v;
    else ((bf16_t*)P.C)[m * P.ldc + n] = f2bf(v);
  }
}

template <int TM, int FA, int FB>
hipError_t launch_rows(const Fp8Args& P, hipStream_t s) {
  const int nw = (int)std::min<int64_t>(16, cdiv(P.kb, 4));
  const unsigned grid = (unsigned)cdiv(P.N, 16);
  if (P.c_f32) gemm_fp8_rows_kernel<TM, FA, FB, true><<<grid, 64 * nw, 0, s>>>(P);
  else gemm_fp8_rows_kernel<TM, FA, FB, false><<<grid, 64 * nw, 0, s>>>(P);
  return hipGetLastError();
}

// Blocks of 256 threads that go through n items at the grid's distance.
unsigned element_blocks(int64_t n) { return (unsigned)std::min(cdiv(n, 256), MAX_LAUNCH_THREADS / 256); }

// Sum of the split-K partials in split order, bias, rounding: four columns of
// a row a thread.
__global__ __launch_bounds__(256) void fp8_reduce_kernel(const Fp8Args P) {
  const int64_t nq = (P.N + 3) / 4, total = P.M * P.N;
  for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < P.M * nq; idx += (int64_t)gridDim.x * 256) {
    const int64_t m = idx / nq, n = (idx - m * nq) * 4;
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
}

template <int BM, int BN, int WGM, int WGN, int S, int OCC, int FA, int FB>
hipError_t launch_tiles(const Fp8Args& P, hipStream_t s) {
  const int64_t n = (int64_t)P.tiles_m * P.tiles_n * P.splits;
  const unsigned grid = (unsigned)((n + 7) / 8 * 8);
  constexpr int NT = 64 * WGM * WGN;
  if (P.c_f32) gemm_fp8_kernel<BM, BN, WGM, WGN, S, OCC, FA, FB, true><<<grid, NT, 0, s>>>(P);
  else gemm_fp8_kernel<BM, BN, WGM, WGN, S, OCC, FA, FB, false><<<grid, NT, 0, s>>>(P);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || P.splits == 1) return e;
  fp8_reduce_kernel<<<element_blocks(P.M * cdiv(P.N, 4)), 256, 0, s>>>(P);
  return hipGetLastError();
}

enum TileId { T256x256 = 0, T256x128, T128x128, T64x64, T_ROWS, kNumCfg };
// Estimate of a product's time.  occ workgroups share a CU; a step of 128 k
// takes lo us alone on a CU and hi with the CU full (occ = 1: on an empty and
// on a full chip), a tile fix us besides (first copies, stores), a byte of C
// 1 / gbs ns.  Fitted to 9600 timings of 700 products of 64 to 8192 a side, drawn
// at random, with operands and result in rotation (off by 7 to 12 % of a time);
// on 130 products not among them the choice takes 1.008 of the best tile and
// split's time on average, 1.12 at most (among the 700 1.25), bfloat16 and float32
// results alike.
// [0]: bfloat16 results, [1]: float32.
struct TileCfg {
  int bm, bn, threads, occ;
  struct {
    float lo, hi, fix, gbs;
  } t[2];
};
const TileCfg kCfgs[kNumCfg] = {
    {256, 256, 512, 1, {{1.07f, 1.18f, 5.4f, 4420.f}, {2.26f, 2.50f, 6.5f, 5370.f}}},  // 2 x 4 waves, 2 stages
    {256, 128, 512, 1, {{0.61f, 0.68f, 3.5f, 4450.f}, {1.30f, 1.40f, 4.2f, 5870.f}}},  // 4 x 2 waves, 3 stages
    {128, 128, 256, 2, {{0.47f, 0.74f, 2.6f, 4560.f}, {0.80f, 1.33f, 3.1f, 5700.f}}},  // 2 x 2 waves, 2 stages
    {64, 64, 256, 4, {{0.28f, 0.57f, 1.3f, 3710.f}, {0.39f, 0.95f, 1.8f, 5950.f}}},    // 2 x 2 waves, 2 stages
    {32, 16, 1024, 1, {}},
};

float estimate(int64_t M, int64_t N, int kb, bool f32, const TileCfg& c, int splits) {
  const auto& t = c.t[f32];
  int64_t steps = cdiv(kb, splits);
  if (splits > 1) steps = cdiv(steps, 4) * 4;
  splits = (int)cdiv(kb, steps);
  const int64_t n = cdiv(M, c.bm) * cdiv(N, c.bn) * splits, q = cdiv(n, 256);  // tiles of the fullest CU
  auto step = [&](int64_t k) {
    const float x = c.occ > 1 ? (float)(k - 1) / (c.occ - 1) : std::min(1.f, n / 256.f);
    return t.lo + (t.hi - t.lo) * x;
  };
  float us = (q / c.occ) * (steps * step(c.occ) + t.fix);
  if (q % c.occ) us += steps * step(q % c.occ) + t.fix;
  const float out = (float)M * N * (f32 ? 4.f : 2.f);
  // the partial results are written and read at 4 TB/s, by one launch more
  return splits > 1 ? us + 5.f + splits * (float)M * N * 8.f * 0.25e-6f : us + out * 1e-3f / t.gbs;
}

template <int FA, int FB>
hipError_t launch_cfg(const Fp8Args& P, int cfg, hipStream_t s) {
  switch (cfg) {
    case T256x256: return launch_tiles<256, 256, 2, 4, 2, 1, FA, FB>(P, s);
    case T256x128: return launch_tiles<256, 128, 4, 2, 3, 1, FA, FB>(P, s);
    case T128x128: return launch_tiles<128, 128, 2, 2, 2, 2, FA, FB>(P, s);
    case T64x64: return launch_tiles<64, 64, 2, 2, 2, 4, FA, FB>(P, s);
    default: return P.M <= 16 ? launch_rows<1, FA, FB>(P, s) : launch_rows<2, FA, FB>(P, s);
  }
}

// Columns of C without a product: the bias, or zero.
__global__ __launch_bounds__(256) void fp8_bias_kernel(const Fp8Args P) {
  for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < P.M * P.N; idx += (int64_t)gridDim.x * 256) {
    const int64_t m = idx / P.N, n = idx - m * P.N;
    const float x = P.bias ? P.bias[n] : 0.f;
    if (P.c_f32) ((float*)P.C)[m * P.ldc + n] = x;
    else ((bf16_t*)P.C)[m * P.ldc + n] = f2bf(x);
  }
}

}  // namespace

hipError_t launch_gemm_fp8_cfg(const layup_gemm_fp8_desc& d, int cfg, int splits, hipStream_t s, int64_t max_threads) {
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
    fp8_bias_kernel<<<element_blocks(P.M * P.N), 256, 0, s>>>(P);
    return hipGetLastError();
  }
  if (cfg < 0 || cfg >= kNumCfg || (cfg == T_ROWS && (d.M > 32 || splits > 1))) return hipErrorInvalidValue;
  P.kb_split = (int32_t)(cdiv(cdiv(P.kb, std::max(1, splits)), 4) * 4);
  P.splits = (int32_t)cdiv(P.kb, P.kb_split);
  if (P.splits > 1 && (!d.workspace || d.workspace_bytes < (size_t)P.splits * P.M * P.N * 4)) return hipErrorInvalidValue;
  const bool a4 = d.a_dtype == LAYUP_E4M3, b4 = d.b_dtype == LAYUP_E4M3;
  // What one launch cannot take goes in slices of whole tiles, eight at least
  // (scale blocks of 128 rows stay whole).  The slices' partial results follow
  // one another through the same workspace.
  const TileCfg& t = kCfgs[cfg];
  auto slice = [](int64_t tiles, int64_t most) { return tiles <= most ? tiles : std::max<int64_t>(8, most / 8 * 8); };
  const int64_t most = (max_threads / t.threads - 7) / P.splits;  // a launch's tiles go up to a multiple of 8
  const int64_t rows = slice(cdiv(P.M, t.bm), most) * t.bm, cols = slice(cdiv(P.N, t.bn), most / (rows / t.bm)) * t.bn;
  for (int64_t m = 0; m < d.M; m += rows)
    for (int64_t n = 0; n < d.N; n += cols) {
      Fp8Args Q = P;
      Q.M = std::min(rows, d.M - m);
      Q.N = std::min(cols, d.N - n);
      Q.A += m * P.lda;
      Q.B += n * P.ldb;
      Q.sa += (m >> P.fa) * P.ldsa;
      Q.sb += (n >> P.fb) * P.ldsb;
      Q.C = (char*)P.C + (m * P.ldc + n) * (P.c_f32 ? 4 : 2);
      if (P.bias) Q.bias += n;
      Q.tiles_m = (int32_t)cdiv(Q.M, t.bm);
      Q.tiles_n = (int32_t)cdiv(Q.N, t.bn);
      const hipError_t e = a4 ? (b4 ? launch_cfg<0, 0>(Q, cfg, s) : launch_cfg<0, 1>(Q, cfg, s))
                              : (b4 ? launch_cfg<1, 0>(Q, cfg, s) : launch_cfg<1, 1>(Q, cfg, s));
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

hipError_t launch_gemm_fp8(const layup_gemm_fp8_desc& d, hipStream_t s) {
  if (d.M <= 32) return launch_gemm_fp8_cfg(d, T_ROWS, 1, s);
  const int kb = (int)cdiv(d.K, 128);
  int cfg = T64x64, splits = 1;
  float best = 1e30f;
  for (int c = 0; c < T_ROWS; ++c)
    for (int sp = 1; sp <= 16; sp *= 2) {
      // whole words of scales a split, partial results that fit
      if (sp > 1 && (kb < 4 * sp || !d.workspace || d.workspace_bytes / 4 / sp < (size_t)d.M * d.N)) break;
      const float us = estimate(d.M, d.N, kb, d.c_f32 != 0, kCfgs[c], sp);
      if (us < best) {
        best = us;
        cfg = c;
        splits = sp;
      }
    }
  return launch_gemm_fp8_cfg(d, cfg, splits, s);
}

}  // namespace layup
