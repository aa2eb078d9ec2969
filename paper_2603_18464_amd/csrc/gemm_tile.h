// The kernel template of the half-precision MFMA products C[M,N] = A[M,K] * W[N,K]^T, for the epilogues of gemm_f16.hip and
// head_loss.hip.  An epilogue is a struct with kSpan, the columns of a row that have to be handed over together, and
//   consume<COLS, PITCH, ROWS>(tile, m_base, nb, lane, M): rows m_base .. + ROWS - 1 and columns nb .. + COLS - 1 of
//   the product, element (r, c) at tile[r * PITCH + c] of the LDS; the tile is this wave's own until it returns.
#pragma once
#include <cmath>
#include <type_traits>
#include <utility>

#include "common.h"

namespace vla {

// ---- 8-bit low terms --------------------------------------------------------------------------------------
// Two-term activations may carry their low term as one byte: lo8 = bf8(16 * (a - f16(a))) (1-5-2 format), behind the
// Kw high terms of a block of 32 rows (act_lo8_index).  The low-term product then runs
// on v_mfma_f32_16x16x128 in 8-bit formats (twice the rate of the half-precision instruction) against a second
// copy of the weights, W8 = fp8(w * 16) (1-4-3 format, saturating at +-448, i.e. |w| = 28), so that
// lo8 * W8 = 2^8 * lo * w lands in the same accumulator as hi * (w * 2^8).  The correction term only has to be good
// to a few percent (it is itself 2^-12 of the result), which three and two mantissa bits give.
// Layout: 128 k of lo8 have the geometry of 64 k of hi (4 KiB of 32 rows): the 16-byte chunk c (16 k) of a row lies where
// the 16-byte chunk c (8 k) of the row lies in the halves, and W8 is packed likewise; a lane's operand of the 128-deep product is
// its 16 bytes of k-step 0 followed by its 16 bytes of k-step 1, for both operands.
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
__device__ __forceinline__ f32x4 mfma_lo8(const f16x8& a0, const f16x8& a1, const f16x8& b0, const f16x8& b1,
                                          const f32x4& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8 a = __builtin_shufflevector(__builtin_bit_cast(i32x4, a0), __builtin_bit_cast(i32x4, a1), 0, 1, 2, 3, 4, 5, 6, 7);
  const i32x8 b = __builtin_shufflevector(__builtin_bit_cast(i32x4, b0), __builtin_bit_cast(i32x4, b1), 0, 1, 2, 3, 4, 5, 6, 7);
  // A: bf8 (format 1), B: fp8 (format 0), no block scales
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 1, 0, 0, 0, 0, 0);
#else
  return c;
#endif
}

// ---- the kernel ---------------------------------------------------------------------------------------------
// One kernel template for every size: a workgroup of WGM x WGN waves computes a BM x BN tile (a wave WM x WN of it).
//
// * Slabs of PK k of A and W go straight from global memory into LDS (global_load_lds_dwordx4: lane l of a wave
//   instruction deposits its 16 bytes at the wave-uniform LDS base + 16*l), S slabs of A and SW of W ahead of the MFMAs,
//   through a ring of stages each; one barrier per slab publishes the landed slab and frees the one everybody has in
//   registers.  A comes from the L2 and W, in a launch of few tiles, from HBM: where the 160 KiB do not hold another stage of
//   both they hold a third one of W.  Against two stages of each: 192x256 at 290 rows 79 -> 62 us (qkv), 84 -> 68 (gate/up),
//   191 -> 142 (down), at 18560 rows 1811 -> 1652, 2846 -> 2656, 1760 -> 1493; 256x256 at 290 rows 88 -> 75, 94 -> 82,
//   212 -> 180, at 18560 rows down 1443 -> 1377 and with low terms 2381 -> 2315, 3988 -> 3900, 2125 -> 1987.
// * SPREAD: the weights of a slab are requested a k-step after its activations, so that the loads go out evenly.
// * Both slabs are in fragment order, so that a load is one KiB from one place, with a scalar offset, and a read of the LDS has no
//   bank conflicts.  A row-major A took an address a lane and eight pieces of 128 bytes a load: us, 18560 rows, that / this,
//   gate/up 2450 / 2372, down 1336 / 1314, o 548 / 535, with low terms 4 % (gate/up) and 2.5 % (qkv) less, qkv 0 to 2 % more
//   (1377 / 1404, 1412 / 1427, 1396 / 1394 on three cards); 2338 rows
//   gate/up 346 / 336, down 176 / 173.  On operands of zeros, where the clock does not drop, 1834 / 1741, 1113 / 977, 465 / 434:
//   most of what it saves goes into the power limit.
// * Four waves of 128x128 for the residual add's 256x256 tiles: a third fewer reads of the LDS than eight of 64x128, down 1314 ->
//   1269, o 535 -> 530.  The accumulators are the 256 registers of the accumulation half.  With the other epilogues and with low
//   terms, which two waves a SIMD cover better, gate/up 2372 -> 2450, qkv 1388 -> 1441, qkv with low terms 2190 -> 2349.
// * What bounds the large launches: without the loads of the main loop gate/up takes 2120 of 2546 us (row-major A), without its
//   reads of the LDS too 1568; barriers cost nothing; how the loads are spread over the k-steps makes no difference.
// * Fragments are double buffered in registers: while the MFMAs of one k-step run, the reads of the next
//   are in flight, slotted one by one between the MFMAs.  The compiler cannot tell the stages apart and would wait
//   for ALL outstanding LDS loads before any LDS read, so the reads are inline assembly and the waits explicit.
// * The instruction: 16x16x32.  On real operands the matrix cores are limited by power, not issue: an MFMA-only loop on
//   weight bits (vla_probe) sustains 1.76 PFLOP/s with 16x16x32 (half the accumulator traffic per product) against 1.59
//   with 32x32x16.  In this kernel that is 2.59 ms instead of 2.85 (gate/up, 18560 x 22016 x 4096),
//   1.40 instead of 1.48 (down), 0.56 instead of 0.61 (o).
// * DEEP: the fragments are read a whole slab ahead, for launches of at most 256 of the smallest tiles, where a k-step of four
//   products a wave is shorter than the reads of the next one take.  With eight waves of 32x32 instead of four of 32x64 and
//   four stages (whose number costs instructions where it is not a power of two) a slab of the 64x128 tile is 0.25 us instead
//   of 0.33: 290 rows, N 768: K 2048 12.7 -> 9.6 us, K 768 7.3 -> 6.2; N 4096 K 4096 from the caches 25 -> 20, with weights
//   from HBM 27 and 28 (K 11008 67 and 67).  Larger tiles gain nothing (128x256 at 290 and 2338 rows +-1 %).
// * A pass of 8-bit low terms (LO8) follows on 16x16x128: both k-steps of a slab are one product, so the two register
//   buffers hold one slab and there is none to spare for the next.  Each register is refilled as soon as its last
//   product has issued instead: a slab runs as two halves of the wave's rows, the first half's A fragments are refilled
//   during the second half, a column's B fragments behind their last product there, and the second half's A fragments
//   at its end, so that every refill has half a slab of products to arrive under.
//   Against 4 waves of 128x128 with 32x32x16 and 32x32x64 the 7B policy step of 64 takes 244.5 instead of 247.5 ms (its
//   4 two-term layers are a sixth of it), of 8 54.0 instead of 54.2, the 12-layer model's of 32 6.24 instead of 6.29;
//   with 128x256 tiles at every size 247.9, 54.3 and 6.22.
// * Every variant runs the same sequence of MFMAs per output element (k ascending, one chain), so a sequence's bits do
//   not depend on which tile its batch selects.

// 16 bytes per lane from global memory straight into LDS at lds_wave_base + 16 * lane.  base and soff (bytes) are the same
// for the whole wave and live in scalar registers, off is the lane's offset in bytes: a buffer load takes the three as
// they are, where a 64-bit address per lane would cost an addition and two registers a load (with the pass of low terms
// those registers spilled).  The builtins only exist in the device pass; the host pass just needs the kernel's stub.
__device__ __forceinline__ void load_to_lds_16(const f16* base, unsigned off, unsigned soff, f16* lds_wave_base) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, -1, 0x00027000);   // raw, 4 GiB
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds_wave_base, 16, off, soff, 0, 0);
#else
  (void)base;
  (void)off;
  (void)soff;
  (void)lds_wave_base;
#endif
}
// One fragment read with a compile-time byte offset (no wait: the register must not be touched before wait_lds() and
// hold() have been executed).
template <int OFF>
__device__ __forceinline__ void read_frag_asm(f16x8& dst, unsigned addr) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF) : "memory");
#endif
}
// Until at most N of the reads issued so far are outstanding (they return in order; a scalar load in flight counts as
// well, which can only make the wait longer).
template <int N = 0>
__device__ __forceinline__ void wait_lds() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N < 15 ? N : 15) : "memory");
#endif
}
// Ties a fragment to the wait before it: nothing that uses it can be scheduled above.
__device__ __forceinline__ void hold(f16x8& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
#endif
}
#define VLA_INLINE __attribute__((always_inline))    // the kernel's lambdas: a call would put the captured arrays in memory
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  [&]<int... I>(std::integer_sequence<int, I...>) VLA_INLINE { (f(std::integral_constant<int, I>{}), ...); }
  (std::make_integer_sequence<int, N>{});
}

// acc += a * b, the sum in the registers of acc.  With two loops over the same accumulators the compiler gives the
// products of the first separate source and result registers, and the 256 of a wave run out (12 spilled, reloaded in
// the loop with a wait for every load in flight).  The compiler does not know the latency of the statement: settle()
// before anything but another of these touches the accumulators.
// AGPR: the accumulators are in the accumulation half of the register file (a wave of 128x128 has 256 of them, which is all of
// it; left to itself the compiler moves them back and forth).
template <bool AGPR>
__device__ __forceinline__ void mfma_in_place(f32x4& acc, const f16x8& a, const f16x8& b) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (AGPR) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
#endif
}
// The wait on both sides of a run of such products (8 issue slots behind a product, 2 in front of one; 32 given), eight
// accumulators a statement.  It takes them and gives them back, so whatever reads them, register copies included,
// depends on it.
template <bool AGPR, int MT, int NT>
__device__ __forceinline__ void settle(f32x4 (&acc)[MT][NT]) {
  static_assert(MT * NT % 4 == 0, "whole groups of eight, and one of four");
#if defined(__HIP_DEVICE_COMPILE__)
#define VLA_ACC(c, j) "+" c(acc[(g + j) / NT][(g + j) % NT])
#define VLA_SETTLE4(c) asm volatile("s_nop 15\n\ts_nop 15" : VLA_ACC(c, 0), VLA_ACC(c, 1), VLA_ACC(c, 2), VLA_ACC(c, 3))
#define VLA_SETTLE8(c)                                                                                                            \
  asm volatile("s_nop 15\n\ts_nop 15" : VLA_ACC(c, 0), VLA_ACC(c, 1), VLA_ACC(c, 2), VLA_ACC(c, 3), VLA_ACC(c, 4), VLA_ACC(c, 5), \
               VLA_ACC(c, 6), VLA_ACC(c, 7))
  constexpr int EIGHTS = MT * NT / 8 * 8;
#pragma unroll
  for (int g = 0; g < EIGHTS; g += 8) {
    if constexpr (AGPR) VLA_SETTLE8("a");
    else VLA_SETTLE8("v");
  }
  if constexpr (EIGHTS < MT * NT) {
    constexpr int g = EIGHTS;
    if constexpr (AGPR) VLA_SETTLE4("a");
    else VLA_SETTLE4("v");
  }
#undef VLA_SETTLE8
#undef VLA_SETTLE4
#undef VLA_ACC
#endif
}

constexpr int PK = 64;                                 // k of a slab (a slab of low terms is one 128-deep product)

// What an epilogue may ask of the kernel besides:
//   kRaw 1: W is not packed but bfloat16 rows [N, K], raw_ld apart, of which raw_rows exist: re-encoded (w * kWeightScale)
//        between the LDS and the matrix cores.  K % 64 == 0.
//   kRaw 2: W is bfloat16 rows [K, N], raw_ld apart, of which raw_rows (contraction) and raw_cols (a multiple of 8) exist;
//        read transposed from the LDS.  raw_rows > K - 64; A must be zero where its contraction goes past raw_rows.
//   kSliced: tiles of each of `slices` slices of the contraction; slice() is told which one.
//   kPair: two products in one launch, the second one's operands, sizes and tiles in the epilogue, its workgroups from `split` (a
//        multiple of 8) on; `second` tells the epilogue which it is.
//   begin(lane): once a wave, in front of the first consume.
template <class Epi> consteval int raw_w() {
  if constexpr (requires { Epi::kRaw; }) return Epi::kRaw;
  else return 0;
}
template <class Epi> consteval bool sliced() {
  if constexpr (requires { Epi::kSliced; }) return Epi::kSliced;
  else return false;
}
template <class Epi> consteval bool paired() {
  if constexpr (requires { Epi::kPair; }) return Epi::kPair;
  else return false;
}
template <class Epi> __device__ __forceinline__ int slices_of_launch(const Epi& e) {
  if constexpr (paired<Epi>()) return e.second ? e.head.slices : e.hidden.slices;
  else if constexpr (sliced<Epi>()) return e.slices;
  else return 1;
}
template <class Epi> __device__ __forceinline__ int raw_rows_of(const Epi& e) {
  if constexpr (requires { e.raw_rows; }) return e.raw_rows;
  else return 1;
}
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
// Four k of one column a lane, of a block of 4 k x 16 columns that 16 lanes address in pieces of four columns (no wait).
template <int OFF>
__device__ __forceinline__ void read_transposed_asm(u32x2& dst, unsigned addr) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF) : "memory");
#endif
}
__device__ __forceinline__ void hold(u32x2& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
}
// Eight bfloat16 weights as the half-precision operands of the matrix cores.
__device__ __forceinline__ f16x8 encode_weights(const u32x4& v) {
  f16x8 o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    o[2 * j] = (f16)(__builtin_bit_cast(float, v[j] << 16) * kWeightScale);
    o[2 * j + 1] = (f16)(__builtin_bit_cast(float, v[j] & 0xffff0000u) * kWeightScale);
  }
  return o;
}

template <class Epi> __device__ __forceinline__ const f16* epi_a_lo(const Epi&) { return nullptr; }

// The accumulators of a wave's 16 MT x 16 NT, rows m_wave .. and column group wn of a tile's columns n0 .., through LDS to the
// epilogue.
template <int MT, int NT, int WGN, class Epi>
__device__ __forceinline__ void store_tile(f32x4 (&acc)[MT][NT], const Epi& epi, unsigned char* smem, int wave, int wn, int lane,
                                           int m_wave, int n0, int M) {
  // The pitch keeps the stores of a 32-row group conflict free: the four row groups a store instruction covers start 16
  // banks apart.
  constexpr bool PAIR = 16 * NT < Epi::kSpan;               // two waves side by side share a staging tile
  static_assert(!PAIR || (WGN % 2 == 0 && 32 * NT >= Epi::kSpan), "an epilogue's span is one or two wave tiles");
  constexpr int COLS = PAIR ? 32 * NT : 16 * NT, PITCH = COLS + 4, ROWS = PAIR ? 16 : 32;
  float* tile = (float*)smem + (PAIR ? wave >> 1 : wave) * 32 * PITCH;
  const int side = PAIR ? wn & 1 : 0;
#pragma unroll
  for (int mb = 0; mb < MT / 2; ++mb) {
    if constexpr (PAIR) {
      if (mb > 0) __syncthreads();                     // the partner has read the previous rows
    }
#pragma unroll
    for (int mi = 0; mi < 2; ++mi)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          tile[(mi * 16 + 4 * (lane >> 4) + e) * PITCH + side * 16 * NT + nt * 16 + (lane & 15)] = acc[mb * 2 + mi][nt][e];
    if constexpr (PAIR) __syncthreads();
    epi.template consume<COLS, PITCH, ROWS>(tile + side * ROWS * PITCH, m_wave + mb * 32 + side * ROWS,
                                            n0 + (PAIR ? wn >> 1 : wn) * COLS, lane, M);
  }
  if constexpr (MT % 2 != 0) {                         // the last 16 rows
    if constexpr (PAIR) __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        tile[(4 * (lane >> 4) + e) * PITCH + side * 16 * NT + nt * 16 + (lane & 15)] = acc[MT - 1][nt][e];
    if constexpr (PAIR) __syncthreads();
    epi.template consume<COLS, PITCH, ROWS / 2>(tile + side * (ROWS / 2) * PITCH, m_wave + (MT - 1) * 16 + side * (ROWS / 2),
                                                n0 + (PAIR ? wn >> 1 : wn) * COLS, lane, M);
  }
}

// LO8: the launch has slabs of 8-bit low terms (W8 != nullptr): K == 1.5 * Kw, A row = [hi: Kw halves | lo8: Kw bytes].
// Otherwise K == Kw, or K == 2 * Kw (half-precision low terms behind the high terms: the weight slabs wrap).
// SPLITK (with EpiPartial; one row of tiles, M <= BM): the low terms of two-term operands are in a second buffer of the order of
// the first, tiles_m is the number of K slices, and workgroup (tile column tn, slice kz) accumulates slice kz of K only.
template <int WGM, int WGN, int WM, int WN, int S, int SW, int OCC, bool DEEP, bool SPREAD, class Epi, bool LO8, bool SPLITK>
__global__ __launch_bounds__(WGM* WGN * 64, OCC) void gemm_f16_kernel(const f16* __restrict__ A, int lda,
                                                                   const f16* __restrict__ Wp,
                                                                   const f16* __restrict__ W8, int M, int K, int Kw,
                                                                   int tiles_m, int tiles_n, Epi epi_in) {
  constexpr int NW = WGM * WGN, BM = WGM * WM, BN = WGN * WN, MT = WM / 16, NT = WN / 16;
  constexpr bool AGPR = MT * NT == 64;
  static_assert(!AGPR || !LO8, "the products of low terms leave their accumulators to the compiler");
  constexpr int KS = PK / 32, KS16 = PK / 16;          // k-steps of a slab; 16-k blocks of a slab
  // KiB pieces per wave and slab.  Where those of A do not divide among the waves (REST of them are left for the last round),
  // piece i of a wave is piece i * NW + wave of the slab, and the last round's are loaded by several waves: the same bytes to
  // the same place, so that every wave counts the same loads (160 rows: 56 pieces a slab for 52, 224 rows: 64 for 60; what the
  // four cost has not been timed apart).
  constexpr int A_ALL = BM * PK / 512, AP = (A_ALL + NW - 1) / NW, WP = BN * PK / 512 / NW, LPS = AP + WP;
  constexpr int REST = A_ALL % NW;
  static_assert(A_ALL * 512 == BM * PK && WP * NW * 512 == BN * PK, "slab must divide among the waves");
  static_assert(BM % 32 == 0, "whole blocks of A");
  // Rings of one depth are one ring of [A slab | W slab], with one offset a stage (two rings: 128x256 tiles 0.6 % slower,
  // 128x128 0.3 %); else they follow one another.
  constexpr int A_HALVES = BM * PK, W_HALVES = BN * PK, A_STAGE = A_HALVES + (SW == S ? W_HALVES : 0);
  constexpr int W_STAGE = SW == S ? A_STAGE : W_HALVES, W0_HALVES = SW == S ? A_HALVES : S * A_HALVES;
  static_assert(SW == S || SW == S + 1, "the counts of loads in flight below");
  static_assert(!SPREAD || (SW == S + 1 && !DEEP && !LO8), "as counted below");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  f16* lds = (f16*)smem;                               // [S][A slab | W slab], or [S][A slab], [SW][W slab]

  // XCD-aware tile order: consecutive workgroup ids land on different XCDs, so give each XCD a contiguous run of
  // tiles, walked in groups of GM row-tiles that share the same weight columns (4 and 8 measure alike for the small
  // tiles and for those of 224 rows, 26 products within +-1.2 % and one 2.4 % better with 8; the 256-row tile is 4 % slower with 8
  // at 18560 rows, where the L2 then holds too few weight columns).
  if constexpr (paired<Epi>()) {
    if (blockIdx.x >= epi_in.split) {
      A = epi_in.A, lda = epi_in.lda, Wp = epi_in.Wp, M = epi_in.M, K = Kw = epi_in.K, tiles_m = epi_in.tiles_m, tiles_n = epi_in.tiles_n;
      epi_in.second = true;
    }
  }
  const int nblk = tiles_m * tiles_n;
  int per_xcd = gridDim.x >> 3;
  int pid = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if constexpr (paired<Epi>()) {
    per_xcd = (epi_in.second ? gridDim.x - epi_in.split : epi_in.split) >> 3;
    pid = (blockIdx.x & 7) * per_xcd + ((epi_in.second ? blockIdx.x - epi_in.split : blockIdx.x) >> 3);
  }
  int tm, tn, kz = 0;
  if constexpr (sliced<Epi>()) {
    kz = pid / nblk;
    if (kz >= slices_of_launch(epi_in)) return;
    pid -= kz * nblk;
  } else if (pid >= nblk) {
    return;
  }
  if constexpr (SPLITK) {                              // consecutive workgroups of an XCD share a K slice (the A slabs)
    tm = 0;
    tn = pid % tiles_n;
    kz = pid / tiles_n;
  } else {
    constexpr int GM = BM >= 256 ? 4 : 8;
    const int per_group = GM * tiles_n;
    const int grp = pid / per_group;
    const int first_m = grp * GM;
    const int gm = min(tiles_m - first_m, GM);
    const int in_grp = pid - grp * per_group;
    tm = first_m + in_grp % gm;
    tn = in_grp / gm;
  }
  const int m0 = tm * BM, n0 = tn * BN;
  Epi epi = epi_in;

  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const int KB16 = Kw >> 4;
  int KT = K / PK, KTw = Kw / PK;                      // slabs; of which the first KTw are high terms
  size_t kb0 = 0;                                      // first 16-k block of this workgroup's K range
  if constexpr (SPLITK) {
    const int u0 = (int)((long long)kz * KTw / tiles_m), u1 = (int)((long long)(kz + 1) * KTw / tiles_m);
    kb0 = (size_t)u0 * KS16;
    KTw = u1 - u0;
    KT = K > Kw ? 2 * KTw : KTw;                       // the low-term slabs of the slice follow its high-term slabs
    epi.part += (size_t)kz * epi.plane_rows * epi.N;
  }
  if constexpr (sliced<Epi>()) {
    const int u0 = (int)((long long)kz * KTw / slices_of_launch(epi)), u1 = (int)((long long)(kz + 1) * KTw / slices_of_launch(epi));
    kb0 = (size_t)u0 * KS16;
    KT = KTw = u1 - u0;
    epi.slice(kz);
  }

  const unsigned lane16 = (unsigned)lane * 16u;        // lane offset in an operand in fragment order
  const f16* a_base = A + (size_t)m0 * lda + kb0 * 512;
  const f16* a_lo_base = SPLITK && epi_a_lo(epi) ? epi_a_lo(epi) + kb0 * 512 : a_base;
  const f16* w_base = Wp + ((size_t)(n0 / 32) * KB16 + kb0) * 512;
  const f16* w8_base = LO8 ? W8 + (size_t)(n0 / 32) * KB16 * 256 : w_base;
  const unsigned a_block = 64u * (unsigned)lda;        // bytes of a block of 32 rows of A
  const int a_last = (M - 1 - m0) >> 5;                // last block there is (a launch's rows are allocated in whole blocks)
  // The lanes of rows past M ask for what others do, so that a last tile of few rows has few lines of A to wait for: its workgroup
  // runs ahead of the others of the same columns and XCD, which find the weights in the L2.  us with whole blocks / this, cold
  // weights, N 4096: 580 rows K 4096 41.2 / 38.7, K 11008 94 / 88, with low terms 137 / 127; 1160 rows 61 / 57.6, 138 / 133.
  const unsigned lane_last = (unsigned)(min(lane & 31, (M - 1 - m0) & 31) + (lane & 32)) * 16u;      // in block a_last
  // Unpacked W: a wave's pieces of a KiB are 8 rows of 64 k, or 1024 / (2 BN) rows of the contraction, 16 bytes a lane.  The chunks
  // of 16 bytes of a row are swizzled so that the reads of the LDS have no more bank conflicts than bytes: by the row
  // (reads of 16 rows), and in pairs (32 bytes) by the rows of the contraction that a transposed read takes together.
  constexpr int RAW = raw_w<Epi>();
  static_assert(!RAW || (!LO8 && !AGPR && !SPLITK), "products left to the compiler, one pass");
  [[maybe_unused]] unsigned raw_off[RAW ? WP : 1], raw_row[RAW == 2 ? WP : 1];
  [[maybe_unused]] const int raw_n0 = RAW == 1 ? min(n0, raw_rows_of(epi_in) - 1) : 0;      // (a tile may be all padding)
  if constexpr (RAW == 1) {
#pragma unroll
    for (int i = 0; i < WP; ++i) {
      const int row = (wave * WP + i) * 8 + (lane >> 3);
      raw_off[i] = (unsigned)min(row, epi.raw_rows - 1 - raw_n0) * 2u * (unsigned)epi.raw_ld + (unsigned)((lane & 7) ^ ((row >> 1) & 7)) * 16u;
    }
  }
  constexpr int RPP = RAW == 2 ? 512 / BN : 1;         // rows of a piece
  if constexpr (RAW == 2) {
#pragma unroll
    for (int i = 0; i < WP; ++i) {
      const int row = (wave * WP + i) * RPP + lane / (64 / RPP), f = (row & 3) | ((row >> 3) & 1) << 2;
      raw_row[i] = row;
      raw_off[i] = (unsigned)min(n0 / 8 + ((lane % (64 / RPP)) ^ (f << 1)), epi.raw_cols / 8 - 1) * 16u;
    }
  }
  const int a_back = REST ? wave - wave % (REST ? REST : 1) : 0;     // pieces a wave's last one is moved back by
  auto issue_one = [&](int kt, auto I) VLA_INLINE {    // piece I of this wave's share of slab kt (clamped), A first
    constexpr int i = decltype(I)::value;
    const int ks = min(kt, KT - 1), kw = ks >= KTw ? ks - KTw : ks;
    if constexpr (i < AP) {                            // piece j of the slab: block row j / KS16 (clamped), 16-k block j % KS16
      const int j = REST ? i * NW + wave - (i == AP - 1 ? a_back : 0) : wave * AP + i;
      const unsigned blk = (unsigned)min(j / KS16, a_last) * a_block + (unsigned)(j % KS16) * 1024u;
      const bool low = SPLITK && ks >= KTw;
      load_to_lds_16(low ? a_lo_base : a_base, j / KS16 < a_last ? lane16 : j / KS16 == a_last ? lane_last : 0u, blk + 1024u * KS16 * (unsigned)(SPLITK ? kw : ks), lds + (kt % S) * A_STAGE + j * 512);
    } else {
      const int j = wave * WP + i - AP;                // piece of the slab: block row j / KS16, 16-k block j % KS16
      if constexpr (RAW == 1) {
        load_to_lds_16((const f16*)Wp + (size_t)raw_n0 * epi.raw_ld + kb0 * 16, raw_off[i - AP], 128u * (unsigned)kw, lds + W0_HALVES + (kt % SW) * W_STAGE + j * 512);
        return;
      }
      if constexpr (RAW == 2) {
        const size_t k0 = kb0 * 16 + (size_t)kw * PK;
        const unsigned row = min(raw_row[i - AP], (unsigned)(epi.raw_rows - 1 - (int)k0));
        load_to_lds_16((const f16*)Wp + k0 * epi.raw_ld, raw_off[i - AP] + row * 2u * (unsigned)epi.raw_ld, 0u, lds + W0_HALVES + (kt % SW) * W_STAGE + j * 512);
        return;
      }
      const bool low = LO8 && ks >= KTw;
      const unsigned blk = (unsigned)(j / KS16 * KB16) * (low ? 512u : 1024u) + (unsigned)(j % KS16) * 1024u;
      load_to_lds_16(low ? w8_base : w_base, lane16, blk + 1024u * KS16 * (unsigned)kw, lds + W0_HALVES + (kt % SW) * W_STAGE + j * 512);
    }
  };

  auto issue_next = [&](int kt, auto I) VLA_INLINE {   // piece I of what takes the stages of slab kt
    issue_one(decltype(I)::value < AP ? kt + S : kt + SW, I);
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // LDS byte addresses of this lane's fragments inside stage 0.  A lane of a fragment is (row l % 16, k group
  // l / 16 of 8 k); in fragment order its 16 bytes are at 16 * (row & 31) + 512 * (group & 1) of 16-k block group / 2.
  const unsigned lds0 = (unsigned)(size_t)((__attribute__((address_space(3))) unsigned char*)smem);
  const int fgrp = lane >> 4;
  const unsigned in_block = (unsigned)(fgrp >> 1) * 1024u + (unsigned)(fgrp & 1) * 512u + (unsigned)(lane & 15) * 16u;
  // first fragment of A of this wave, and what is added for every second one: of wave tiles of an odd number of fragments the
  // second begins in the middle of a block
  const int a_frag = wm * MT;
  const unsigned a_even = lds0 + (unsigned)(a_frag >> 1) * (KS16 * 1024u) + (unsigned)(a_frag & 1) * 256u + in_block;
  const unsigned a_odd = MT % 2 ? a_even + (a_frag & 1 ? KS16 * 1024u - 512u : 0u) : a_even;
  const unsigned w_b = lds0 + 2u * (unsigned)(W0_HALVES + wn * (WN / 32) * KS16 * 512) + in_block;

  constexpr int NBUF = DEEP ? 2 * KS : 2;              // register buffers, a k-step each
  f16x8 af[NBUF][MT], bf[NBUF][NT];
  [[maybe_unused]] u32x2 bt[RAW == 2 ? NBUF : 1][NT][2];     // transposed reads
  [[maybe_unused]] f16x8 bc[RAW ? NT : 1];                   // of the k-step, re-encoded
  [[maybe_unused]] unsigned w_raw[RAW == 2 ? NT : 2];
  if constexpr (RAW == 1) {
#pragma unroll
    for (int ss = 0; ss < 2; ++ss)
      w_raw[ss] = lds0 + 2u * (unsigned)W0_HALVES + (unsigned)(wn * WN + (lane & 15)) * 128u + (unsigned)((4 * ss + fgrp) ^ ((lane & 15) >> 1)) * 16u;
  }
  if constexpr (RAW == 2) {
    const unsigned row = (unsigned)(8 * fgrp + ((lane & 15) >> 2)), f = ((lane >> 2) & 3) | (fgrp & 1) << 2;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      w_raw[nt] = lds0 + 2u * (unsigned)W0_HALVES + row * (2u * BN) + ((unsigned)(wn * NT + nt) ^ f) * 32u + (unsigned)(lane & 3) * 8u;
  }
  constexpr int R = MT + NT, MF = MT * NT;             // reads and products of a k-step
  struct Stages { unsigned a, b; };                    // byte offsets of a slab's stages
  auto stages_of = [&](int kt) VLA_INLINE {
    return Stages{(unsigned)(kt % S) * (2u * A_STAGE), (unsigned)(kt % SW) * (2u * W_STAGE)};
  };
  // fragment reads of k-step ss of the slab in stages so (block j of an operand in fragment order: 32 rows hold two
  // fragments)
  auto read_a = [&](Stages so, f16x8& dst, auto SS, auto J) VLA_INLINE {
    constexpr int ss = decltype(SS)::value, j = decltype(J)::value;
    read_frag_asm<(j / 2 * KS16 + 2 * ss) * 1024 + (j & 1) * 256>(dst, (j & 1 ? a_odd : a_even) + so.a);
  };
  auto read_b = [&](Stages so, f16x8& dst, auto SS, auto J) VLA_INLINE {
    constexpr int ss = decltype(SS)::value, j = decltype(J)::value;
    if constexpr (RAW == 1) read_frag_asm<j * 2048>(dst, w_raw[ss] + so.b);
    else read_frag_asm<(j / 2 * KS16 + 2 * ss) * 1024 + (j & 1) * 256>(dst, w_b + so.b);
  };
  auto read_one = [&](Stages so, int f, auto SS, auto I) VLA_INLINE {   // I-th fragment read of a k-step
    constexpr int x = decltype(I)::value;
    if constexpr (x < MT) read_a(so, af[f][x], SS, I);
    else if constexpr (RAW == 2) {
      constexpr int off = 32 * decltype(SS)::value * 2 * BN;
      read_transposed_asm<off>(bt[f][x - MT][0], w_raw[x - MT] + so.b);
      read_transposed_asm<off + 4 * 2 * BN>(bt[f][x - MT][1], w_raw[x - MT] + so.b);
    } else read_b(so, bf[f][x - MT], SS, std::integral_constant<int, x - MT>{});
  };
  auto arrived = [&](int f) VLA_INLINE {
    wait_lds();
#pragma unroll
    for (int i = 0; i < MT; ++i) hold(af[f][i]);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if constexpr (RAW == 2) {
        hold(bt[f][j][0]);
        hold(bt[f][j][1]);
      } else {
        hold(bf[f][j]);
      }
    }
  };
  // One k-step of slab kt: the MFMAs, and between them fragment reads (in the first three quarters, so that they have
  // landed at the end) and the loads that take slab kt's stages (A of slab kt + S, W of slab kt + SW).
  // Read ahead by a k-step: the k-steps alternate between two buffers, P is the slab's first one.  The reads of the last
  // k-step belong to slab kt + 1, which must have landed, and slab kt is in everybody's registers: its stage takes the loads.
  // DEEP, read ahead by a slab: P is the half of the buffers slab kt is in, and all of this holds from its first k-step on.
  auto step = [&](int kt, auto P, auto SS) VLA_INLINE {
    constexpr int p = decltype(P)::value, ss = decltype(SS)::value;
    constexpr bool last = ss == KS - 1, next = DEEP || last;        // next: the reads are of slab kt + 1
    constexpr int f = DEEP ? p * KS + ss : (p + ss) & 1, g = DEEP ? (p ^ 1) * KS + ss : f ^ 1;
    constexpr int n_rd = MF * 3 / 4 > 0 ? MF * 3 / 4 : 1;
    if constexpr (DEEP ? ss == 0 : last) {
      wait_vmcnt<(S - 2) * LPS + (SW - S) * WP>();
      __builtin_amdgcn_s_barrier();
    }
    const Stages so = stages_of(kt + (next ? 1 : 0));
    static_for<MF>([&](auto I) VLA_INLINE {
      constexpr int i = decltype(I)::value, mt = i / NT, nt = i % NT;
      if constexpr (RAW && mt == 0) {
        if constexpr (RAW == 2) bc[nt] = encode_weights(u32x4{bt[f][nt][0][0], bt[f][nt][0][1], bt[f][nt][1][0], bt[f][nt][1][1]});
        else bc[nt] = encode_weights(__builtin_bit_cast(u32x4, bf[f][nt]));
      }
      if constexpr (RAW != 0) acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(af[f][mt], bc[nt], acc[mt][nt], 0, 0, 0);
      else if constexpr (LO8 || AGPR) mfma_in_place<AGPR>(acc[mt][nt], af[f][mt], bf[f][nt]);
      else acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(af[f][mt], bf[f][nt], acc[mt][nt], 0, 0, 0);
      constexpr int r0 = i < n_rd ? i * R / n_rd : R, r1 = i < n_rd ? (i + 1) * R / n_rd : R;
      static_for<r1 - r0>([&](auto J) VLA_INLINE {
        read_one(so, g, std::integral_constant<int, DEEP ? ss : (last ? 0 : ss + 1)>{}, std::integral_constant<int, r0 + decltype(J)::value>{});
      });
      if constexpr (SPREAD) {                          // last k-step: A; the next one: W
        constexpr int n = last ? AP : WP, l0 = i * n / MF, l1 = (i + 1) * n / MF;
        static_for<l1 - l0>([&](auto J) VLA_INLINE {
          issue_next(last ? kt : kt - 1, std::integral_constant<int, (last ? 0 : AP) + l0 + decltype(J)::value>{});
        });
      } else if constexpr (next) {
        constexpr int at = DEEP ? ss * MF + i : i, of = DEEP ? KS * MF : MF;
        constexpr int l0 = at * LPS / of, l1 = (at + 1) * LPS / of;
        static_for<l1 - l0>([&](auto J) VLA_INLINE { issue_next(kt, std::integral_constant<int, l0 + decltype(J)::value>{}); });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (!DEEP) arrived(g);
    else if constexpr (last) static_for<KS>([&](auto J) VLA_INLINE { arrived((p ^ 1) * KS + decltype(J)::value); });
  };
  auto slab = [&](int kt, auto P) VLA_INLINE {
    static_for<KS>([&](auto SS) VLA_INLINE { step(kt, P, SS); });
  };
  constexpr std::integral_constant<int, 0> c0{};
  constexpr std::integral_constant<int, 1> c1{};
  constexpr std::integral_constant<int, DEEP ? 1 : 0> cn{};       // P of an odd slab
  static_for<S>([&](auto I) VLA_INLINE { static_for<LPS>([&](auto J) VLA_INLINE { issue_one(decltype(I)::value, J); }); });
  if constexpr (!SPREAD)
    static_for<SW - S>([&](auto I) VLA_INLINE {
      static_for<WP>([&](auto J) VLA_INLINE { issue_one(S + decltype(I)::value, std::integral_constant<int, AP + decltype(J)::value>{}); });
    });
  wait_vmcnt<(S - 1) * LPS + (SPREAD ? 0 : (SW - S) * WP)>();
  __builtin_amdgcn_s_barrier();
  static_for<DEEP ? KS : 1>([&](auto SS) VLA_INLINE {
    static_for<R>([&](auto I) VLA_INLINE { read_one(stages_of(0), decltype(SS)::value, SS, I); });
  });
  static_for<DEEP ? KS : 1>([&](auto SS) VLA_INLINE { arrived(decltype(SS)::value); });
  const int KTh = LO8 ? KTw : KT;
  int kt = 0;
  if constexpr (LO8 || AGPR) settle<AGPR>(acc);        // the zeros are written
  if constexpr (LO8) {
    if constexpr (DEEP) {
      for (; kt + 1 < KTh; kt += 2) {
        slab(kt, c0);
        slab(kt + 1, cn);
      }
      if (kt < KTh) slab(kt++, c0);
    } else {
      for (; kt < KTh; ++kt) slab(kt, c0);
    }
    settle<AGPR>(acc);
    // Fragments of one slab, k-steps 0 and 1: variables of their own, read afresh, since the product wants the two in
    // adjacent registers and the loop above must not be bound by that.  Reads are issued in the order: first-half A
    // fragments, B fragments column by column, second-half A fragments.
    constexpr int H = MT / 2;
    f16x8 al[2][MT], bl[2][NT];
    auto refill_a = [&](Stages so, auto J) VLA_INLINE {
      read_a(so, al[0][decltype(J)::value], c0, J);
      read_a(so, al[1][decltype(J)::value], c1, J);
    };
    auto refill_b = [&](Stages so, auto J) VLA_INLINE {
      read_b(so, bl[0][decltype(J)::value], c0, J);
      read_b(so, bl[1][decltype(J)::value], c1, J);
    };
    auto hold_a = [&](int i) VLA_INLINE {
      hold(al[0][i]);
      hold(al[1][i]);
    };
    auto product = [&](auto MI, auto NI) VLA_INLINE {
      constexpr int mt = decltype(MI)::value, nt = decltype(NI)::value;
      acc[mt][nt] = mfma_lo8(al[0][mt], al[1][mt], bl[0][nt], bl[1][nt], acc[mt][nt]);
    };
    auto low_slab = [&](int t) VLA_INLINE {
      static_for<NT>([&](auto NI) VLA_INLINE {         // rows of the first half
        constexpr int nt = decltype(NI)::value;
        wait_lds<2 * (NT - 1 - nt) + 2 * (MT - H)>();
        if constexpr (nt == 0) {
#pragma unroll
          for (int i = 0; i < H; ++i) hold_a(i);
        }
        hold(bl[0][nt]);
        hold(bl[1][nt]);
        static_for<H>([&](auto MI) VLA_INLINE { product(MI, NI); });
        __builtin_amdgcn_sched_barrier(0);
      });
      wait_lds();
#pragma unroll
      for (int i = H; i < MT; ++i) hold_a(i);
      wait_vmcnt<(S - 2) * LPS + (SW - S) * WP>();                     // slab t + 1 has landed, slab t is in everybody's registers
      __builtin_amdgcn_s_barrier();
      const Stages so = stages_of(t + 1);
      static_for<NT>([&](auto NI) VLA_INLINE {         // rows of the second half
        constexpr int nt = decltype(NI)::value;
        static_for<MT - H>([&](auto MI) VLA_INLINE {
          product(std::integral_constant<int, H + decltype(MI)::value>{}, NI);
          if constexpr (decltype(MI)::value == 0) {
            if constexpr (nt == 0) static_for<H>([&](auto J) VLA_INLINE { refill_a(so, J); });
            else refill_b(so, std::integral_constant<int, nt - 1>{});
          }
        });
        constexpr int l0 = nt * LPS / NT, l1 = (nt + 1) * LPS / NT;
        static_for<l1 - l0>([&](auto J) VLA_INLINE { issue_next(t, std::integral_constant<int, l0 + decltype(J)::value>{}); });
        __builtin_amdgcn_sched_barrier(0);
      });
      refill_b(so, std::integral_constant<int, NT - 1>{});
      static_for<MT - H>([&](auto J) VLA_INLINE { refill_a(so, std::integral_constant<int, H + decltype(J)::value>{}); });
    };
    const Stages so0 = stages_of(kt);
    static_for<H>([&](auto J) VLA_INLINE { refill_a(so0, J); });
    static_for<NT>([&](auto J) VLA_INLINE { refill_b(so0, J); });
    static_for<MT - H>([&](auto J) VLA_INLINE { refill_a(so0, std::integral_constant<int, H + decltype(J)::value>{}); });
    for (; kt < KT; ++kt) low_slab(kt);
    wait_lds();                                        // the last slab's refills
#pragma unroll
    for (int i = 0; i < MT; ++i) hold_a(i);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      hold(bl[0][j]);
      hold(bl[1][j]);
    }
  } else {
    // The tile of the fewest rows, whose sums nothing averages, adds up sums of 512 k instead of one chain: an eighth of the
    // magnitude at most of its roundings.  (The launch waits for HBM; the additions cost nothing that could be measured.)
    constexpr bool kParts = RAW == 1 && DEEP;
    f32x4 sum[kParts ? MT : 1][kParts ? NT : 1] = {};
    for (; kt + 1 < KTh; kt += 2) {
      slab(kt, c0);
      slab(kt + 1, cn);
      if constexpr (kParts) {
        if (kt % 8 == 6) {
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) sum[i][j] += acc[i][j], acc[i][j] = f32x4{};
        }
      }
    }
    if (kt < KTh) slab(kt, c0);
    if constexpr (kParts) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] += sum[i][j];
    }
  }
  if constexpr (AGPR) settle<AGPR>(acc);
  wait_vmcnt<0>();                                     // the clamped tail loads still target this workgroup's LDS
  __syncthreads();                                     // every wave is done with the slabs: LDS becomes epilogue staging

  if constexpr (requires { epi.begin(lane); }) epi.begin(lane);
  store_tile<MT, NT, WGN>(acc, epi, smem, wave, wn, lane, m0 + wm * WM, n0, M);
}

template <int WGM, int WGN, int WM, int WN, int S, int SW, int OCC, bool DEEP, bool SPREAD, bool LO8, bool SPLITK, class Epi>
static void launch_tiles(const f16* A, int lda, const f16* Wp, const f16* W8, int M, int K, int Kw, int tiles_m,
                         int tiles_n, const Epi& epi, hipStream_t st) {
  int wgs = tiles_m * tiles_n;
  if constexpr (paired<Epi>()) wgs = (int)epi.split + epi.tiles_m * epi.tiles_n * epi.head.slices;
  else if constexpr (sliced<Epi>()) wgs *= epi.slices;
  const int grid = (wgs + 7) / 8 * 8;
  constexpr size_t slabs = ((size_t)S * WGM * WM + (size_t)SW * WGN * WN) * PK * sizeof(f16);
  constexpr bool pair = WN < Epi::kSpan;
  constexpr size_t stage = (size_t)WGM * WGN / (pair ? 2 : 1) * 32 * ((pair ? 2 : 1) * WN + 4) * sizeof(float);
  constexpr size_t smem = slabs > stage ? slabs : stage;
  auto kern = gemm_f16_kernel<WGM, WGN, WM, WN, S, SW, OCC, DEEP, SPREAD, Epi, LO8, SPLITK>;
  static bool attr_set = false;
  if (!attr_set) {
    (void)hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    attr_set = true;
  }
  hipLaunchKernelGGL(kern, dim3(grid), dim3(WGM * WGN * 64), smem, st, A, lda, Wp, W8, M, K, Kw, tiles_m, tiles_n, epi);
}
template <int WGM, int WGN, int WM, int WN, int S, int SW, int OCC, bool DEEP, bool SPREAD, bool LO8, class Epi>
static void launch(const GemmF16& g, const Epi& epi, hipStream_t st) {
  launch_tiles<WGM, WGN, WM, WN, S, SW, OCC, DEEP, SPREAD, LO8, false>(g.A, g.lda, g.Wp, g.W8, g.M, g.K, g.Kw,
                                                               (g.M + WGM * WM - 1) / (WGM * WM), g.N / (WGN * WN), epi, st);
}

// The forms a launch can take (gemm_f16_variant picks one, see there).
constexpr int kFewHeights = 7;                            // gemm_few_kernel's tiles: 32, 48, ... 128 rows
enum Variant {
  V_FEW, V_FEW_AHEAD = V_FEW + kFewHeights,              // (the first of each; ahead: with workgroups that read the weights ahead)
  V_64x128_8W = V_FEW_AHEAD + kFewHeights, V_64x128, V_64x128_ROUNDS, V_128x128, V_64x256, V_128x256, V_160x256, V_192x256,
  V_224x256, V_256x256, V_256x256_SPREAD, V_COUNT
};

}  // namespace vla
