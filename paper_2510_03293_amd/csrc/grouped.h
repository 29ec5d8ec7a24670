// A tile of a product whose rows fall into groups: BM token rows times BN weight rows,
// contracted over their common axis (both operands row-major along it), fp32 accumulation.
//
// Both operands travel memory -> LDS without passing through registers, in steps of 128
// bytes per row (64 bf16 or 32 fp32 values); ST steps share a ring, of which ST - 1 are in
// flight while one is multiplied, with one barrier per step.  A wavefront's load instruction
// takes 8 rows x 128 contiguous bytes.  Where the 16-byte piece c of row r lies in its LDS
// row is c ^ (r / 2 % 8): the 16 rows x 4 pieces that a wavefront reads as a matrix operand
// (lane l: row l % 16, piece l / 16) then spread over all banks.
//
// The weights are the A operand and the tokens the B operand, so that a lane's accumulator
// registers hold four neighbouring outputs of one token (register i of lane l: output row
// 4 (l / 16) + i, token l % 16 of the 16 x 16 block).
#pragma once

#include "laser_internal.h"

namespace laser {

typedef __attribute__((ext_vector_type(8))) __bf16 mma_bf16x8;
typedef __attribute__((ext_vector_type(4))) float mma_f32x4;
typedef unsigned int mma_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int mma_u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) unsigned char* lds_bytes;
typedef __attribute__((address_space(3))) mma_u32x4* lds_piece;

constexpr int kStepBytes = 128;

// What lanes load whose piece lies behind the end of the rows (both operands then hold zeros).
static __device__ __align__(16) const unsigned int zero_piece[4] = {0, 0, 0, 0};

// 64 x 16 bytes, lane l's to LDS byte `lds` + 16 l.  Only vmcnt says when they are there.
__device__ __forceinline__ void load_to_lds(const unsigned char* from, unsigned lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)(size_t)lds, 16, 0, 0);
}

__device__ __forceinline__ mma_u32x4 read_lds(unsigned at) { return *(lds_piece)(size_t)at; }

// One step of the contraction of a 16 x 16 block: a lane's 16 bytes are 8 bf16 slots of one
// instruction or 4 fp32 slots of four; which slot is which column is the same for a and b.
template <bool F32>
__device__ __forceinline__ mma_f32x4 multiply(mma_u32x4 a, mma_u32x4 b, mma_f32x4 c) {
  if constexpr (F32) {
    const mma_f32x4 x = __builtin_bit_cast(mma_f32x4, a), y = __builtin_bit_cast(mma_f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
    return c;
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mma_bf16x8, a), __builtin_bit_cast(mma_bf16x8, b),
                                                   c, 0, 0, 0);
  }
}

__device__ __forceinline__ unsigned bf16_bits(float x) {  // round to nearest even, NaN stays NaN
  return __builtin_bit_cast(unsigned short, (__bf16)x);
}
__device__ __forceinline__ float bf16_value(unsigned bits) { return __builtin_bit_cast(float, bits << 16); }

// Four neighbouring values of an output row, rounded to the output's type.
template <bool F32>
__device__ __forceinline__ void store4(void* row, size_t at, mma_f32x4 v) {
  if constexpr (F32) {
    *(reinterpret_cast<mma_f32x4*>(static_cast<float*>(row) + at)) = v;
  } else {
    mma_u32x2 b;
    b[0] = bf16_bits(v[0]) | bf16_bits(v[1]) << 16;
    b[1] = bf16_bits(v[2]) | bf16_bits(v[3]) << 16;
    *(reinterpret_cast<mma_u32x2*>(static_cast<unsigned short*>(row) + at)) = b;
  }
}
template <bool F32>
__device__ __forceinline__ mma_f32x4 load4(const void* row, size_t at) {
  if constexpr (F32) {
    return *(reinterpret_cast<const mma_f32x4*>(static_cast<const float*>(row) + at));
  } else {
    const mma_u32x2 b = *(reinterpret_cast<const mma_u32x2*>(static_cast<const unsigned short*>(row) + at));
    return mma_f32x4{bf16_value(b[0] & 0xffffu), bf16_value(b[0] >> 16), bf16_value(b[1] & 0xffffu),
                     bf16_value(b[1] >> 16)};
  }
}

// WM x WN wavefronts, each with (BM / WM) x (BN / WN) of the tile.
template <bool F32, int BM_, int BN_, int WM_, int WN_, int ST_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, ST = ST_;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int MB = BM / WM / 16, NB = BN / WN / 16;  // 16 x 16 blocks of a wavefront
  static constexpr int kLoads = (BM + BN) / 8 / kWaves;       // load instructions of a wavefront per step
  static constexpr int kStage = (BM + BN) * kStepBytes;
  static constexpr int kLdsBytes = ST * kStage;
  static_assert(kLoads * 8 * kWaves == BM + BN && kWaves % 2 == 0 && ST >= 2, "whole load instructions per wavefront");
  static_assert((ST - 2) * kLoads < 64, "vmcnt counts to 63");

  // Tile row that load i of this wavefront brings for this lane (tokens 0 .. BM - 1, then
  // weights), and the piece of that row: the same for all i, as kWaves is even.
  __device__ static int row(int wave, int lane, int i) { return (wave + i * kWaves) * 8 + (lane >> 3); }
  __device__ static int piece(int wave, int lane) { return (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4)); }

  // from[i]: where load i of this lane begins (row start + 16 * piece).  `bytes`: length of
  // the rows, a multiple of 16.  Ends with every wavefront through with its reads of LDS.
  __device__ static void run(const unsigned char* (&from)[kLoads], int bytes, unsigned lds, int wave, int lane,
                             mma_f32x4 (&acc)[NB][MB]) {
    const int steps = (bytes + kStepBytes - 1) / kStepBytes;
    const bool in_last = piece(wave, lane) * 16 < bytes - (steps - 1) * kStepBytes;
    const unsigned put = __builtin_amdgcn_readfirstlane(lds + wave * 8 * kStepBytes);
    auto issue = [&](int step, int slot) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const unsigned char* p = from[i];
        from[i] += kStepBytes;
        if (step == steps - 1) p = in_last ? p : reinterpret_cast<const unsigned char*>(zero_piece);
        load_to_lds(p, put + slot * kStage + i * kWaves * 8 * kStepBytes);
      }
    };
    const int wm = wave % WM, wn = wave / WM;
    // (piece s * 4 + lane / 16 of row lane % 16, s = 0, 1)
    const unsigned get = (lane & 15) * kStepBytes + ((lane >> 4) ^ ((lane & 15) >> 1)) * 16;
    const unsigned get_t = lds + wm * (BM / WM) * kStepBytes + get;
    const unsigned get_w = lds + (BM + wn * (BN / WN)) * kStepBytes + get;

#pragma unroll
    for (int s = 0; s < ST - 1; ++s)
      if (s < steps) issue(s, s);
    int slot = 0;
    for (int step = 0; step < steps; ++step) {
      // this wavefront's loads of the step are there, and its reads of the step before
      // are done, for which the slot that is loaded next was waiting
      if (step + ST - 1 <= steps)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((ST - 2) * kLoads) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (step + ST - 1 < steps) issue(step + ST - 1, slot == 0 ? ST - 1 : slot - 1);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        mma_u32x4 w[NB], t[MB];
#pragma unroll
        for (int n = 0; n < NB; ++n) w[n] = read_lds((get_w + slot * kStage + n * 16 * kStepBytes) ^ (s * 64));
#pragma unroll
        for (int m = 0; m < MB; ++m) t[m] = read_lds((get_t + slot * kStage + m * 16 * kStepBytes) ^ (s * 64));
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int m = 0; m < MB; ++m) acc[n][m] = multiply<F32>(w[n], t[m], acc[n][m]);
      }
      slot = slot == ST - 1 ? 0 : slot + 1;
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
};

// Number `v` of `total` workgroups that the eight XCDs take in turn -> the tile it computes,
// so that an XCD has one contiguous run of tiles (they share rows through its L2).
__device__ __forceinline__ int xcd_run(int v, int total) {
  const int q = total >> 3, r = total & 7, x = v & 7;
  return x * q + min(x, r) + (v >> 3);
}

}  // namespace laser
