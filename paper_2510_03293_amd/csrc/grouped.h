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
typedef __attribute__((address_space(3))) mma_f32x4* lds_f32x4;
typedef __attribute__((address_space(3))) mma_u32x2* lds_u32x2;

constexpr int kStepBytes = 128;
struct true_c {
  static constexpr bool value = true;
  __device__ constexpr operator bool() const { return true; }
};
struct false_c {
  static constexpr bool value = false;
  __device__ constexpr operator bool() const { return false; }
};

// What lanes load whose piece lies behind the end of the rows (both operands then hold zeros).
static __device__ __align__(16) const unsigned int zero_piece[4] = {0, 0, 0, 0};

// 64 x 16 bytes, lane l's to LDS byte `lds` + 16 l.  Only vmcnt says when they are there.
// (ONCE: past the caches)
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const unsigned char* from, unsigned lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)(size_t)lds, 16, 0, ONCE ? 2 : 0);
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

// The products of a ring's step: COUNT pieces of the axis of N x M blocks, added to acc.  fp32: a step's products are
// summed by themselves (`own`), and that joins acc a step later, when it is there; an eighth of the
// roundings are then made at the size of the sum (333 tokens, 516 x 212: off by 3e-7, 6e-7 in one
// chain).  last() adds the last step's.
template <bool F32, int COUNT, int N, int M>
struct StepProducts {
  mma_f32x4 own[F32 ? N : 1][F32 ? M : 1];
  __device__ StepProducts() {
#pragma unroll
    for (int n = 0; n < (F32 ? N : 1); ++n)
#pragma unroll
      for (int m = 0; m < (F32 ? M : 1); ++m) own[n][m] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  __device__ void add(const mma_u32x4 (&w)[COUNT][N], const mma_u32x4 (&t)[COUNT][M], int blocks, mma_f32x4 (&acc)[N][M]) {
    if constexpr (F32) {
#pragma unroll
      for (int m = 0; m < M; ++m) {
        if (m >= blocks) continue;
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n][m] += own[n][m];
#pragma unroll
        for (int s = 0; s < COUNT; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n)
              own[n][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  __builtin_bit_cast(mma_f32x4, w[s][n])[i], __builtin_bit_cast(mma_f32x4, t[s][m])[i],
                  s == 0 && i == 0 ? mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f} : own[n][m], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int s = 0; s < COUNT; ++s)
#pragma unroll
        for (int m = 0; m < M; ++m)
          if (m < blocks)
#pragma unroll
            for (int n = 0; n < N; ++n) acc[n][m] = multiply<false>(w[s][n], t[s][m], acc[n][m]);
    }
  }
  __device__ void last(mma_f32x4 (&acc)[N][M]) const {
    if constexpr (F32) {
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n][m] += own[n][m];
    }
  }
};

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

// WM x WN wavefronts, each with (BM / WM) x (BN / WN) of the tile.  ONCE: the operand that nobody else
// reads.
enum Operand { kNeither, kTokens, kWeights };
template <bool F32, int BM_, int BN_, int WM_, int WN_, int ST_, Operand ONCE = kNeither>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, ST = ST_;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int MB = BM / WM / 16, NB = BN / WN / 16;  // 16 x 16 blocks of a wavefront
  static constexpr int kLoads = (BM + BN) / 8 / kWaves;       // load instructions of a wavefront per step
  static constexpr int kStage = (BM + BN) * kStepBytes;
  static constexpr int kLdsBytes = ST * kStage;
  static_assert(kLoads * 8 * kWaves == BM + BN && kWaves % 2 == 0 && ST >= 2, "whole load instructions per wavefront");
  static_assert((ST - 1) * kLoads < 64, "vmcnt counts to 63");

  // Tile row that load i of this wavefront brings for this lane (tokens 0 .. BM - 1, then
  // weights), and the piece of that row: the same for all i, as kWaves is even.
  __device__ static int row(int wave, int lane, int i) { return (wave + i * kWaves) * 8 + (lane >> 3); }
  __device__ static int piece(int wave, int lane) { return (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4)); }

  // The product of one tile.  from[i]: where load i of this lane begins (row start + 16 *
  // piece + kStepBytes * turn); `bytes`: length of the rows, a multiple of 16.  start() puts the
  // first steps on their way to LDS, which nobody may be reading any more; run() does the rest and
  // ends with every wavefront through with its reads of LDS.
  int steps, bytes;
  bool in_last;    // whether this lane's piece of the last step is inside the rows
  unsigned put;    // where this wavefront's loads go in slot 0
  unsigned get_t, get_w;  // this lane's operands in slot 0, first half of the step

  __device__ Tile(int bytes_, unsigned lds, int wave, int lane) : bytes(bytes_), turn(0), column(0) {
    steps = (bytes + kStepBytes - 1) / kStepBytes;
    in_last = piece(wave, lane) * 16 < bytes - (steps - 1) * kStepBytes;
    put = __builtin_amdgcn_readfirstlane(lds + wave * 8 * kStepBytes);
    const unsigned get = (lane & 15) * kStepBytes + ((lane >> 4) ^ ((lane & 15) >> 1)) * 16;
    get_t = lds + wave % WM * 16 * kStepBytes + get;
    get_w = lds + (BM + wave / WM * (BN / WN)) * kStepBytes + get;
  }

  // Which columns a tile begins with: rows whose length is a multiple of a step may be walked
  // from any step on and around (`turn`).  Rows often lie a power of two apart, and then all tiles
  // that are at the same step read from the same few memory channels.
  int turn;    // step of the rows that is loaded first
  int column;  // ... next
  __device__ void turn_to(int which) {
    turn = steps * kStepBytes == bytes ? which % steps : 0;
    column = turn;
  }
  // bytes from this step of the rows to the next one loaded
  __device__ int stride() {
    const bool around = column == steps - 1;
    column = around ? 0 : column + 1;
    return around ? kStepBytes - steps * kStepBytes : kStepBytes;
  }

  template <typename LAST>
  __device__ void load(const unsigned char* (&from)[kLoads], LAST last, unsigned slot, int i, int by) const {
    const unsigned char* p = from[i];
    from[i] += by;
    if (last) p = in_last ? p : reinterpret_cast<const unsigned char*>(zero_piece);
    // (which operand load i brings is known here where no load brings both)
    if (BM % (8 * kWaves) == 0 && ONCE == (i < BM / (8 * kWaves) ? kTokens : kWeights))
      load_to_lds<true>(p, put + slot + i * kWaves * 8 * kStepBytes);
    else
      load_to_lds<false>(p, put + slot + i * kWaves * 8 * kStepBytes);
  }
  template <typename LAST>
  __device__ void load_all(const unsigned char* (&from)[kLoads], LAST last, unsigned slot) {
    const int by = stride();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(from, last, slot, i, by);
  }
  // Blocks of 16 tokens go to the WM wavefronts of a column in turn, so that a tile with few
  // rows is work for all of them: row of token block m, and how many blocks have rows at all.
  __device__ static int block_row(int wave, int m) { return (m * WM + wave % WM) * 16; }
  __device__ static int blocks_of(int wave, int rows) { return ((rows + 15) / 16 - wave % WM + WM - 1) / WM; }

  // operand block m (or n) of half s of the step in `slot`
  __device__ mma_u32x4 token_block(unsigned slot, int s, int m) const {
    return read_lds(((get_t + slot) ^ (s * 64)) + m * WM * 16 * kStepBytes);
  }
  __device__ mma_u32x4 weight_block(unsigned slot, int s, int n) const {
    return read_lds(((get_w + slot) ^ (s * 64)) + n * 16 * kStepBytes);
  }

  __device__ void start(const unsigned char* (&from)[kLoads]) {
#pragma unroll
    for (int s = 0; s < ST; ++s)
      if (s < steps) load_all(from, s == steps - 1, s * kStage);
  }

  // `blocks`: this wavefront's token blocks that have rows; the others' products are left out.  AFTER:
  // with `after`, so many stores at least have been issued since start(); two slots' waits leave them on
  // their way.
  template <int AFTER = 0>
  __device__ void run(const unsigned char* (&from)[kLoads], int blocks, mma_f32x4 (&acc)[NB][MB], bool after = false) {
    if constexpr (ST == 2)
      run_interleaved<AFTER>(from, blocks, acc, after);
    else
      run_ring(from, blocks, acc);
    lds_barrier();
  }

  // ST slots.  A step's operands are read before the products of its first half: left to itself the
  // compiler reads the second half behind them (16 tokens of 8 wide experts: 169 us instead of 166).
  // With that a step's slot is free and loaded again while the products are made.  (Operands of the
  // step after read ahead as well: no faster anywhere, and twice the registers for operands.)
  __device__ void run_ring(const unsigned char* (&from)[kLoads], int blocks, mma_f32x4 (&acc)[NB][MB]) {
    unsigned slot = 0;
    if (steps >= ST)
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((ST - 1) * kLoads) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    StepProducts<F32, 2, NB, MB> products;
    for (int step = 0; step < steps; ++step) {
      mma_u32x4 w[2][NB], t[2][MB];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int n = 0; n < NB; ++n) w[s][n] = weight_block(slot, s, n);
#pragma unroll
        for (int m = 0; m < MB; ++m)
          if (m < blocks) t[s][m] = token_block(slot, s, m);
      }
      __builtin_amdgcn_sched_barrier(0);
      products.add(w, t, blocks, acc);
      if (step + 1 == steps) break;
      // the next step is there, and everybody has read this one
      if (step + ST <= steps)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((ST - 2) * kLoads) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (step + ST < steps) load_all(from, step + ST == steps - 1, slot);
      slot = slot == (ST - 1) * kStage ? 0 : slot + kStage;
    }
    products.last(acc);
  }

  // A ring of 64 x 128 for eight wavefronts of which four take the first half of every step and four the
  // second, each with 32 tokens x 64 weight rows: 6 blocks read from LDS for 8 products, where
  // 16 tokens x 64 rows of a whole step read 10.  Both halves' sums are left in LDS, see half_sums().
  __device__ void run_halves(const unsigned char* (&from)[kLoads], unsigned lds, int wave, int lane) {
    static_assert(BM == 64 && BN == 128 && kWaves == 8 && kLdsBytes >= 2 * 32 * 1024, "eight parts of 32 x 64");
    const int half = wave >> 2, rows = wave >> 1 & 1, columns = wave & 1;
    const unsigned get = lds + (lane & 15) * kStepBytes + ((((lane >> 4) ^ ((lane & 15) >> 1)) * 16) ^ (half * 64));
    const unsigned tokens = get + rows * 32 * kStepBytes, weights = get + (BM + columns * 64) * kStepBytes;
    mma_f32x4 acc[4][2];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int m = 0; m < 2; ++m) acc[n][m] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    unsigned slot = 0;
    if (steps >= ST)
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((ST - 1) * kLoads) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    StepProducts<F32, 1, 4, 2> products;
    for (int step = 0; step < steps; ++step) {
      mma_u32x4 w[1][4], t[1][2];
#pragma unroll
      for (int m = 0; m < 2; ++m) t[0][m] = read_lds(tokens + slot + m * 16 * kStepBytes);
#pragma unroll
      for (int n = 0; n < 4; ++n) w[0][n] = read_lds(weights + slot + n * 16 * kStepBytes);
      __builtin_amdgcn_sched_barrier(0);
      products.add(w, t, 2, acc);
      if (step + 1 == steps) break;
      if (step + ST <= steps)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((ST - 2) * kLoads) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (step + ST < steps) load_all(from, step + ST == steps - 1, slot);
      slot = slot == (ST - 1) * kStage ? 0 : slot + kStage;
    }
    products.last(acc);
    lds_barrier();
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int m = 0; m < 2; ++m)
        *(lds_f32x4)(size_t)(lds + (((half * 4 + rows * 2 + m) * 8 + columns * 4 + n) * 64 + lane) * 16) = acc[n][m];
    lds_barrier();
  }
  // block `n` of weight rows and `m` of tokens, after run_halves()
  static __device__ mma_f32x4 half_sums(unsigned lds, int m, int n, int lane) {
    const unsigned at = lds + ((m * 8 + n) * 64 + lane) * 16;
    return *(lds_f32x4)(size_t)at + *(lds_f32x4)(size_t)(at + 32 * 1024);
  }

  // Two slots, and a fixed order of everything within a step: 2 MB groups of NB products that
  // share a token block, each with one read from LDS for the group kAhead later and, behind the
  // barrier, one load of the step after the next.  The barrier lies where the last read of the
  // step's slot has been made, kAhead groups before its products are; what follows it reads the
  // other slot and refills this one.  (Left to itself the compiler puts the reads of half a
  // step right before their use, where both wavefronts of a SIMD wait for them at once: 8192 x
  // 8192 x 4096 in bf16 took 462 us instead of 387, with one more memory round trip exposed per
  // step; the matrix instructions alone, on the same operands, take 345: the card lowers its
  // clock under them.  Loads in bursts of two per group: 404; the barrier two groups later: 394.)
  template <int AFTER>
  __device__ void run_interleaved(const unsigned char* (&from)[kLoads], int blocks, mma_f32x4 (&acc)[NB][MB], bool after) {
    static_assert(kLoads + AFTER < 64, "vmcnt counts to 63");
    constexpr int kGroups = 2 * MB, kAhead = MB - 1;
    mma_u32x4 w[2][NB], t[MB];
    unsigned slot = 0;
    auto step = [&](auto next, auto issued, auto last) {  // `next`: another step follows; `issued`: and one more
      const int by = decltype(issued)::value ? stride() : 0;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const int behind = g - (kGroups - kAhead);  // groups since the barrier
        if (next && behind == 0) {
          if (AFTER != 0 && after) {  // (the first step's)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(AFTER) : "memory");
            after = false;
          } else {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          }
        }
        if (behind < 0 || next) {
          const int r = (g + kAhead) % kGroups;
          t[r % MB] = token_block(behind < 0 ? slot : slot ^ kStage, r / MB, r % MB);
        }
        if (g < NB) w[1][g] = weight_block(slot, 1, g);
        if (next && behind >= 0) {
#pragma unroll
          for (int n = 0; n < NB; ++n)
            if (n * kAhead / NB == behind) w[0][n] = weight_block(slot ^ kStage, 0, n);
          if constexpr (decltype(issued)::value) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
              if (i * kAhead / kLoads == behind) load(from, last, slot, i, by);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (g % MB < blocks)
#pragma unroll
          for (int n = 0; n < NB; ++n) acc[n][g % MB] = multiply<F32>(w[g / MB][n], t[g % MB], acc[n][g % MB]);
        __builtin_amdgcn_sched_barrier(0);
      }
      slot ^= kStage;
    };
    static_assert((kStage & (kStage - 1)) == 0 && NB <= MB, "slots that differ in one bit; weights of half a step read within it");
    if (steps == 1)
      asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    else if (AFTER != 0 && after)
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLoads + AFTER) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLoads) : "memory");
#pragma unroll
    for (int n = 0; n < NB; ++n) w[0][n] = weight_block(0, 0, n);
#pragma unroll
    for (int g = 0; g < kAhead; ++g) t[g] = token_block(0, 0, g);
    int left = steps - 1;
    for (; left > 2; --left) step(true_c{}, true_c{}, false_c{});
    if (left == 2) step(true_c{}, true_c{}, true_c{}), --left;
    if (left == 1) step(true_c{}, false_c{}, false_c{});
    step(false_c{}, false_c{}, false_c{});
  }
};

// Results -> memory by whole lines: a wavefront puts the blocks of its part of the tile into a
// piece of LDS of its own (`lds`: the first of them, BYTES each; the whole ring, or room beside it), as
// many token blocks at a time as fit, and reads them back row by row.  value(n, m): the four
// outputs of column block n < NC that this lane holds; place(row, column): where the 16 bytes
// beginning at that row and (wavefront's) column go, or NULL.  (Stores straight from the accumulators reach 16 rows with 32 or 64 bytes each:
// 98304 x 2048 x 1408 in bf16 took 525 us so and 485 this way, with fp32 results 560 and 515,
// with none 412.  They go past the caches: nobody reads them soon.)
template <bool F32, class TL, int NC, int BYTES = TL::kLdsBytes / TL::kWaves, typename VALUE, typename PLACE>
__device__ __forceinline__ void store_tile(unsigned lds, int wave, int lane, VALUE value, PLACE place) {
  constexpr int kBytes = BYTES;
  constexpr int kRow = NC * 16 * (F32 ? 4 : 2);      // bytes of a row
  constexpr int kFit = kBytes / (16 * kRow);
  constexpr int kPass = kFit < TL::MB ? kFit : TL::MB;      // token blocks at a time
  constexpr int kPieces = kRow / 16, kRows = 64 / kPieces;  // pieces of a row; rows per store instruction
  static_assert(kPass >= 1 && kPieces <= 16 && (kPieces & (kPieces - 1)) == 0, "whole instructions");
  const unsigned mine = lds + wave * kBytes;
  const int tok = lane & 15, quad = lane >> 4;
  constexpr int kTurn = kPieces - 1;  // (pieces are turned by the row, against bank conflicts)
#pragma unroll
  for (int m0 = 0; m0 < TL::MB; m0 += kPass) {
#pragma unroll
    for (int m = m0; m < m0 + kPass && m < TL::MB; ++m)
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const mma_f32x4 v = value(n, m);
        const unsigned row = mine + ((m - m0) * 16 + tok) * kRow;
        if constexpr (F32) {
          *(lds_f32x4)(size_t)(row + ((n * 4 + quad) ^ (tok & kTurn)) * 16) = v;
        } else {
          mma_u32x2 b;
#pragma unroll
          for (int i = 0; i < 2; ++i)
            b[i] = bf16_bits(v[2 * i]) | bf16_bits(v[2 * i + 1]) << 16;
          *(lds_u32x2)(size_t)(row + ((n * 2 + (quad >> 1)) ^ (tok & kTurn)) * 16 + (quad & 1) * 8) = b;
        }
      }
    asm volatile("" ::: "memory");  // (LDS serves a wavefront in order)
    constexpr int kStores = (kPass * 16 + kRows - 1) / kRows;
    mma_u32x4 d[kStores];
    mma_u32x4* to[kStores];
#pragma unroll
    for (int i = 0; i < kStores; ++i) {
      const int r = i * kRows + lane / kPieces, c = lane % kPieces;
      const int row = TL::block_row(wave, m0 + r / 16) + r % 16;
      const bool is = r < kPass * 16 && m0 + r / 16 < TL::MB;
      to[i] = is ? static_cast<mma_u32x4*>(place(row, c * (F32 ? 4 : 8))) : nullptr;
      d[i] = read_lds(mine + min(r, kPass * 16 - 1) * kRow + (c ^ (r & kTurn)) * 16);
    }
#pragma unroll
    for (int i = 0; i < kStores; ++i)
      if (to[i] != nullptr) __builtin_nontemporal_store(d[i], to[i]);
    asm volatile("" ::: "memory");
  }
}

// Number `v` of `total` workgroups that the eight XCDs take in turn -> the tile it computes,
// so that an XCD has one contiguous run of tiles (they share rows through its L2).
__device__ __forceinline__ int xcd_run(int v, int total) {
  const int q = total >> 3, r = total & 7, x = v & 7;
  return x * q + min(x, r) + (v >> 3);
}

}  // namespace laser
