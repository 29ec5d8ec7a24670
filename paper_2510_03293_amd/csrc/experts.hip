// The experts of a layer over the routing tables: laser_experts_up and laser_experts_down.
#include <algorithm>
#include <type_traits>

#include "../../include/laser.h"
#include "grouped.h"

namespace laser {

// What experts_down keeps of a slot until its token's sum is taken: the weighted product in fp32, whatever the
// type of the call.  Experts of a token may cancel, so that no rounding of a summand is small beside out's own.
// Written and read once each, these values are the largest part of a large call's traffic: 16384 tokens,
// 6 of 64 experts, H = 2048: 805 MB each way.
constexpr int kMostSlices = 16;  // of the contraction axis, experts_down

struct ExpertArgs {
  const unsigned char* x;    // rows of the token operand
  const unsigned char* w;    // [E, rows of an expert, K]
  const int32_t* permutation;  // NULL: one group, position = slot = row
  const int32_t* offsets;      // [E + 1] of the call's experts
  const float* weights;
  void* out;
  int slices;      // experts_down: parts of the contraction axis; out is [slices, slots, H] fp32
  int slots;   // T * k
  int k;
  int E;
  int K;       // bytes of a row of either operand
  int F;       // experts_up: columns of act
  int H;       // experts_down: columns of out
};

// The sum over the lanes up to this one.  (Lane exchanges inside the registers: through LDS it takes a microsecond
// per call where both sizes of tiles are counted.)
__device__ __forceinline__ int sum_up_to(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes before, in rows of 16,
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the last lane of rows 0 and 2 to rows 1 and 3,
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
  return x;
}

// The call's experts, one per lane: where their positions begin, how many there are, and, for tiles of
// BM rows, how many tiles the experts before have.
struct ExpertTiles {
  int lo, cnt, before, total;
  __device__ void init(const ExpertArgs& a, int lane) {
    if (a.offsets == nullptr) {
      lo = 0;
      cnt = lane == 0 ? a.slots : 0;
    } else {
      // (offsets are the caller's: whatever they hold, positions stay inside the tables)
      lo = lane < a.E ? min(max(a.offsets[lane], 0), a.slots) : 0;
      cnt = lane < a.E ? max(min(max(a.offsets[lane + 1], 0), a.slots) - lo, 0) : 0;
      if (a.slots > 1 << 24) {
        // (... and sums of what they may hold do not pass 32 bits: no position twice)
        int end = lo + cnt;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) end = max(end, __shfl_up(end, d));
        const int before_me = __shfl_up(end, 1);
        if (lane > 0) {
          cnt = max(lo + cnt - max(lo, before_me), 0);
          lo = max(lo, before_me);
        }
      }
    }
  }
  __device__ void count(int BM) {
    const int tiles = (int)(((unsigned)cnt + BM - 1) / BM);
    const int sum = sum_up_to(tiles);
    before = sum - tiles;
    total = __builtin_amdgcn_readlane(sum, 63);
  }
  // Tile `id` < total * nt of an order that goes expert by expert, so that the tiles which run side
  // by side share its rows: up to kGroup tiles of rows walk its nt tiles of columns together.
  __device__ void find(int id, int nt, int BM, int& e, int& p0, int& rows, int& column) const {
    constexpr int kGroup = 8;
    e = 63 - __builtin_clzll(__ballot(cnt > 0 && before <= id / nt));
    const int n = __builtin_amdgcn_readlane(cnt, e), mts = (int)(((unsigned)n + BM - 1) / BM);
    const int in_e = id - __builtin_amdgcn_readlane(before, e) * nt;
    const int g = in_e / (kGroup * nt), gm = min(kGroup, mts - g * kGroup), in = in_e - g * kGroup * nt;
    column = in / gm;
    const int row = (g * kGroup + in - column * gm) * BM;
    p0 = __builtin_amdgcn_readlane(lo, e) + row;
    rows = min(n - row, BM);
  }
};

constexpr int kBesideBytes = 2048;  // of a wavefront: 16 rows of 128 bytes of results

template <bool F32>
__device__ __forceinline__ float silu(float g) {
  // g / (1 + exp(-g)); a large negative g divides by infinity and gives -0
  if constexpr (F32) return g / (1.0f + expf(-g));
  return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}

// A workgroup computes tiles v, v + grid, ...; what the next one needs first is fetched while
// the one before is computed: its rows' entries of the permutation before run(), its first
// steps before the results are written.
template <bool F32, bool UP, class TL, bool SLICES = false>
__device__ __forceinline__ void experts_tiles(const ExpertArgs& a, unsigned char* ring, ExpertTiles tiles, int lane, int wave) {
  constexpr int BM = TL::BM, BN = TL::BN, NB = TL::NB, MB = TL::MB;
  static_assert(BM <= TL::kThreads, "one thread per row of the tile");
  // behind the ring: per row of the tile its token (UP) or its slot and weight
  int* const row_of = reinterpret_cast<int*>(ring + TL::kLdsBytes);
  float* const weight_of = reinterpret_cast<float*>(row_of + 2 * BM);
  tiles.count(BM);
  constexpr int kCols = UP ? BN / 2 : BN;  // output columns of a tile
  constexpr int kWaveCols = kCols / TL::WN;
  const int cols = UP ? a.F : a.H;
  const int nt = (cols + kCols - 1) / kCols;
  const int total = tiles.total * nt;
  const int wn = wave / TL::WM;
  const unsigned lds = (unsigned)(size_t)(lds_bytes)ring;
  // (slices of whole steps)
  const int steps = (a.K + kStepBytes - 1) / kStepBytes, slice = SLICES ? blockIdx.y : 0;
  const int begin_at = SLICES ? (int)((long long)steps * slice / a.slices) * kStepBytes : 0;
  const int end_at = SLICES ? min((int)((long long)steps * (slice + 1) / a.slices) * kStepBytes, a.K) : a.K;
  TL tile(end_at - begin_at, lds, wave, lane);

  int e, p0, rows, c0;
  auto find = [&](int v) {
    int column;
    tiles.find(xcd_run(v, total), nt, BM, e, p0, rows, column);
    c0 = column * kCols;
  };
  // this thread's row of the tile: its slot (rows past the end repeat the last one)
  auto slot_of = [&]() {
    const int p = p0 + min((int)threadIdx.x, rows - 1);
    return a.permutation != nullptr && threadIdx.x < BM ? a.permutation[p] : p;
  };
  auto put_row = [&](int slot, int buf) {
    slot = min(max(slot, 0), a.slots - 1);
    if (threadIdx.x < BM) row_of[buf * BM + threadIdx.x] = UP ? slot / a.k : slot;
    return slot;
  };
  const unsigned char* from[TL::kLoads];
  auto begin = [&](int buf, int lane) {
    // (wide tiles of an expert share its weights through L2 while they are at the same step; narrow
    // ones read them once: 64 experts, 64 tokens 146 -> 130 us with turns, 8 experts, 16 tokens 175 -> 162)
    tile.turn_to(TL::ST == 2 ? e : e * 5 + c0 / kCols);
    const int piece = TL::piece(wave, lane) * 16 + tile.turn * kStepBytes + begin_at;
#pragma unroll
    for (int i = 0; i < TL::kLoads; ++i) {
      const int r = TL::row(wave, lane, i);
      if (r < BM) {
        const int row = UP ? row_of[buf * BM + r] : p0 + min(r, rows - 1);
        from[i] = a.x + (size_t)row * a.K + piece;
      } else {
        int n = r - BM, row;
        if constexpr (UP) {  // a wavefront's rows: first of the gate matrix, then the same of the up matrix
          const int half = n % (2 * kWaveCols) / kWaveCols;
          row = half * a.F + min(c0 + n / (2 * kWaveCols) * kWaveCols + n % kWaveCols, a.F - 1);
        } else {
          row = min(c0 + n, a.H - 1);
        }
        from[i] = a.w + ((size_t)e * (UP ? 2 * a.F : a.H) + row) * a.K + piece;
      }
    }
  };

  // With two slots the results are staged beside the ring, so that both slots are filled meanwhile, and
  // the stores of a tile without gaps (kStores of a wavefront, 1 KiB each) are still on their way while the
  // next tile's first steps are multiplied.
  constexpr bool kBeside = TL::ST == 2;
  constexpr int kStores = !kBeside ? 0 : UP ? MB * (NB / 2) / 2 : MB * NB;
  int v = blockIdx.x, buf = 0;
  bool after = false;
  if (v >= total) return;
  find(v);
  int slot = put_row(slot_of(), buf);
  lds_barrier();
  begin(buf, lane);
  tile.start(from);
  for (;;) {
    const int now_p0 = p0, now_rows = rows, now_c0 = c0;
    float weight = 1.0f;
    if (!UP && a.weights != nullptr && threadIdx.x < BM) weight = a.weights[slot];
    v += gridDim.x;
    if (v < total) {
      find(v);
      slot = slot_of();
    }
    mma_f32x4 acc[NB][MB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int m = 0; m < MB; ++m) acc[n][m] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    tile.template run<kStores>(from, TL::blocks_of(wave, now_rows), acc, after);
    after = now_rows == BM && now_c0 + kCols <= cols;

    if (!UP && threadIdx.x < BM) weight_of[threadIdx.x] = weight;
    if (v < total) slot = put_row(slot, buf ^ 1);
    lds_barrier();
    // (what follows depends on the lane alone: kept from moving out of the loop, where it would
    // occupy the registers that the products need)
    int l = lane;
    asm volatile("" : "+v"(l));
    if (v < total) {
      begin(buf ^ 1, l);
      if (kBeside) {
        tile.start(from);
        asm volatile("" ::: "memory");  // (`after` counts what is issued behind these loads)
      }
    }
    constexpr int kRoom = kBeside ? kBesideBytes : TL::kLdsBytes / TL::kWaves;
    const unsigned staging = kBeside ? lds + TL::kLdsBytes + TL::BM * 12 : lds;
    if constexpr (UP) {
      store_tile<F32, TL, NB / 2, kRoom>(
          staging, wave, l,
          [&](int n, int m) {
            mma_f32x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = silu<F32>(acc[n][m][i]) * acc[NB / 2 + n][m][i];
            return y;
          },
          [&](int r, int c) -> void* {
            const int f = now_c0 + wn * kWaveCols + c;
            return r < now_rows && f < a.F ? static_cast<char*>(a.out) + ((size_t)(now_p0 + r) * a.F + f) * (F32 ? 4 : 2)
                                           : nullptr;
          });
    } else {
      float by[MB];
#pragma unroll
      for (int m = 0; m < MB; ++m) by[m] = weight_of[TL::block_row(wave, m) + (l & 15)];
      // (beside the ring there is room for half of a wavefront's columns at a time)
      constexpr int kAtOnce = kBeside ? NB / 2 : NB;
#pragma unroll
      for (int n0 = 0; n0 < NB; n0 += kAtOnce)
        store_tile<true, TL, kAtOnce, kRoom>(
            staging, wave, l, [&](int n, int m) { return acc[n0 + n][m] * by[m]; },
            [&](int r, int c) -> void* {
              const int h = now_c0 + wn * kWaveCols + n0 * 16 + c;
              const size_t slot = (size_t)slice * a.slots + row_of[buf * BM + r];
              return r < now_rows && h < a.H ? static_cast<float*>(a.out) + slot * a.H + h : nullptr;
            });
    }
    if (v >= total) break;
    if (!kBeside) {
      lds_barrier();  // (everybody's results have left the ring)
      tile.start(from);
    }
    buf ^= 1;
  }
}

// How many rows the call's experts have, and how they fill tiles, is known on the device only: a call
// that wide tiles may suit is launched with wide ones and with others, and one of the two
// launches finds that it is not meant.
//
// What the two would take, in twentieths of a microsecond: as many rounds of tiles as workgroups run
// side by side, of so much per step and so much before and behind the steps (fitted to the figures
// below; of a compute unit's two workgroups with 128 x 128 each has half of the steps' rate).
//   us with 128 x 128, 256 x 256:  up of H = 2048, F = 1408, 64 experts, 2048 tokens 226, 204, 4096 tokens 354,
//   303;  down of the same 164, 139 and 262, 239;  16 of the 64 experts, down of 1910 rows 35, 39, of 3763 rows 44,
//   51;  8 experts, H = 4096, up of F = 2048 and 1024 tokens 114, 92, down of F = 4096 and 1500 tokens 156, 130
struct Wide {
  using TL = Tile<false, 256, 256, 2, 4, 2>;
  static constexpr int kPerCu = 1, kStep = 25, kTile = 120, kOnce = 120;
};
struct Medium {
  using TL = Tile<false, 128, 128, 2, 2, 2>;
  static constexpr int kPerCu = 2, kStep = 19, kTile = 120, kOnce = 0;
};
template <class HOW, bool UP>
__device__ __forceinline__ long long cost_of(const ExpertArgs& a, ExpertTiles& tiles, unsigned units) {
  tiles.count(HOW::TL::BM);
  constexpr int kCols = UP ? HOW::TL::BN / 2 : HOW::TL::BN;
  const long long all = (long long)tiles.total * (((UP ? a.F : a.H) + kCols - 1) / kCols);
  // (a division in 64 bits would take longer than the rest)
  const unsigned most = (unsigned)(all < (1 << 30) ? all : (1 << 30));
  const unsigned rounds = (most + HOW::kPerCu * units - 1) / (HOW::kPerCu * units);
  // (in integers: the two launches have to come to the same)
  return (long long)rounds * (HOW::kStep * ((a.K + kStepBytes - 1) / kStepBytes) + HOW::kTile) + HOW::kOnce;
}

enum Choose { kSure, kIfWide, kIfMedium };
template <bool F32, bool UP, class TL, Choose WHEN>
__global__ __launch_bounds__(TL::kThreads) void experts_kernel(ExpertArgs a, unsigned units) {
  extern __shared__ __align__(1024) unsigned char ring[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  ExpertTiles tiles;
  tiles.init(a, lane);
  if constexpr (WHEN != kSure) {
    const bool wide = cost_of<Wide, UP>(a, tiles, units) <= cost_of<Medium, UP>(a, tiles, units);
    if (wide != (WHEN == kIfWide)) return;
  }
  experts_tiles<F32, UP, TL>(a, ring, tiles, lane, wave);
}

// Sums over slices of the contraction axis.
template <bool F32, class TL>
__global__ __launch_bounds__(TL::kThreads) void experts_slices_kernel(ExpertArgs a) {
  extern __shared__ __align__(1024) unsigned char ring[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  ExpertTiles tiles;
  tiles.init(a, lane);
  experts_tiles<F32, false, TL, true>(a, ring, tiles, lane, wave);
}

// ---- a few tokens -------------------------------------------------------------------
// Up to kFewTokens tokens, whose assignments nearly all go to experts of their own: products of
// matrices with single vectors, bound by reading the weights once.  A wavefront takes whole rows
// of them, 1 KiB per load instruction, and a lane multiplies its 16 bytes with the same piece of
// the vector; no LDS on the way and nothing to wait for, so that all of a row's loads are in
// flight.  (One token, 6 of 64 experts, H = 2048, F = 1408: the tiles' kernel has 132 workgroups
// for that, each with one vector in 64 rows' place.)

constexpr int kFewTokens = 4;
constexpr int kFewSlots = 64;   // (one per lane)

template <bool F32>
__device__ __forceinline__ float dot16(mma_u32x4 a, mma_u32x4 b, float sum) {
  if constexpr (F32) {
    const mma_f32x4 x = __builtin_bit_cast(mma_f32x4, a), y = __builtin_bit_cast(mma_f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = fmaf(x[i], y[i], sum);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum = fmaf(bf16_value(a[i] & 0xffffu), bf16_value(b[i] & 0xffffu), sum);
      sum = fmaf(__builtin_bit_cast(float, a[i] & 0xffff0000u), __builtin_bit_cast(float, b[i] & 0xffff0000u), sum);
    }
  }
  return sum;
}
__device__ __forceinline__ float lanes_sum(float x) {  // in all lanes, one fixed order
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// sum[r] += row[r] times vector over the lane's pieces of chunks begin .. end - 1 (1 KiB each).
// ONCE: nobody reads the rows again, so they go past the caches.  One token (no expert twice): up
// 16.9 -> 14.2 us, down 12.6 -> 11.7; four tokens of 8 experts: down 111 -> 132.
template <bool F32, bool ONCE, int ROWS, int BATCH>
__device__ __forceinline__ void row_products(const unsigned char* const (&row)[ROWS], const unsigned char* vector, int bytes,
                                             int begin, int end, int lane, float (&sum)[ROWS]) {
  for (int c = begin; c < end; c += BATCH) {
    mma_u32x4 x[BATCH], w[BATCH][ROWS];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int at = (c + i) * 1024 + lane * 16;
      const bool in = c + i < end && at < bytes;
      const int from = in ? at : 0;
      x[i] = *reinterpret_cast<const mma_u32x4*>(vector + from);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        w[i][r] = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const mma_u32x4*>(row[r] + from))
                       : *reinterpret_cast<const mma_u32x4*>(row[r] + from);
        if (!in) w[i][r] = mma_u32x4{0, 0, 0, 0};
      }
      if (!in) x[i] = mma_u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
#pragma unroll
      for (int r = 0; r < ROWS; ++r) sum[r] = dot16<F32>(w[i][r], x[i], sum[r]);
  }
}

// The expert (of the call's) whose range of positions holds p, or -1; the same p in all lanes.
__device__ __forceinline__ int expert_of(const ExpertTiles& t, int p) {
  const unsigned long long has = __ballot(p >= t.lo && p < t.lo + t.cnt);
  return has == 0 ? -1 : __builtin_ctzll(has);
}

// blockIdx.x: the position; blockIdx.y: 4 wavefronts x COLUMNS columns of act (one token: 12.9 us with
// one column, 14.2 with two; four tokens 42.8 and 42.3).
template <bool F32, bool ONCE, int COLUMNS>
__global__ __launch_bounds__(256) void experts_up_few_kernel(ExpertArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int p = blockIdx.x, f0 = (blockIdx.y * 4 + wave) * COLUMNS;
  ExpertTiles tiles;
  tiles.init(a, lane);
  const int e = expert_of(tiles, p);
  if (e < 0 || f0 >= a.F) return;
  const int t = a.permutation != nullptr ? min(max(a.permutation[p], 0), a.slots - 1) / a.k : p;
  const unsigned char* row[2 * COLUMNS];
#pragma unroll
  for (int i = 0; i < COLUMNS; ++i) {
    row[i] = a.w + ((size_t)e * 2 * a.F + min(f0 + i, a.F - 1)) * a.K;
    row[COLUMNS + i] = row[i] + (size_t)a.F * a.K;
  }
  float sum[2 * COLUMNS] = {};
  row_products<F32, ONCE, 2 * COLUMNS, 4>(row, a.x + (size_t)t * a.K, a.K, 0, (a.K + 1023) >> 10, lane, sum);
#pragma unroll
  for (int i = 0; i < COLUMNS; ++i) {
    const float y = silu<F32>(lanes_sum(sum[i])) * lanes_sum(sum[COLUMNS + i]);
    if (lane == 0 && f0 + i < a.F) {
      if constexpr (F32) static_cast<float*>(a.out)[(size_t)p * a.F + f0 + i] = y;
      else static_cast<unsigned short*>(a.out)[(size_t)p * a.F + f0 + i] = (unsigned short)bf16_bits(y);
    }
  }
}

// ROWS rows of the matrices (columns of out) per workgroup, as many as leave two workgroups for every
// compute unit (H = 2048, one token: eight rows 11.7 us, four 11.1; H = 128, three tokens: eight 26.8,
// two 19.4).  Its wavefronts take the slots in turn, and where there are fewer slots than wavefronts,
// parts of the rows as well; what they find waits in LDS for its place in the sums, which run in slot order.
constexpr int kFewWaves = 8;
template <bool F32, bool ONCE, int ROWS>
__global__ __launch_bounds__(64 * kFewWaves) void experts_down_few_kernel(ExpertArgs a, const int32_t* ids, int first,
                                                                          const void* base, void* out, int T) {
  __shared__ float found[kFewSlots * ROWS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h0 = blockIdx.x * ROWS;
  ExpertTiles tiles;
  tiles.init(a, lane);
  // the slot at this lane's position (positions and slots: one per lane)
  const int at = lane < a.slots ? (a.permutation != nullptr ? a.permutation[lane] : lane) : -1;
  const int parts = a.slots <= kFewWaves / 4 ? 4 : a.slots <= kFewWaves / 2 ? 2 : 1;
  const int chunks = (a.K + 1023) >> 10;
  auto mine = [&](int slot) { return ids == nullptr || (unsigned)(ids[slot] - first) < (unsigned)a.E; };
  for (int u = wave; u < a.slots * parts; u += kFewWaves) {
    const int slot = u / parts, part = u - slot * parts;
    const unsigned long long where = __ballot(at == slot);
    const int p = where == 0 ? -1 : __builtin_ctzll(where);
    const int e = p < 0 ? -1 : expert_of(tiles, p);
    float sum[ROWS] = {};
    if (e >= 0 && mine(slot)) {
      const unsigned char* row[ROWS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) row[r] = a.w + ((size_t)e * a.H + min(h0 + r, a.H - 1)) * a.K;
      row_products<F32, ONCE, ROWS, 3>(row, a.x + (size_t)p * a.K, a.K, chunks * part / parts, chunks * (part + 1) / parts,
                                     lane, sum);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float s = lanes_sum(sum[r]);
      if (lane == 0) found[u * ROWS + r] = s;
    }
  }
  __syncthreads();
  const int r = threadIdx.x % ROWS, t = threadIdx.x / ROWS, h = h0 + r;
  if (t >= T || h >= a.H) return;
  float y = 0.0f;
  if (base != nullptr)
    y = F32 ? static_cast<const float*>(base)[(size_t)t * a.H + h]
            : bf16_value(static_cast<const unsigned short*>(base)[(size_t)t * a.H + h]);
  for (int slot = t * a.k; slot < (t + 1) * a.k; ++slot) {
    if (!mine(slot)) continue;
    float z = 0.0f;
    for (int part = 0; part < parts; ++part) z += found[(slot * parts + part) * ROWS + r];
    y += z * (a.weights != nullptr ? a.weights[slot] : 1.0f);
  }
  if constexpr (F32) static_cast<float*>(out)[(size_t)t * a.H + h] = y;
  else static_cast<unsigned short*>(out)[(size_t)t * a.H + h] = (unsigned short)bf16_bits(y);
}

// out[t,:] = base[t,:] + the products of the token's slots that the call's experts hold, in
// slot order.  One thread per four columns; the rows of kBatch slots are under way at a time.
template <bool F32>
__global__ __launch_bounds__(256) void experts_combine_kernel(const float* z, const int32_t* ids, const void* base, void* out,
                                                              int T, int H, int k, int first, int E) {
  constexpr int kBatch = 4;
  const int pieces = H / 4;
  const size_t all = (size_t)T * pieces;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (size_t)gridDim.x * 256) {
    const size_t t = i / pieces;
    const int h = (int)(i - t * pieces) * 4;
    mma_f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
    if (base != nullptr) y = load4<F32>(base, t * H + h);
    for (int j = 0; j < k; j += kBatch) {
      mma_f32x4 row[kBatch];
      bool is[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        is[u] = j + u < k && (ids == nullptr || (unsigned)(ids[t * k + min(j + u, k - 1)] - first) < (unsigned)E);
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (is[u]) row[u] = __builtin_nontemporal_load(reinterpret_cast<const mma_f32x4*>(z + (t * k + j + u) * H + h));
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (is[u]) y += row[u];
    }
    store4<F32>(out, t * H + h, y);
  }
}

// The same from sums of slices, [slices, T k, H] fp32: a slot's slices first.  One thread per four columns.
template <bool F32>
__global__ __launch_bounds__(256) void experts_join_kernel(const float* parts, int slices, const int32_t* ids, const void* base,
                                                           void* out, int T, int H, int k, int first, int E) {
  const int pieces = H / 4;
  const size_t all = (size_t)T * pieces, next = (size_t)T * k * H;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (size_t)gridDim.x * 256) {
    const size_t t = i / pieces;
    const int h = (int)(i - t * pieces) * 4;
    mma_f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
    if (base != nullptr) y = load4<F32>(base, t * H + h);
    for (int j = 0; j < k; ++j) {
      if (ids != nullptr && (unsigned)(ids[t * k + j] - first) >= (unsigned)E) continue;
      const float* const row = parts + (t * k + j) * H + h;
      mma_f32x4 part[kMostSlices];
#pragma unroll
      for (int s = 0; s < kMostSlices; ++s)
        part[s] = s < slices ? *reinterpret_cast<const mma_f32x4*>(row + s * next) : mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      mma_f32x4 sum = part[0];
#pragma unroll
      for (int s = 1; s < kMostSlices; ++s) sum += part[s];
      y += sum;
    }
    store4<F32>(out, t * H + h, y);
  }
}

constexpr int kGridMost = 1 << 20;

template <class TL>
constexpr int lds_of() {  // the ring, the table of the tile's rows, and with two slots room for results
  return TL::kLdsBytes + TL::BM * 12 + (TL::ST == 2 ? kBesideBytes * TL::kWaves : 0);
}
template <class TL, bool UP>
static long long grid_of(const ExpertArgs& a) {
  // (every expert with rows has at most one tile that is not full, and every tile a row)
  const long long mt = std::min<long long>(a.slots, a.slots / TL::BM + std::min(a.E, a.slots));
  const int cols = UP ? TL::BN / 2 : TL::BN;
  return mt * (((UP ? a.F : a.H) + cols - 1) / cols);
}

template <bool F32, bool UP, class TL, Choose WHEN>
static hipError_t launch_experts(const ExpertArgs& a, long long most, hipStream_t s) {
  static LdsAttr attr;
  const void* fn = reinterpret_cast<const void*>(&experts_kernel<F32, UP, TL, WHEN>);
  hipError_t err = allow_dynamic_lds(fn, lds_of<TL>(), attr);
  if (err != hipSuccess) return err;
  const unsigned grid = (unsigned)std::min(grid_of<TL, UP>(a), most);
  hipLaunchKernelGGL((experts_kernel<F32, UP, TL, WHEN>), dim3(grid), dim3(TL::kThreads), lds_of<TL>(), s, a,
                     (unsigned)compute_units());
  return hipGetLastError();
}

// Which tiles.  bf16, by the rows per expert if they were even, of which the host knows an upper bound
// (the call's experts may be a share of the layer's): few, 64 x 128, whose weights go past the caches and are read
// again where an expert has more than 64 rows; more, what cost_of says.  (64 x 128 and 128 x 128, up of H = 2048,
// F = 1408, 64 experts, popularity even: 48 rows per expert 128, 142 us, 58 rows 153, 141, 66 rows 195, 145, 94 rows
// 231, 152; skewed: 52 rows 152, 154, 58 rows 163, 154.  Down of the same, even: 48 rows 84, 86, 58 rows 93, 89,
// 94 rows 144, 99.)  Where the rows have so few steps that 256 x 256 cannot win, 128 x 128 (8000 tokens, 2000 rows per expert, 128 x 128 and 256 x 256: down of
// F = 320 76, 85, F = 1024 118, 125; up of H = 136 62, 80, H = 640 103, 102, H = 1024 145, 141).
// fp32 is bound by its matrix instructions (a sixteenth of the rate) as soon as there are tiles for
// all compute units; before that, small tiles are more of them (333 tokens, 33 experts, 516 x 212: 30 us
// with tiles of 64 x 128, 19 with 32 x 64; 4000 tokens, 8 experts, 1024 x 1024: 354 and 425).
constexpr int kSomeRows = 56, kWideSteps = 18;
template <bool F32, bool UP>
static hipError_t launch_products(const ExpertArgs& a, hipStream_t s) {
  // (most experts then have one tile of rows, so their weights are read once: 64 tokens on 64 experts 128 us,
  // past the caches 114; 16 on 8 wide ones 162, 145.  With 128 x 128 it is the other way round: 200, 211)
  using LOW = Tile<F32, 64, 128, 2, 2, 3, F32 ? kNeither : kWeights>;
  if constexpr (F32) {
    if (grid_of<LOW, UP>(a) < compute_units())
      return launch_experts<F32, UP, Tile<F32, 32, 64, 2, 2, 6>, kSure>(a, kGridMost, s);
  } else if (a.slots >= (long long)kSomeRows * a.E) {
    const long long most = Medium::kPerCu * 2 * compute_units();
    if (a.K < kWideSteps * kStepBytes) return launch_experts<F32, UP, Medium::TL, kSure>(a, most, s);
    const hipError_t err = launch_experts<F32, UP, Wide::TL, kIfWide>(a, Wide::kPerCu * compute_units(), s);
    return err != hipSuccess ? err : launch_experts<F32, UP, Medium::TL, kIfMedium>(a, most, s);
  }
  return launch_experts<F32, UP, LOW, kSure>(a, kGridMost, s);
}

// experts_down with few tiles and a long way along the contraction axis takes that in slices, at least
// kSliceSteps steps each, as many as make kSliceWorkgroups of the tiles.  (69 tokens on 5 experts, H = 248, F = 12760:
// 119 us in one, 16 in slices; 16 on 8, H = 512, F = 2416 27, 14; 300 on 4, H = 512, F = 1024 16.4, 14; 700 on one,
// H = 1024, F = 2048 30, 17.)  Half of that where an expert's tiles do not share its weights, which then
// bound the call: 500 on 4, H = 1024, F = 4096 with 256 47 us, with 512 27; 16 on 8, H = 4096, F = 14336 145, 170.
constexpr int kSliceSteps = 8, kSliceWorkgroups = 512, kSharedRows = 32;
template <bool F32>
using SliceTile = Tile<F32, 64, 128, 2, 2, 3>;
template <bool F32>
static int slices_of(const ExpertArgs& a) {
  const long long units = grid_of<SliceTile<F32>, false>(a), steps = (a.K + kStepBytes - 1) / kStepBytes;
  const int workgroups = a.slots >= (long long)kSharedRows * a.E ? kSliceWorkgroups : kSliceWorkgroups / 2;
  return (int)std::max<long long>(1, std::min<long long>({kMostSlices, workgroups / units, steps / kSliceSteps}));
}
// (values times slices are at most those of kSliceWorkgroups tiles)
static size_t slices_bytes(size_t slots, int H) {
  return std::min<size_t>(slots * H * kMostSlices, (size_t)kSliceWorkgroups * 64 * 128) * 4;
}
template <bool F32>
static hipError_t launch_slices(const ExpertArgs& a, hipStream_t s) {
  using TL = SliceTile<F32>;
  static LdsAttr attr;
  const void* fn = reinterpret_cast<const void*>(&experts_slices_kernel<F32, TL>);
  hipError_t err = allow_dynamic_lds(fn, lds_of<TL>(), attr);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((experts_slices_kernel<F32, TL>), dim3((unsigned)grid_of<TL, false>(a), a.slices), dim3(TL::kThreads),
                     lds_of<TL>(), s, a);
  return hipGetLastError();
}

static int check_experts(int32_t T, int32_t H, int32_t F, int32_t E, const laser_experts_params_t* p) {
  if (!p) return LASER_E_NULL;
  if (p->struct_bytes != sizeof(laser_experts_params_t)) return LASER_E_STRUCT;
  if (T < 0 || H < 1 || F < 1 || E < 1 || p->k < 1 || p->first_expert < 0) return LASER_E_RANGE;
  if ((int64_t)T * p->k > 0x7fffffffLL || F > (1 << 28) || H > (1 << 28)) return LASER_E_RANGE;
  if (p->dtype != LASER_DTYPE_F32 && p->dtype != LASER_DTYPE_BF16) return LASER_E_RANGE;
  if (p->k > LASER_MAX_K || E > LASER_MAX_E - p->first_expert) return LASER_E_UNSUPPORTED;
  const int whole = p->dtype == LASER_DTYPE_F32 ? 4 : 8;
  if (H % whole != 0 || F % whole != 0) return LASER_E_ALIGN;
  return LASER_OK;
}

// Whether a call goes as products with single vectors, `rows` rows of an expert's matrices for each slot.  (F: a
// dimension of the grid.)  Rows that are shorter than a load instruction leave lanes without work, which
// tiles do not once there are many: 8 slots, up of H = 248, F = 8320 39 us so, 22 in tiles, of H = 400, F = 1408 7.6,
// 7.7; 18 slots, up of H = 400, F = 1408 15.7, 12.9, down of F = 400, H = 1024 11.6, 15.
constexpr int kShortBytes = 1024, kShortRows = 1 << 15;
static bool are_few(int T, const ExpertArgs& a, long long rows) {
  return T <= kFewTokens && a.slots <= kFewSlots && a.F <= 1 << 17 && (a.K >= kShortBytes || a.slots * rows <= kShortRows);
}

static size_t whole_256(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
static size_t summands_bytes(size_t slots, int H) { return whole_256(slots * H * 4); }
static bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Without tables: one expert that takes every token once.
static int check_tables(const int32_t* permutation, const int32_t* offsets, int32_t E,
                        const laser_experts_params_t* p) {
  if (permutation && offsets) return LASER_OK;
  if (permutation || offsets) return LASER_E_NULL;
  return E == 1 && p->k == 1 && p->first_expert == 0 ? LASER_OK : LASER_E_NULL;
}

}  // namespace laser

using namespace laser;

extern "C" int laser_experts_up(const void* hidden, const void* w_up, int32_t T, int32_t H, int32_t F, int32_t E,
                                const laser_experts_params_t* params, const int32_t* permutation,
                                const int32_t* expert_offsets, void* act, void* hip_stream) {
  int rc = check_experts(T, H, F, E, params);
  if (rc != LASER_OK) return rc;
  if (T == 0) return LASER_OK;
  if (!hidden || !w_up || !act) return LASER_E_NULL;
  rc = check_tables(permutation, expert_offsets, E, params);
  if (rc != LASER_OK) return rc;
  if (misaligned(hidden) || misaligned(w_up) || misaligned(act)) return LASER_E_ALIGN;
  const bool f32 = params->dtype == LASER_DTYPE_F32;
  ExpertArgs a = {};
  a.x = static_cast<const unsigned char*>(hidden);
  a.w = static_cast<const unsigned char*>(w_up);
  a.permutation = permutation;
  a.offsets = expert_offsets ? expert_offsets + params->first_expert : nullptr;
  a.out = act;
  a.slots = T * params->k;
  a.k = params->k;
  a.E = E;
  a.K = H * (f32 ? 4 : 2);
  a.F = F;
  a.H = H;
  clear_stale_error();
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (are_few(T, a, 2ll * F)) {
    const int columns = T == 1 ? 1 : 2;
    const dim3 grid(a.slots, (F + 4 * columns - 1) / (4 * columns));
    auto* const kernel = f32 ? (T == 1 ? &experts_up_few_kernel<true, true, 1> : &experts_up_few_kernel<true, false, 2>)
                             : (T == 1 ? &experts_up_few_kernel<false, true, 1> : &experts_up_few_kernel<false, false, 2>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? LASER_OK : LASER_E_LAUNCH;
  }
  const hipError_t err = f32 ? launch_products<true, true>(a, s) : launch_products<false, true>(a, s);
  return err == hipSuccess ? LASER_OK : LASER_E_LAUNCH;
}

extern "C" size_t laser_experts_workspace_bytes(int32_t T, int32_t H, int32_t F, int32_t E,
                                                const laser_experts_params_t* params) {
  if (check_experts(T, H, F, E, params) != LASER_OK) return 0;
  const size_t slots = (size_t)T * params->k;
  return summands_bytes(slots, H) + whole_256(slices_bytes(slots, H)) + 256;
}

extern "C" int laser_experts_down(const void* act, const void* w_down, int32_t T, int32_t H, int32_t F, int32_t E,
                                  const laser_experts_params_t* params, const int32_t* permutation,
                                  const int32_t* expert_offsets, const int32_t* expert_ids, const float* weights,
                                  const void* base, void* out, void* workspace, size_t workspace_bytes,
                                  void* hip_stream) {
  int rc = check_experts(T, H, F, E, params);
  if (rc != LASER_OK) return rc;
  if (T == 0) return LASER_OK;
  if (!act || !w_down || !out || !workspace) return LASER_E_NULL;
  rc = check_tables(permutation, expert_offsets, E, params);
  if (rc != LASER_OK) return rc;
  if (misaligned(act) || misaligned(w_down) || misaligned(out) || misaligned(base)) return LASER_E_ALIGN;
  if ((uintptr_t)workspace & 255) return LASER_E_ALIGN;
  if (workspace_bytes < laser_experts_workspace_bytes(T, H, F, E, params)) return LASER_E_WORKSPACE;
  const bool f32 = params->dtype == LASER_DTYPE_F32;
  ExpertArgs a = {};
  a.x = static_cast<const unsigned char*>(act);
  a.w = static_cast<const unsigned char*>(w_down);
  a.permutation = permutation;
  a.offsets = expert_offsets ? expert_offsets + params->first_expert : nullptr;
  a.weights = weights;
  a.out = workspace;
  a.slots = T * params->k;
  a.k = params->k;
  a.E = E;
  a.K = F * (f32 ? 4 : 2);
  a.F = F;
  a.H = H;
  clear_stale_error();
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (are_few(T, a, H)) {
    const int rows = H >= 16 * compute_units() ? 8 : H >= 8 * compute_units() ? 4 : 2;
    const dim3 grid((H + rows - 1) / rows), block(64 * kFewWaves);
    auto pick = [&](auto is32, auto once) {
      constexpr bool k32 = decltype(is32)::value, kOnce = decltype(once)::value;
      return rows == 8   ? &experts_down_few_kernel<k32, kOnce, 8>
             : rows == 4 ? &experts_down_few_kernel<k32, kOnce, 4>
                         : &experts_down_few_kernel<k32, kOnce, 2>;
    };
    auto* const kernel = f32 ? (T == 1 ? pick(std::true_type{}, std::true_type{}) : pick(std::true_type{}, std::false_type{}))
                             : (T == 1 ? pick(std::false_type{}, std::true_type{}) : pick(std::false_type{}, std::false_type{}));
    hipLaunchKernelGGL(kernel, grid, block, 0, s, a, expert_ids, params->first_expert, base, out, T);
    return hipGetLastError() == hipSuccess ? LASER_OK : LASER_E_LAUNCH;
  }
  a.slices = f32 ? slices_of<true>(a) : slices_of<false>(a);
  if (a.slices > 1) {
    float* const parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + summands_bytes(a.slots, H));
    a.out = parts;
    const hipError_t err = f32 ? launch_slices<true>(a, s) : launch_slices<false>(a, s);
    if (err != hipSuccess) return LASER_E_LAUNCH;
    const unsigned grid = (unsigned)std::min<size_t>(((size_t)T * (H / 4) + 255) / 256, 1 << 16);
    auto* const join = f32 ? &experts_join_kernel<true> : &experts_join_kernel<false>;
    hipLaunchKernelGGL(join, dim3(grid), dim3(256), 0, s, parts, a.slices, expert_ids, base, out, T, H, params->k,
                       params->first_expert, E);
    return hipGetLastError() == hipSuccess ? LASER_OK : LASER_E_LAUNCH;
  }
  const hipError_t err = f32 ? launch_products<true, false>(a, s) : launch_products<false, false>(a, s);
  if (err != hipSuccess) return LASER_E_LAUNCH;
  const unsigned grid = (unsigned)std::min<size_t>(((size_t)T * (H / 4) + 255) / 256, 1 << 16);
  auto* const combine = f32 ? &experts_combine_kernel<true> : &experts_combine_kernel<false>;
  hipLaunchKernelGGL(combine, dim3(grid), dim3(256), 0, s, static_cast<const float*>(workspace), expert_ids, base, out, T, H,
                     params->k, params->first_expert, E);
  return hipGetLastError() == hipSuccess ? LASER_OK : LASER_E_LAUNCH;
}
