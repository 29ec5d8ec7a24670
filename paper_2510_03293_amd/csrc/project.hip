// A projection that all rows of a batch share, and beside it the low-rank adapters that the
// requests of the batch bring along: laser_project_adapted.
//
//   out[t, :] = W x_t + U_m (scale_m D_m x_t),   m the adapter of row t's request
//
// Where there is little to do side by side (see launch_project) the contraction axis is cut into
// slices: one launch for sums over slices, of W and of the adapters' inner matrices alike, and one
// that joins them.  Else: the inner values v = scale D x of all rows, then the shared product with U v
// added to its accumulators; a gate's few columns do all of that in one launch.
//
// v stays in fp32 quality up to the second product: bf16 calls hand it over in three bf16 values
// that add up to it (8 + 8 + 8 bits), each multiplied by U on its own.  Infinities on either side come out as in fp32:
// see split3() and without_infinities().
#include <algorithm>

#include "../../include/laser.h"
#include "grouped.h"

namespace laser {

constexpr int kMostSlices = 8, kThinWaves = 4;

struct ProjectArgs {
  const unsigned char* x;  // [T, K]
  const unsigned char* w;  // [N, K]
  const unsigned char* a_down;  // [M, R, K]
  const unsigned char* a_up;    // [M, N, R]
  const float* scales;     // [M] or NULL
  const int32_t* request_offsets;
  const int32_t* request_adapters;
  void* out;               // [T, N]
  void* inner;             // v: [T, 3, R] bf16 or [T, R] fp32
  float* parts;            // sums of slices: v, not scaled, [slices, T, R] ...
  float* shared;           // ... and W x, [slices, T, N]
  int32_t* adapter;        // [T] the row's adapter, or -1
  int T, N, M, R, requests;
  int K;                   // bytes of a row of x, w and a_down
  int lanes;               // workgroups that share the distinct adapters of 16 rows
  int slices;              // parts of the contraction axis
  bool in_parts;           // v is left in sums of slices
};

// How many of request_offsets[0 .. requests - 1] are <= t; the same t in all lanes.
__device__ __forceinline__ int requests_begun(const ProjectArgs& a, int t, int lane) {
  int lo = 0, len = a.requests;
  while (len > 64) {  // 64 probes at a time
    const int gap = (len + 63) >> 6, at = lane * gap;
    const int below = __popcll(__ballot(at < len && a.request_offsets[lo + min(at, len - 1)] <= t));
    if (below == 0) return lo;
    lo += (below - 1) * gap + 1;
    len = min(gap - 1, len - (below - 1) * gap - 1);
  }
  return lo + __popcll(__ballot(lane < len && a.request_offsets[lo + min(lane, max(len - 1, 0))] <= t));
}

// The adapter of row t0 + lane % ROWS, or -1.  A row belongs to the last request that begins at or
// before it, if that one has not ended.
template <int ROWS>
__device__ __forceinline__ int adapter_of_row(const ProjectArgs& a, int t0, int lane) {
  const int own = lane & (ROWS - 1), t = t0 + own;
  // 64 requests at a time, from the one that row t0 may belong to
  int m = -1;
  for (int at = a.requests <= 64 ? 0 : max(requests_begun(a, t0, lane) - 1, 0); at < a.requests; at += 64) {
    const bool is = at + lane < a.requests;
    const int q = is ? at + lane : 0;
    const int begin = a.request_offsets[q], end = a.request_offsets[q + 1], adapter = a.request_adapters[q];
    int n = 0;  // of these, how many begin at or before this lane's row
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int c = __popcll(__ballot(is && begin <= t0 + i));
      if (own == i) n = c;
    }
    const int last = max(n - 1, 0), its_end = __shfl(end, last), its_adapter = __shfl(adapter, last);
    if (n > 0) m = t < its_end ? its_adapter : -1;
    if (__ballot(is && begin <= t0 + ROWS - 1) != ~0ull) break;
  }
  return t < a.T && (unsigned)m < (unsigned)a.M ? m : -1;
}

// acc[b] += rows (16 b + lane % 16) of `rows` times the 16 token rows, columns of k-steps (64
// bytes) from `begin` to `end`.  Operands go memory -> registers, a batch of steps at a time.
// Pieces behind the rows' end are zero in both operands: what lies there may be anything.
constexpr int kThinBatch = 4;
__device__ __forceinline__ mma_u32x4 thin_piece(const unsigned char* row, int bytes, int k, int end, int lane) {
  const int at = k * 64 + (lane >> 4) * 16;
  const bool in = k < end && at < bytes;
  const mma_u32x4 x = *reinterpret_cast<const mma_u32x4*>(row + (in ? at : 0));
  return in ? x : mma_u32x4{0, 0, 0, 0};
}
// The first batch of the token rows, for a caller that has something else to wait for meanwhile.
struct ThinTokens {
  mma_u32x4 t[kThinBatch];
  __device__ ThinTokens(const unsigned char* tokens, int bytes, int begin, int end, int lane) {
#pragma unroll
    for (int i = 0; i < kThinBatch; ++i) t[i] = thin_piece(tokens, bytes, begin + i, end, lane);
  }
};
template <bool F32, int B>
__device__ __forceinline__ void thin_product(const ThinTokens& head, const unsigned char* tokens,
                                             const unsigned char* const (&rows)[B], int bytes, int begin, int end, int lane,
                                             mma_f32x4 (&acc)[B]) {
  constexpr int kBatch = B <= 4 ? kThinBatch : 2;
  for (int k = begin; k < end; k += kBatch) {
    mma_u32x4 t[kBatch], r[kBatch][B];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      t[i] = k == begin ? head.t[i] : thin_piece(tokens, bytes, k + i, end, lane);
#pragma unroll
      for (int b = 0; b < B; ++b) r[i][b] = thin_piece(rows[b], bytes, k + i, end, lane);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
#pragma unroll
      for (int b = 0; b < B; ++b) acc[b] = multiply<F32>(r[i][b], t[i], acc[b]);
  }
}

// The wavefronts' sums of B blocks, added in their order; value i of a lane is row
// 4 (lane / 16) + i, token lane % 16.
template <int B, typename USE>
__device__ __forceinline__ void join_wavefronts(mma_f32x4 (&acc)[B], float* part, int wave, int lane, USE use) {
#pragma unroll
  for (int b = 0; b < B; ++b) *reinterpret_cast<mma_f32x4*>(part + ((b * kThinWaves + wave) * 64 + lane) * 4) = acc[b];
  __syncthreads();
  for (int b = wave; b < B; b += kThinWaves) {
    mma_f32x4 sum = *reinterpret_cast<const mma_f32x4*>(part + (b * kThinWaves * 64 + lane) * 4);
#pragma unroll
    for (int w = 1; w < kThinWaves; ++w) sum += *reinterpret_cast<const mma_f32x4*>(part + ((b * kThinWaves + w) * 64 + lane) * 4);
    use(b, sum);
  }
  __syncthreads();
}

// x = hi + mid + lo, three bf16 values.  Bits are cut off, not rounded: what is above the largest bf16 stays
// finite.  An infinity or NaN (a quiet one, as x comes from a product) is hi alone.
__device__ __forceinline__ void split3(float x, unsigned (&piece)[3]) {
  const bool finite = fabsf(x) < __builtin_inff();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    piece[i] = __builtin_bit_cast(unsigned, x) >> 16;
    x -= bf16_value(piece[i]);
    if (i == 0) x = finite ? x : 0.0f;
  }
}

// An infinite entry of U is multiplied with hi alone: mid and lo of a finite inner value may be zero, and that times an
// infinity would be NaN.  Whether any of eight bf16 values is infinite or NaN: an exponent of ones carries.
__device__ __forceinline__ unsigned no_number(mma_u32x4 u) {
  unsigned any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= (u[i] & 0x7f807f80u) + 0x00800080u;
  return any & 0x80008000u;
}
__device__ __forceinline__ mma_u32x4 without_infinities(mma_u32x4 u) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((u[i] & 0x7fffu) == 0x7f80u) u[i] &= 0xffff0000u;
    if ((u[i] & 0x7fff0000u) == 0x7f800000u) u[i] &= 0xffffu;
  }
  return u;
}

// v[t, r .. r + 3] as the second product reads it
template <bool F32>
__device__ __forceinline__ void put_inner(const ProjectArgs& a, int t, int r, mma_f32x4 v) {
  if constexpr (F32) {
    store4<true>(a.inner, (size_t)t * a.R + r, v);
  } else {
    unsigned p[4][3];
#pragma unroll
    for (int i = 0; i < 4; ++i) split3(v[i], p[i]);
#pragma unroll
    for (int j = 0; j < 3; ++j)
      *reinterpret_cast<mma_u32x2*>(static_cast<unsigned short*>(a.inner) + ((size_t)t * 3 + j) * a.R + r) =
          mma_u32x2{p[0][j] | p[1][j] << 16, p[2][j] | p[3][j] << 16};
  }
}

// Thin calls.  Workgroup (x, y, z): 16 rows, every lanes-th of their distinct adapters from y on, slice z
// of the contraction axis, cut over the wavefronts; behind the first `lanes` y the shared
// projection, 16 columns each.
template <bool F32, int B>
__global__ __launch_bounds__(64 * kThinWaves) void adapter_thin_kernel(ProjectArgs a) {
  __shared__ __align__(16) float part[B * kThinWaves * 256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x * 16, t = t0 + (lane & 15);
  const int steps = (a.K + 63) >> 6, parts = kThinWaves * a.slices, own = kThinWaves * (int)blockIdx.z + wave;
  const int begin = (int)((long long)steps * own / parts), end = (int)((long long)steps * (own + 1) / parts);
  const unsigned char* const tokens = a.x + (size_t)min(t, a.T - 1) * a.K;
  const ThinTokens head(tokens, a.K, begin, end, lane);
  if ((int)blockIdx.y >= a.lanes) {
    const int n0 = (blockIdx.y - a.lanes) * 16;
    const unsigned char* rows[1] = {a.w + (size_t)min(n0 + (lane & 15), a.N - 1) * a.K};
    mma_f32x4 acc[1] = {mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
    thin_product<F32, 1>(head, tokens, rows, a.K, begin, end, lane, acc);
    join_wavefronts<1>(acc, part, wave, lane, [&](int, mma_f32x4 sum) {
      if (t >= a.T) return;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + 4 * (lane >> 4) + i;
        if (n < a.N) a.shared[((size_t)blockIdx.z * a.T + t) * a.N + n] = sum[i];
      }
    });
    return;
  }
  const int m = adapter_of_row<16>(a, t0, lane);
  if (blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < 16 && t < a.T) a.adapter[t] = m;
  unsigned todo = (unsigned)__ballot(m >= 0) & 0xffffu;
  for (int nth = 0; todo != 0; ++nth) {
    const int ad = __builtin_amdgcn_readlane(m, __builtin_ctz(todo));
    const bool mine = m == ad;
    todo &= ~(unsigned)__ballot(mine);
    if (nth % a.lanes != (int)blockIdx.y) continue;
    const unsigned char* rows[B];
#pragma unroll
    for (int b = 0; b < B; ++b) rows[b] = a.a_down + ((size_t)ad * a.R + min(b * 16 + (lane & 15), a.R - 1)) * a.K;
    mma_f32x4 acc[B];
#pragma unroll
    for (int b = 0; b < B; ++b) acc[b] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    thin_product<F32, B>(head, tokens, rows, a.K, begin, end, lane, acc);
    join_wavefronts<B>(acc, part, wave, lane, [&](int b, mma_f32x4 sum) {
      const int r = b * 16 + 4 * (lane >> 4);
      if (mine && r < a.R) store4<true>(a.parts, ((size_t)blockIdx.z * a.T + t) * a.R + r, sum);  // (R: a multiple of 4)
    });
  }
}

// The second launch of calls in slices: one workgroup per row and as many columns as it has threads.  All
// that does not wait for another load is under way at once: the slices, the first 16 values of
// the column's row of U.
template <bool F32, bool OUT32>
__global__ __launch_bounds__(256) void adapter_join_kernel(ProjectArgs a) {
  __shared__ float v[LASER_MAX_RANK];
  const int t = blockIdx.x, n = blockIdx.y * blockDim.x + threadIdx.x, column = min(n, a.N - 1);
  const int m = a.adapter[t];
  float part[kMostSlices];
#pragma unroll
  for (int s = 0; s < kMostSlices; ++s)
    part[s] = s < a.slices ? a.shared[((size_t)s * a.T + t) * a.N + column] : 0.0f;
  float y = 0.0f;
#pragma unroll
  for (int s = 0; s < kMostSlices; ++s) y += part[s];
  if (m >= 0) {  // (the same for the whole workgroup)
    const size_t row = ((size_t)m * a.N + column) * a.R;
    mma_f32x4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = load4<F32>(a.a_up, row + min(4 * i, a.R - 4));
    for (int r = threadIdx.x; r < a.R; r += blockDim.x) {
#pragma unroll
      for (int s = 0; s < kMostSlices; ++s)
        part[s] = s < a.slices ? a.parts[((size_t)s * a.T + t) * a.R + r] : 0.0f;
      float sum = 0.0f;
#pragma unroll
      for (int s = 0; s < kMostSlices; ++s) sum += part[s];
      v[r] = sum * (a.scales != nullptr ? a.scales[m] : 1.0f);
    }
    __syncthreads();
    float d = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * j < a.R)
#pragma unroll
        for (int i = 0; i < 4; ++i) d = fmaf(u[j][i], v[4 * j + i], d);
    for (int r = 16; r < a.R; r += 4) {
      const mma_f32x4 more = load4<F32>(a.a_up, row + r);
#pragma unroll
      for (int i = 0; i < 4; ++i) d = fmaf(more[i], v[r + i], d);
    }
    y += d;
  }
  if (n >= a.N) return;
  const size_t at = (size_t)t * a.N + n;
  if constexpr (OUT32) static_cast<float*>(a.out)[at] = y;
  else static_cast<unsigned short*>(a.out)[at] = (unsigned short)bf16_bits(y);
}

// Many rows: tiles of 64 rows against 128 rows of inner matrices at a time, the first adapters that
// the 64 rows have, then the next, through LDS (blockIdx.z: every lanes-th of those passes; behind them
// the shared projection's columns).  blockIdx.y: slice of the contraction axis where there are not
// tiles enough for all compute units; then sums of slices, joined below.
// (4096 rows, H = 4096, rank 64: 16 rows per workgroup, as thin calls do, read the matrices four times
// as often and not by whole lines; 41 us, 22 this way.)
template <bool F32, int RB>
__global__ __launch_bounds__(512) void adapter_tiles_kernel(ProjectArgs a) {
  using TL = Tile<F32, 64, 128, 4, 2, 3>;
  constexpr int kRoom = 8 / RB;
  extern __shared__ __align__(1024) unsigned char ring[];
  int* const ids = reinterpret_cast<int*>(ring + TL::kLdsBytes);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (slices of whole steps)
  const int steps = (a.K + kStepBytes - 1) / kStepBytes, slice = blockIdx.y;
  const int begin = (int)((long long)steps * slice / a.slices) * kStepBytes;
  const int end = min((int)((long long)steps * (slice + 1) / a.slices) * kStepBytes, a.K);
  TL tile(end - begin, (unsigned)(size_t)(lds_bytes)ring, wave, lane);
  const int tok = lane & 15, quad = lane >> 4, wm = wave % 4, wn = wave / 4;
  const int t0 = blockIdx.x * 64;
  const bool shared = (int)blockIdx.z >= a.lanes;  // rows of W instead of adapters'
  const int n0 = ((int)blockIdx.z - a.lanes) * 128;
  int id = -1, m = -1;
  if (!shared) {
    if (wn == 0) {
      m = adapter_of_row<16>(a, t0 + wm * 16, lane);
      const int t = t0 + wm * 16 + lane;
      if (lane < 16) {
        ids[wm * 16 + lane] = m;
        if (t < a.T && slice == 0 && blockIdx.z == 0) a.adapter[t] = m;
      }
    }
    lds_barrier();
    id = ids[lane];
    m = ids[wm * 16 + tok];
  }
  const int t = t0 + wm * 16 + tok;
  unsigned long long todo = shared ? 1 : __ballot(id >= 0);
  const unsigned char* from[TL::kLoads];
  for (int pass = 0; todo != 0; ++pass) {
    int held[kRoom];
#pragma unroll
    for (int q = 0; q < kRoom; ++q) {
      held[q] = -1;
      if (todo != 0 && !shared) {
        held[q] = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        todo &= ~__ballot(id == held[q]);
      }
    }
    if (shared) todo = 0;
    else if (pass % a.lanes != (int)blockIdx.z) continue;
    tile.turn_to(blockIdx.x + blockIdx.z);
    const int piece = TL::piece(wave, lane) * 16 + tile.turn * kStepBytes + begin;
#pragma unroll
    for (int i = 0; i < TL::kLoads; ++i) {
      const int r = TL::row(wave, lane, i);
      if (r < 64) {
        from[i] = a.x + (size_t)min(t0 + r, a.T - 1) * a.K + piece;
      } else if (shared) {
        from[i] = a.w + (size_t)min(n0 + r - 64, a.N - 1) * a.K + piece;
      } else {
        const int x = r - 64, which = x / (16 * RB);  // (the same for all lanes of a load instruction)
        int ad = -1;
#pragma unroll
        for (int q = 0; q < kRoom; ++q) ad = which == q ? held[q] : ad;
        if (ad < 0) ad = held[0];
        from[i] = a.a_down + ((size_t)ad * a.R + min(x % (16 * RB), a.R - 1)) * a.K + piece;
      }
    }
    mma_f32x4 acc[4][1];
#pragma unroll
    for (int n = 0; n < 4; ++n) acc[n][0] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    tile.start(from);
    tile.run(from, 1, acc);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int block = wn * 4 + n;
      if (shared) {
        const int c = n0 + block * 16 + 4 * quad;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t < a.T && c + i < a.N) a.shared[((size_t)slice * a.T + t) * a.N + c + i] = acc[n][0][i];
        continue;
      }
      const int r = block % RB * 16 + 4 * quad;
      int ad = -1;
#pragma unroll
      for (int q = 0; q < kRoom; ++q) ad = block / RB == q ? held[q] : ad;
      if (ad < 0 || m != ad || r >= a.R) continue;
      if (a.in_parts)
        store4<true>(a.parts, ((size_t)slice * a.T + t) * a.R + r, acc[n][0]);
      else
        put_inner<F32>(a, t, r, acc[n][0] * (a.scales != nullptr ? a.scales[ad] : 1.0f));
    }
  }
}

// The slices' sums of the rows that have an adapter.
template <bool F32>
__global__ __launch_bounds__(256) void adapter_slices_kernel(ProjectArgs a) {
  const int quads = a.R >> 2;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, t = i / quads;
  if (t >= a.T) return;
  const int m = a.adapter[t], r = (int)(i - t * quads) * 4;
  if (m < 0) return;
  mma_f32x4 part[kMostSlices];
#pragma unroll
  for (int s = 0; s < kMostSlices; ++s)
    part[s] = s < a.slices ? *reinterpret_cast<const mma_f32x4*>(a.parts + ((size_t)s * a.T + t) * a.R + r)
                           : mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  mma_f32x4 sum = part[0];
#pragma unroll
  for (int s = 1; s < kMostSlices; ++s) sum += part[s];
  put_inner<F32>(a, (int)t, r, sum * (a.scales != nullptr ? a.scales[m] : 1.0f));
}

// U v added to a wavefront's accumulators: per block of 16 tokens and distinct adapter in it, 32
// values of v at a time (fp32: 16), the rows of other adapters as zeros.
template <bool F32, class TL>
__device__ __forceinline__ void add_adapters(const ProjectArgs& a, int t0, int n0, int blocks, int wave, int lane,
                                             mma_f32x4 (&acc)[TL::NB][TL::MB]) {
  constexpr int NB = TL::NB, MB = TL::MB, kPieces = F32 ? 1 : 3;
  constexpr int kSize = F32 ? 4 : 2, kOwn = 16 / kSize;  // values of v that a lane holds at a time
  constexpr int kAhead = MB <= 4 ? MB : 2;  // (registers)
  int ids[MB];
  bool any = false;
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    const int t = t0 + TL::block_row(wave, m) + (lane & 15);
    ids[m] = t < a.T ? a.adapter[t] : -1;
    any |= ids[m] >= 0;
  }
  if (__ballot(any) == 0) return;
  for (int r0 = 0; r0 < a.R; r0 += 4 * kOwn) {
    const int r = r0 + (lane >> 4) * kOwn;
    const bool in = r < a.R;
    int held = -1;  // the adapter whose rows are in u
    bool limits = false;  // ... and whether these hold infinities or NaN (bf16)
    mma_u32x4 u[NB], ahead[kAhead][kPieces];
    auto load_u = [&](int ad) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int row = min(n0 + n * 16 + (lane & 15), a.N - 1);
        u[n] = *reinterpret_cast<const mma_u32x4*>(a.a_up + (((size_t)ad * a.N + row) * a.R + (in ? r : 0)) * kSize);
        if (!in) u[n] = mma_u32x4{0, 0, 0, 0};
      }
    };
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      if (m % kAhead == 0) {  // v of the next blocks, all under way at once
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int t = min(t0 + TL::block_row(wave, min(m + k, MB - 1)) + (lane & 15), a.T - 1);
#pragma unroll
          for (int j = 0; j < kPieces; ++j)
            ahead[k][j] = *reinterpret_cast<const mma_u32x4*>(static_cast<const unsigned char*>(a.inner) +
                                                              (((size_t)t * kPieces + j) * a.R + (in ? r : 0)) * kSize);
        }
      }
      unsigned todo = (unsigned)__ballot(ids[m] >= 0) & 0xffffu;
      if (todo == 0) continue;
      mma_u32x4 (&v)[kPieces] = ahead[m % kAhead];
      while (todo != 0) {
        const int ad = __builtin_amdgcn_readlane(ids[m], __builtin_ctz(todo));
        const bool mine = ids[m] == ad;
        todo &= ~(unsigned)__ballot(mine);
        if (ad != held) {
          held = ad;
          load_u(ad);
          if constexpr (!F32) {
            unsigned any = 0;
#pragma unroll
            for (int n = 0; n < NB; ++n) any |= no_number(u[n]);
            limits = __ballot(any != 0) != 0;
          }
        }
        mma_f32x4 d[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) d[n] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (!F32 && limits)
#pragma unroll
          for (int n = 0; n < NB; ++n) u[n] = without_infinities(u[n]);
#pragma unroll
        for (int j = kPieces - 1; j >= 0; --j) {
          if (!F32 && j == 0 && limits) {  // (loaded again: a second set of registers would spill)
            asm volatile("" ::: "memory");
            load_u(ad);
          }
          const mma_u32x4 b = mine && in ? v[j] : mma_u32x4{0, 0, 0, 0};
#pragma unroll
          for (int n = 0; n < NB; ++n) d[n] = multiply<F32>(u[n], b, d[n]);
        }
        // (not added to rows of other adapters: a zero times an infinity in u is no zero)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[n][m][i] += mine ? d[n][i] : 0.0f;
      }
    }
  }
}

// A wavefront's results (NC blocks of columns from n0 on) to out: whole 16-byte pieces where the
// rows of out consist of them, values one by one where they do not.
template <bool OUT32, class TL, int NC>
__device__ __forceinline__ void store_columns(const ProjectArgs& a, unsigned lds, int wave, int lane, int t0, int rows, int n0,
                                              mma_f32x4 (&y)[NC][TL::MB]) {
  constexpr int kSize = OUT32 ? 4 : 2;
  if (a.N % (16 / kSize) == 0) {
    store_tile<OUT32, TL, NC>(
        lds, wave, lane, [&](int n, int m) { return y[n][m]; },
        [&](int r, int c) -> void* {
          return r < rows && n0 + c < a.N ? static_cast<char*>(a.out) + ((size_t)(t0 + r) * a.N + n0 + c) * kSize : nullptr;
        });
    return;
  }
#pragma unroll
  for (int m = 0; m < TL::MB; ++m) {
    const int r = TL::block_row(wave, m) + (lane & 15);
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = n0 + n * 16 + 4 * (lane >> 4) + i;
        if (r >= rows || c >= a.N) continue;
        const size_t at = (size_t)(t0 + r) * a.N + c;
        if constexpr (OUT32) static_cast<float*>(a.out)[at] = y[n][m][i];
        else static_cast<unsigned short*>(a.out)[at] = (unsigned short)bf16_bits(y[n][m][i]);
      }
  }
}

template <bool F32, bool OUT32, class TL>
__global__ __launch_bounds__(TL::kThreads) void project_kernel(ProjectArgs a) {
  extern __shared__ __align__(1024) unsigned char ring[];
  const unsigned lds = (unsigned)(size_t)(lds_bytes)ring;
  constexpr int BM = TL::BM, BN = TL::BN, NB = TL::NB, MB = TL::MB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nt = (a.N + BN - 1) / BN, mt = (a.T + BM - 1) / BM, total = mt * nt;
  const int wn = wave / TL::WM;
  TL tile(a.K, lds, wave, lane);
  for (int v = blockIdx.x; v < total; v += gridDim.x) {
    const int id = xcd_run(v, total);
    constexpr int kGroup = 8;
    const int g = id / (kGroup * nt), gm = min(kGroup, mt - g * kGroup), in = id - g * kGroup * nt;
    const int t0 = (g * kGroup + in % gm) * BM, n0 = in / gm * BN + wn * (BN / TL::WN);
    const unsigned char* from[TL::kLoads];
    // (an XCD's tiles share rows while they are at the same step: 8192 x 4096 x 4096 of rank 16 248 us, 260 with
    // a turn for every tile)
    tile.turn_to(v & 7);
    const int piece = TL::piece(wave, lane) * 16 + tile.turn * kStepBytes;
#pragma unroll
    for (int i = 0; i < TL::kLoads; ++i) {
      const int r = TL::row(wave, lane, i);
      from[i] = (r < BM ? a.x + (size_t)min(t0 + r, a.T - 1) * a.K
                        : a.w + (size_t)min(in / gm * BN + r - BM, a.N - 1) * a.K) + piece;
    }
    mma_f32x4 acc[NB][MB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int m = 0; m < MB; ++m) acc[n][m] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int rows = min(a.T - t0, BM), blocks = TL::blocks_of(wave, rows);
    tile.start(from);
    tile.run(from, blocks, acc);
    int l = lane;
    asm volatile("" : "+v"(l));
    add_adapters<F32, TL>(a, t0, n0, blocks, wave, l, acc);
    store_columns<OUT32, TL, NB>(a, lds, wave, l, t0, rows, n0, acc);
    lds_barrier();  // (the ring is free again)
  }
}

// Up to 64 columns (a gate) and adapters of rank up to 64: one launch that reads x once.  The
// weight rows of a tile are W's and behind them 64 rows of inner matrices, of the first adapters
// that its 64 rows have.  For the second product each of four wavefronts has 16 rows, all columns and their v,
// whose accumulator layout (row 4 (lane / 16) + i) serves as the operand as it is: which
// slot of a matrix instruction is which r is free, as long as U's rows are read the same way.
// A tile with more adapters makes another pass over its rows for every 128 rows of them.
// (16384 rows, H = 2048, 64 columns, rank 16: 22 us against 50 with a launch of its own for v, which
// reads x a second time; reading x alone takes 13 us at the rate of a large copy.  What bounds it is the time of
// a step, half a microsecond: 24 KiB to LDS, 48 KiB read there, a barrier.  With 80 KiB read, 16 rows and whole
// steps per wavefront, 23.)
constexpr int kNarrowColumns = 64, kNarrowRank = 64;
template <bool F32, bool OUT32, int RB>  // RB: blocks of 16 that hold an adapter's rows
__global__ __launch_bounds__(512) void project_narrow_kernel(ProjectArgs a) {
  using TL = Tile<F32, 64, 128, 4, 2, 6, kTokens>;
  constexpr int kRoom = 4 / RB;  // adapters beside W, twice that without
  extern __shared__ __align__(1024) unsigned char ring[];
  int* const ids = reinterpret_cast<int*>(ring + TL::kLdsBytes);
  const unsigned lds = (unsigned)(size_t)(lds_bytes)ring;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TL tile(a.K, lds, wave, lane);
  const int tok = lane & 15, quad = lane >> 4, wm = wave % 4, wn = wave / 4;
  const int tiles = (a.T + 63) >> 6;
  for (int v = blockIdx.x; v < tiles; v += gridDim.x) {
    const int t0 = xcd_run(v, tiles) * 64, rows = min(a.T - t0, 64);
    if (wn == 0) {
      const int m = adapter_of_row<16>(a, t0 + wm * 16, lane);
      if (lane < 16) ids[wm * 16 + lane] = m;
    }
    lds_barrier();
    const int id = ids[lane], m = ids[wm * 16 + tok];  // of row t0 + lane; of this lane's token
    unsigned long long todo = __ballot(id >= 0);
    const unsigned char* from[TL::kLoads];
    mma_f32x4 y[4][1];  // the tile's results (wavefronts 0 .. 3)
    for (bool first = true; first || todo != 0; first = false) {
      // the adapters of this pass, in order; rows of inner matrices that are not needed repeat others
      int held[2 * kRoom];
#pragma unroll
      for (int q = 0; q < 2 * kRoom; ++q) {
        held[q] = -1;
        if (todo != 0 && (q < kRoom || !first)) {
          held[q] = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
          todo &= ~__ballot(id == held[q]);
        }
      }
      tile.turn_to(v);
      const int piece = TL::piece(wave, lane) * 16 + tile.turn * kStepBytes;
#pragma unroll
      for (int i = 0; i < TL::kLoads; ++i) {
        const int r = TL::row(wave, lane, i), w = r - 64;  // (rows 0 .. 63 are tokens)
        if (r < 64) {
          from[i] = a.x + (size_t)min(t0 + r, a.T - 1) * a.K + piece;
        } else if (first && w < 64) {
          from[i] = a.w + (size_t)min(w, a.N - 1) * a.K + piece;
        } else {
          const int x = first ? w - 64 : w, which = x / (16 * RB);  // (the same for all lanes of a load instruction)
          int ad = -1;
#pragma unroll
          for (int q = 0; q < 2 * kRoom; ++q) ad = which == q ? held[q] : ad;
          if (ad < 0) ad = held[0];
          from[i] = (ad < 0 ? a.w : a.a_down + ((size_t)ad * a.R + min(x % (16 * RB), a.R - 1)) * a.K) + piece;
        }
      }
      tile.start(from);
      tile.run_halves(from, lds, wave, lane);
      if (wn == 1) {
        lds_barrier();
        continue;
      }
      if (first)
#pragma unroll
        for (int n = 0; n < 4; ++n) y[n][0] = TL::half_sums(lds, wm, n, lane);
      const int inner_at = first ? 4 : 0;  // block of the pass's first inner rows
#pragma unroll
      for (int q = 0; q < 2 * kRoom; ++q) {
        if (held[q] < 0 || __ballot(m == held[q]) == 0) continue;
        const bool mine = m == held[q];
        const float scale = a.scales != nullptr ? a.scales[held[q]] : 1.0f;
        mma_f32x4 d[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) d[n] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int b = 0; b < RB; b += F32 ? 1 : 2) {
          mma_f32x4 inner[2];  // blocks b and, bf16, b + 1
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            inner[h] = TL::half_sums(lds, wm, inner_at + q * RB + min(b + h, RB - 1), lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) inner[h][i] = mine && b + h < RB ? inner[h][i] * scale : 0.0f;
          }
          const int r = 16 * b + 4 * quad;
          auto row_of = [&](int n) { return ((size_t)held[q] * a.N + min(16 * n + tok, a.N - 1)) * a.R; };
          if constexpr (F32) {
            const mma_f32x4 x = r < a.R ? inner[0] : mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              mma_f32x4 u = {0.0f, 0.0f, 0.0f, 0.0f};
              if (r < a.R) u = load4<true>(a.a_up, row_of(n) + r);
              d[n] = multiply<true>(__builtin_bit_cast(mma_u32x4, u), __builtin_bit_cast(mma_u32x4, x), d[n]);
            }
          } else {
            mma_u32x4 u[4], p[3];
            unsigned any = 0;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              const unsigned short* const up = reinterpret_cast<const unsigned short*>(a.a_up) + row_of(n);
              u[n] = mma_u32x4{0, 0, 0, 0};
              if (r < a.R) {
                const mma_u32x2 lo = *reinterpret_cast<const mma_u32x2*>(up + r);
                u[n][0] = lo[0], u[n][1] = lo[1];
              }
              if (b + 1 < RB && r + 16 < a.R) {
                const mma_u32x2 hi = *reinterpret_cast<const mma_u32x2*>(up + r + 16);
                u[n][2] = hi[0], u[n][3] = hi[1];
              }
              any |= no_number(u[n]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const bool in = r + 16 * h < a.R;  // (rows past the rank repeat the last one: not used)
              unsigned s[4][3];
#pragma unroll
              for (int i = 0; i < 4; ++i) split3(in ? inner[h][i] : 0.0f, s[i]);
#pragma unroll
              for (int j = 0; j < 3; ++j) {
                p[j][2 * h] = s[0][j] | s[1][j] << 16;
                p[j][2 * h + 1] = s[2][j] | s[3][j] << 16;
              }
            }
            const bool limits = __ballot(any != 0) != 0;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              mma_u32x4 rest = u[n];
              if (limits) rest = without_infinities(rest);
              d[n] = multiply<false>(rest, p[2], d[n]);
              d[n] = multiply<false>(rest, p[1], d[n]);
              d[n] = multiply<false>(u[n], p[0], d[n]);
            }
          }
        }
        // (not added to rows of other adapters: a zero times an infinity in u is no zero)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) y[n][0][i] += mine ? d[n][i] : 0.0f;
      }
      lds_barrier();
    }
    if (wn == 0) store_columns<OUT32, TL, 4>(a, lds, wave, lane, t0, rows, 0, y);
    lds_barrier();  // (the ring and the ids are free again)
  }
}

// ---- host ---------------------------------------------------------------------------

// Which way a call goes (launch_project), and what it keeps in the workspace.
constexpr int kThinRows = 512, kThinValues = 1 << 16;
static bool is_thin(int T, int N) { return T <= kThinRows && (long long)T * N <= kThinValues; }
// slices so that `units` tiles become about as many workgroups as there are compute units
constexpr int kWorkgroups = 256, kSliceWorkgroups = 512;
static int slices_for(long long units, int K, int workgroups) {
  const int steps = (K + kStepBytes - 1) / kStepBytes;
  return (int)std::max<long long>(1, std::min<long long>({kMostSlices, workgroups / units, steps}));
}

static size_t whole(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
struct ProjectLayout {
  size_t adapter, inner, parts, shared, total;
};
// (each part grows with T.  Rows times slices, and values of out times slices, are at most those of kSliceWorkgroups
// tiles of 64 rows and of 64 x 128)
static ProjectLayout project_layout(int T, int N, const laser_adapter_params_t* p) {
  ProjectLayout L;
  L.adapter = 0;
  L.inner = whole((size_t)T * 4);
  L.parts = L.inner + whole((size_t)T * p->rank * (p->dtype == LASER_DTYPE_F32 ? 4 : 6));
  L.shared = L.parts + whole(std::min<size_t>((size_t)T * kMostSlices, kSliceWorkgroups * 64) * p->rank * 4);
  L.total = L.shared + whole(std::min<size_t>((size_t)T * N * kMostSlices, kSliceWorkgroups * 64 * 128) * 4) + 256;
  return L;
}

static int check_project(int32_t T, int32_t H, int32_t N, const laser_adapter_params_t* p) {
  if (!p) return LASER_E_NULL;
  if (p->struct_bytes != sizeof(laser_adapter_params_t)) return LASER_E_STRUCT;
  if (T < 0 || H < 1 || N < 1 || p->adapters < 0 || p->requests < 0) return LASER_E_RANGE;
  if (T > (1 << 27) || H > (1 << 28) || N > (1 << 28) || p->requests > (1 << 28)) return LASER_E_RANGE;
  if (p->dtype != LASER_DTYPE_F32 && p->dtype != LASER_DTYPE_BF16) return LASER_E_RANGE;
  if (p->out_dtype != LASER_DTYPE_F32 && p->out_dtype != p->dtype) return LASER_E_RANGE;
  if (p->rank < 1) return LASER_E_RANGE;
  if (p->rank > LASER_MAX_RANK) return LASER_E_UNSUPPORTED;
  const int pieces = p->dtype == LASER_DTYPE_F32 ? 4 : 8;
  if (H % pieces != 0 || p->rank % pieces != 0) return LASER_E_ALIGN;
  return LASER_OK;
}

template <bool F32>
static hipError_t launch_thin(const ProjectArgs& a, hipStream_t s) {
  const dim3 grid((a.T + 15) / 16, a.lanes + (a.N + 15) / 16, a.slices), block(64 * kThinWaves);
  auto* const kernel = a.R <= 16   ? &adapter_thin_kernel<F32, 1>
                       : a.R <= 32 ? &adapter_thin_kernel<F32, 2>
                       : a.R <= 64 ? &adapter_thin_kernel<F32, 4>
                                   : &adapter_thin_kernel<F32, 8>;
  hipLaunchKernelGGL(kernel, grid, block, 0, s, a);
  return hipGetLastError();
}

template <bool F32, bool OUT32, class TL>
static hipError_t launch_tiles(const ProjectArgs& a, hipStream_t s) {
  static LdsAttr attr;
  const void* fn = reinterpret_cast<const void*>(&project_kernel<F32, OUT32, TL>);
  hipError_t err = allow_dynamic_lds(fn, TL::kLdsBytes, attr);
  if (err != hipSuccess) return err;
  const long long grid = (long long)((a.T + TL::BM - 1) / TL::BM) * ((a.N + TL::BN - 1) / TL::BN);
  hipLaunchKernelGGL((project_kernel<F32, OUT32, TL>), dim3((unsigned)std::min(grid, 1ll << 20)), dim3(TL::kThreads),
                     TL::kLdsBytes, s, a);
  return hipGetLastError();
}

template <bool F32, int RB>
static hipError_t launch_inner_tiles(const ProjectArgs& a, int columns, hipStream_t s) {
  static LdsAttr attr;
  constexpr int kLds = Tile<F32, 64, 128, 4, 2, 3>::kLdsBytes + 64 * 4;
  const void* fn = reinterpret_cast<const void*>(&adapter_tiles_kernel<F32, RB>);
  const hipError_t err = allow_dynamic_lds(fn, kLds, attr);
  if (err != hipSuccess) return err;
  const dim3 grid((a.T + 63) / 64, a.slices, a.lanes + (columns + 127) / 128);
  hipLaunchKernelGGL((adapter_tiles_kernel<F32, RB>), grid, dim3(512), kLds, s, a);
  return hipGetLastError();
}
// (columns: of the shared projection, 0 if they are not its business)
template <bool F32>
static hipError_t launch_inner(const ProjectArgs& a, int columns, hipStream_t s) {
  return a.R <= 16   ? launch_inner_tiles<F32, 1>(a, columns, s)
         : a.R <= 32 ? launch_inner_tiles<F32, 2>(a, columns, s)
         : a.R <= 64 ? launch_inner_tiles<F32, 4>(a, columns, s)
                     : launch_inner_tiles<F32, 8>(a, columns, s);
}

template <bool F32, bool OUT32, int RB>
static hipError_t launch_narrow(const ProjectArgs& a, hipStream_t s) {
  static LdsAttr attr;
  constexpr int kLds = Tile<F32, 64, 128, 4, 2, 6>::kLdsBytes + 64 * 4;
  const void* fn = reinterpret_cast<const void*>(&project_narrow_kernel<F32, OUT32, RB>);
  hipError_t err = allow_dynamic_lds(fn, kLds, attr);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((project_narrow_kernel<F32, OUT32, RB>), dim3(std::min((a.T + 63) / 64, 1 << 20)), dim3(512), kLds, s, a);
  return hipGetLastError();
}

template <bool F32, bool OUT32>
static hipError_t launch_join(const ProjectArgs& a, hipStream_t s) {
  const int threads = a.N <= 64 ? 64 : a.N <= 128 ? 128 : 256;
  hipLaunchKernelGGL((adapter_join_kernel<F32, OUT32>), dim3(a.T, (a.N + threads - 1) / threads), dim3(threads), 0, s, a);
  return hipGetLastError();
}

template <bool F32, bool OUT32>
static hipError_t launch_project(ProjectArgs& a, hipStream_t s) {
  if (is_thin(a.T, a.N)) {
    a.slices = std::min(kMostSlices, std::max(1, (a.K + 63) / 64 / 8));
    a.lanes = std::max(1, std::min(16, a.requests));
    const hipError_t err = launch_thin<F32>(a, s);
    return err != hipSuccess ? err : launch_join<F32, OUT32>(a, s);
  }
  // (a tile's passes side by side; workgroups without one end at once.  Rank 128, 16384 rows of 40
  // requests: 143 us with one, 126 with four)
  a.lanes = std::max(1, std::min(a.requests, 4));
  const long long rows = (a.T + 63) / 64, tiles = rows * ((a.N + 127) / 128);
  // A gate in one launch, unless many requests may meet in a tile, which makes its passes one after the other.
  const bool narrow = a.N <= kNarrowColumns && a.R <= kNarrowRank && (a.requests <= 32 || a.requests <= a.T / 64);
  // Too few tiles for all compute units: all in slices, for one workgroup per compute unit or two, unless the
  // join would have more than kJoinWork products for single threads or there are few steps to cut.  (800 x 247,
  // H = 3624: 67 us in tiles, 22 in slices; 3000 x 256, H = 2048: 44, 33; 1078 x 906, H = 640: 24, 27.)  For a
  // gate's one launch a step takes half a microsecond, twice that with wide adapters, and the second launch and the
  // sums of slices 10.  (24 requests, 64 columns, one launch and slices: 2000 rows, H = 2048, rank 16 21.6, 17.4,
  // H = 1024 14.3, 15.0; 4000 rows, H = 2048, rank 16 21.9, 24.3, rank 64 50.6, 28.1)
  constexpr long long kJoinWork = 1 << 25;
  constexpr int kJoinSteps = 16, kLaunchSteps = 18;
  const int steps = (a.K + kStepBytes - 1) / kStepBytes;
  if (tiles + rows <= kSliceWorkgroups / 2 && steps >= kJoinSteps && (long long)a.T * a.N * a.R <= kJoinWork) {
    a.slices = slices_for(tiles + rows, a.K, tiles + rows <= kWorkgroups / 2 ? kWorkgroups : kSliceWorkgroups);
    if (!narrow || (long long)steps * (a.R > 16 ? 2 : 1) * (a.slices - 1) > kLaunchSteps * a.slices) {
      a.in_parts = true;
      const hipError_t err = launch_inner<F32>(a, a.N, s);
      return err != hipSuccess ? err : launch_join<F32, OUT32>(a, s);
    }
  }
  if (narrow)
    return a.R <= 16   ? launch_narrow<F32, OUT32, 1>(a, s)
           : a.R <= 32 ? launch_narrow<F32, OUT32, 2>(a, s)
                       : launch_narrow<F32, OUT32, 4>(a, s);
  a.slices = slices_for(rows, a.K, kWorkgroups);
  a.in_parts = a.slices > 1;
  hipError_t err = launch_inner<F32>(a, 0, s);
  if (err != hipSuccess) return err;
  if (a.in_parts) {
    const unsigned grid = (unsigned)(((long long)a.T * (a.R / 4) + 255) / 256);
    hipLaunchKernelGGL((adapter_slices_kernel<F32>), dim3(grid), dim3(256), 0, s, a);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  // tiles as large as leaves some for half of the compute units
  auto count = [&](int side) { return (long long)((a.T + side - 1) / side) * ((a.N + side - 1) / side); };
  if constexpr (!F32) {
    if (count(256) >= kWorkgroups / 2) return launch_tiles<F32, OUT32, Tile<F32, 256, 256, 2, 4, 2>>(a, s);
    if (count(128) >= kWorkgroups / 2) return launch_tiles<F32, OUT32, Tile<F32, 128, 128, 2, 2, 2>>(a, s);
  }
  return launch_tiles<F32, OUT32, Tile<F32, 64, 64, 1, 4, 4>>(a, s);
}

}  // namespace laser

using namespace laser;

extern "C" size_t laser_project_workspace_bytes(int32_t T, int32_t H, int32_t N, const laser_adapter_params_t* params) {
  if (check_project(T, H, N, params) != LASER_OK) return 0;
  return project_layout(T, N, params).total;
}

extern "C" int laser_project_adapted(const void* x, const void* w, int32_t T, int32_t H, int32_t N,
                                     const laser_adapter_params_t* params, const void* a_down, const void* a_up,
                                     const float* scales, const int32_t* request_offsets,
                                     const int32_t* request_adapters, void* out, void* workspace,
                                     size_t workspace_bytes, void* hip_stream) {
  const int rc = check_project(T, H, N, params);
  if (rc != LASER_OK) return rc;
  if (T == 0) return LASER_OK;
  if (!x || !w || !out || !workspace) return LASER_E_NULL;
  const int requests = params->adapters > 0 ? params->requests : 0;
  if (requests > 0 && (!a_down || !a_up || !request_offsets || !request_adapters)) return LASER_E_NULL;
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)w | (uintptr_t)a_down | (uintptr_t)a_up | (uintptr_t)out;
  if (bits & 15 || (uintptr_t)workspace & 255) return LASER_E_ALIGN;
  const ProjectLayout L = project_layout(T, N, params);
  if (workspace_bytes < L.total) return LASER_E_WORKSPACE;
  const bool f32 = params->dtype == LASER_DTYPE_F32;
  char* const ws = static_cast<char*>(workspace);
  ProjectArgs a = {};
  a.x = static_cast<const unsigned char*>(x);
  a.w = static_cast<const unsigned char*>(w);
  a.a_down = static_cast<const unsigned char*>(a_down);
  a.a_up = static_cast<const unsigned char*>(a_up);
  a.scales = scales;
  a.request_offsets = request_offsets;
  a.request_adapters = request_adapters;
  a.out = out;
  a.inner = ws + L.inner;
  a.parts = reinterpret_cast<float*>(ws + L.parts);
  a.shared = reinterpret_cast<float*>(ws + L.shared);
  a.adapter = reinterpret_cast<int32_t*>(ws + L.adapter);
  a.T = T;
  a.N = N;
  a.M = params->adapters;
  a.R = params->rank;
  a.requests = requests;
  a.K = H * (f32 ? 4 : 2);
  clear_stale_error();
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t err = f32 ? launch_project<true, true>(a, s)
                         : params->out_dtype == LASER_DTYPE_F32 ? launch_project<false, true>(a, s)
                                                                : launch_project<false, false>(a, s);
  return err == hipSuccess ? LASER_OK : LASER_E_LAUNCH;
}
