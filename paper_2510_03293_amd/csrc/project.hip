// A projection that all rows of a batch share, and beside it the low-rank adapters that the
// requests of the batch bring along: laser_project_adapted.
#include "../../include/laser.h"
#include "grouped.h"

namespace laser {

struct ProjectArgs {
  const unsigned char* x;  // [T, K]
  const unsigned char* w;  // [N, K]
  const unsigned char* a_down;  // [M, R, K]
  const unsigned char* a_up;    // [M, N, R]
  const float* scales;     // [M] or NULL
  const int32_t* request_offsets;
  const int32_t* request_adapters;
  void* out;               // [T, N]
  float* inner;            // [T, R]  scale * (A x) of the row's adapter
  int32_t* adapter;        // [T]     the row's adapter, or -1
  int T, N, M, R, requests;
  int H;
  int K;                   // bytes of a row of x, w and a_down
};

// The adapter of row t (or -1): the last request that begins at or before t, if t is still in it.
__device__ __forceinline__ int adapter_of(const ProjectArgs& a, int t) {
  int lo = 0, hi = a.requests;  // request_offsets[lo - 1] <= t < request_offsets[hi], were there one
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.request_offsets[mid] <= t) lo = mid + 1; else hi = mid;
  }
  if (lo == 0 || t >= a.request_offsets[lo]) return -1;
  const int m = a.request_adapters[lo - 1];
  return (unsigned)m < (unsigned)a.M ? m : -1;
}

// inner[t, r] = scale * sum_h A[r, h] x[t, h]: one wavefront per row.
template <bool F32>
__global__ __launch_bounds__(256) void adapter_inner_kernel(ProjectArgs a) {
  const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.T) return;
  const int m = adapter_of(a, t);
  if (lane == 0) a.adapter[t] = m;
  if (m < 0) return;
  const float scale = a.scales != nullptr ? a.scales[m] : 1.0f;
  for (int r = 0; r < a.R; ++r) {
    float sum = 0.0f;
    for (int h = lane * 4; h < a.H; h += 256) {
      const mma_f32x4 x = load4<F32>(a.x, (size_t)t * a.H + h);
      const mma_f32x4 w = load4<F32>(a.a_down, ((size_t)m * a.R + r) * a.H + h);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = fmaf(x[i], w[i], sum);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) a.inner[(size_t)t * a.R + r] = sum * scale;
  }
}

template <bool F32, bool OUT32, class TL>
__global__ __launch_bounds__(TL::kThreads) void project_kernel(ProjectArgs a) {
  extern __shared__ __align__(1024) unsigned char ring[];
  const unsigned lds = (unsigned)(size_t)(lds_bytes)ring;
  constexpr int BM = TL::BM, BN = TL::BN, NB = TL::NB, MB = TL::MB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nt = (a.N + BN - 1) / BN, total = (a.T + BM - 1) / BM * nt;
  const int wn = wave / TL::WM;
  for (int v = blockIdx.x; v < total; v += gridDim.x) {
    const int id = xcd_run(v, total);
    const int t0 = id / nt * BM, n0 = id % nt * BN;
    const unsigned char* from[TL::kLoads];
    const int piece = TL::piece(wave, lane) * 16;
#pragma unroll
    for (int i = 0; i < TL::kLoads; ++i) {
      const int r = TL::row(wave, lane, i);
      from[i] = (r < BM ? a.x + (size_t)min(t0 + r, a.T - 1) * a.K : a.w + (size_t)min(n0 + r - BM, a.N - 1) * a.K) + piece;
    }
    mma_f32x4 acc[NB][MB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int m = 0; m < MB; ++m) acc[n][m] = mma_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const TL tile(a.K, lds, wave, lane);
    tile.start(from);
    tile.run(from, TL::blocks_of(wave, a.T - t0), acc);
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const int t = t0 + TL::block_row(wave, m) + (lane & 15);
      if (t >= a.T) continue;
      const int ad = a.adapter[t];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int c = n0 + wn * (BN / TL::WN) + n * 16 + 4 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (c + i >= a.N) continue;
          float y = 0.0f;
          if (ad >= 0) {
            const size_t row = ((size_t)ad * a.N + c + i) * a.R;
            for (int r = 0; r < a.R; r += 4) {
              const mma_f32x4 b = load4<F32>(a.a_up, row + r);
#pragma unroll
              for (int j = 0; j < 4; ++j) y = fmaf(b[j], a.inner[(size_t)t * a.R + r + j], y);
            }
          }
          y += acc[n][m][i];
          const size_t at = (size_t)t * a.N + c + i;
          if constexpr (OUT32) static_cast<float*>(a.out)[at] = y;
          else static_cast<unsigned short*>(a.out)[at] = (unsigned short)bf16_bits(y);
        }
      }
    }
  }
}

static size_t inner_bytes(int32_t T, const laser_adapter_params_t* p) { return ((size_t)T * p->rank * 4 + 255) & ~(size_t)255; }

static int check_project(int32_t T, int32_t H, int32_t N, const laser_adapter_params_t* p) {
  if (!p) return LASER_E_NULL;
  if (p->struct_bytes != sizeof(laser_adapter_params_t)) return LASER_E_STRUCT;
  if (T < 0 || H < 1 || N < 1 || p->adapters < 0 || p->requests < 0) return LASER_E_RANGE;
  if (T > (1 << 30) || H > (1 << 28) || N > (1 << 28)) return LASER_E_RANGE;
  if (p->dtype != LASER_DTYPE_F32 && p->dtype != LASER_DTYPE_BF16) return LASER_E_RANGE;
  if (p->out_dtype != LASER_DTYPE_F32 && p->out_dtype != p->dtype) return LASER_E_RANGE;
  if (p->rank < 1) return LASER_E_RANGE;
  if (p->rank > LASER_MAX_RANK) return LASER_E_UNSUPPORTED;
  const int whole = p->dtype == LASER_DTYPE_F32 ? 4 : 8;
  if (H % whole != 0 || p->rank % whole != 0) return LASER_E_ALIGN;
  return LASER_OK;
}

template <bool F32, bool OUT32>
static hipError_t launch_project(const ProjectArgs& a, hipStream_t s) {
  using TL = Tile<F32, 64, 64, 1, 4, 3>;
  static LdsAttr attr;
  const void* fn = reinterpret_cast<const void*>(&project_kernel<F32, OUT32, TL>);
  hipError_t err = allow_dynamic_lds(fn, TL::kLdsBytes, attr);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((adapter_inner_kernel<F32>), dim3((a.T + 3) / 4), dim3(256), 0, s, a);
  err = hipGetLastError();
  if (err != hipSuccess) return err;
  const long long grid = (long long)((a.T + TL::BM - 1) / TL::BM) * ((a.N + TL::BN - 1) / TL::BN);
  hipLaunchKernelGGL((project_kernel<F32, OUT32, TL>), dim3((unsigned)min(grid, 1ll << 20)), dim3(TL::kThreads),
                     TL::kLdsBytes, s, a);
  return hipGetLastError();
}

}  // namespace laser

using namespace laser;

extern "C" size_t laser_project_workspace_bytes(int32_t T, int32_t H, int32_t N, const laser_adapter_params_t* params) {
  if (check_project(T, H, N, params) != LASER_OK) return 0;
  return inner_bytes(T, params) + (((size_t)T * 4 + 256) & ~(size_t)255);
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
  if (workspace_bytes < laser_project_workspace_bytes(T, H, N, params)) return LASER_E_WORKSPACE;
  const bool f32 = params->dtype == LASER_DTYPE_F32;
  ProjectArgs a = {};
  a.x = static_cast<const unsigned char*>(x);
  a.w = static_cast<const unsigned char*>(w);
  a.a_down = static_cast<const unsigned char*>(a_down);
  a.a_up = static_cast<const unsigned char*>(a_up);
  a.scales = scales;
  a.request_offsets = request_offsets;
  a.request_adapters = request_adapters;
  a.out = out;
  a.inner = static_cast<float*>(workspace);
  a.adapter = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + inner_bytes(T, params));
  a.T = T;
  a.N = N;
  a.M = params->adapters;
  a.R = params->rank;
  a.requests = requests;
  a.H = H;
  a.K = H * (f32 ? 4 : 2);
  clear_stale_error();
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t err = f32 ? launch_project<true, true>(a, s)
                         : params->out_dtype == LASER_DTYPE_F32 ? launch_project<false, true>(a, s)
                                                                : launch_project<false, false>(a, s);
  return err == hipSuccess ? LASER_OK : LASER_E_LAUNCH;
}
