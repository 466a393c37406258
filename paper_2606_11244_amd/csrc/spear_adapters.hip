// gfx950 (MI355X) kernels of the low-rank adapters of many requests: the term
//   d[m] = res[m] + s_a B_a (A_a x[m]),   a = ids[m] (d[m] = res[m] without one)
// that the 4-bit product's final store adds in place of a residual. fp32 sums.
#include "spear_device.h"

namespace spear {

// rank of token m's adapter (0: it has none), with its slot in *slot
__device__ __forceinline__ int adapter_of(const AdapterParams& p, int m, int* slot) {
  const int a = p.ids[m];
  *slot = a;
  if (a < 0 || a >= p.L) return 0;
  return p.ranks ? min(max(p.ranks[a], 0), p.R) : p.R;
}

// u[m][j] = s_a sum_k x[m][k] A_a[j][k]: one workgroup per token, one wave per
// rank at a time
template <int DT>
__device__ __forceinline__ void shrink_token(const AdapterParams& p, int m) {
  int a;
  const int r = adapter_of(p, m, &a);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, NW = blockDim.x >> 6;
  const uint16_t* xr = p.x + (size_t)m * p.K;
  const float sc = r > 0 && p.scale ? p.scale[a] : 1.f;
  for (int j = wave; j < r; j += NW) {
    const uint16_t* ar = p.A + (size_t)a * p.a_stride + (size_t)j * p.K;
    float s = 0.f;
    for (int k = 8 * lane; k < p.K; k += 512) {
      const u32x4 xv = ldg16(xr + k), av = ldg16(ar + k);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        s += act2f<DT>(xv[q] & 0xFFFFu) * act2f<DT>(av[q] & 0xFFFFu);
        s += act2f<DT>(xv[q] >> 16) * act2f<DT>(av[q] >> 16);
      }
    }
#pragma unroll
    for (int h = 32; h > 0; h >>= 1) s += __shfl_xor(s, h);
    if (lane == 0) p.u[(size_t)m * p.R + j] = sc * s;
  }
}

template <int DT>
__global__ __launch_bounds__(256) void k_adapter_shrink(AdapterGroup g) {
  const int b = blockIdx.x;
  int i = 0;
#pragma unroll
  for (int j = 1; j < kGroupMax; ++j)
    if (j < g.n && b >= g.shrink_start[j]) i = j;
  shrink_token<DT>(g.p[i], b - g.shrink_start[i]);
}

// d[m][n], one thread each
template <int DT>
__global__ __launch_bounds__(256) void k_adapter_expand(AdapterGroup g) {
  const int b = blockIdx.x;
  int i = 0;
#pragma unroll
  for (int j = 1; j < kGroupMax; ++j)
    if (j < g.n && b >= g.expand_start[j]) i = j;
  const AdapterParams& p = g.p[i];
  const int chunks = (p.N + 255) / 256, bb = b - g.expand_start[i];
  const int m = bb / chunks, n = (bb - m * chunks) * 256 + threadIdx.x;
  if (n >= p.N) return;
  int a;
  const int r = adapter_of(p, m, &a);
  const size_t o = (size_t)m * p.N + n;
  float v = p.res ? act2f<DT>(p.res[o]) : 0.f;
  if (r > 0) {
    const uint16_t* br = p.B + (size_t)a * p.b_stride + (size_t)n * p.R;
    float s = 0.f;
    for (int j = 0; j < r; ++j) s += p.u[(size_t)m * p.R + j] * act2f<DT>(br[j]);
    v += s;
  }
  p.d[o] = f2act<DT>(v);
}

// ---------------------------------------------------------------------------
// launcher
// ---------------------------------------------------------------------------
hipError_t SPEAR_D(launch_adapters)(AdapterGroup& g, hipStream_t st) {
  if (g.n < 1 || g.n > kGroupMax) return hipErrorInvalidValue;
  g.shrink_start[0] = g.expand_start[0] = 0;
  for (int i = 0; i < g.n; ++i) {
    g.shrink_start[i + 1] = g.shrink_start[i] + g.p[i].M;
    g.expand_start[i + 1] = g.expand_start[i] + g.p[i].M * ((g.p[i].N + 255) / 256);
  }
  hipLaunchKernelGGL(k_adapter_shrink<DTC>, dim3(g.shrink_start[g.n]), dim3(256), 0, st, g);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(k_adapter_expand<DTC>, dim3(g.expand_start[g.n]), dim3(256), 0, st, g);
  return hipGetLastError();
}

}  // namespace spear
