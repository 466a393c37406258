// gfx950 (MI355X) kernel of the norms around a block:
//   o = y or RMSNorm(y; post_w), h' = rho h + beta act(gate) (.) o,
//   x = RMSNorm(h'; pre_w) over the stored h'
#include "spear_device.h"

namespace spear {

// sum over the workgroup (a multiple of 64 threads), the same in every thread
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int h = 32; h > 0; h >>= 1) v += __shfl_xor(v, h);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
  for (int i = 0; i < (int)(blockDim.x >> 6); ++i) s += red[i];
  return s;
}

__device__ __forceinline__ float gate_value(int kind, float g) {
  if (kind == BGATE_TANH) return tanhf(g);
  if (kind == BGATE_SIGMOID) return 1.f / (1.f + expf(-g));
  return g;
}

// gate row of token m, or null (no gate)
__device__ __forceinline__ const uint16_t* gate_row(const BlockNormParams& p, int m) {
  if (!p.gate) return nullptr;
  int r = p.n_gates == 1 ? 0 : m;
  if (p.gate_ids) {
    r = p.gate_ids[m];
    if (r < 0 || r >= p.n_gates) return nullptr;
  }
  return p.gate + (size_t)r * p.gate_ld;
}

// Rows of any length and stride: one workgroup per row, element by element.
template <int DT, bool F32>
__device__ __forceinline__ void block_norm_row(const BlockNormParams& p, int m, float* red) {
  const int tid = threadIdx.x, N = p.N;
  const uint16_t* y = p.y + (size_t)m * p.y_ld;
  const uint16_t* gr = gate_row(p, m);
  auto h_at = [&](const void* h, int64_t ld, int n) {
    return F32 ? ((const float*)h)[(size_t)m * ld + n] : act2f<DT>(((const uint16_t*)h)[(size_t)m * ld + n]);
  };
  float ps = 1.f;
  if (p.post_w) {
    float ss = 0.f;
    for (int n = tid; n < N; n += 256) {
      const float v = act2f<DT>(y[n]);
      ss += v * v;
    }
    ps = 1.f / sqrtf(block_sum(ss, red) / (float)N + p.eps);
  }
  float ss = 0.f;
  for (int n = tid; n < N; n += 256) {
    float o = act2f<DT>(y[n]);
    if (p.post_w) o = o * ps * (p.w_offset + act2f<DT>(p.post_w[n]));
    if (gr) o *= gate_value(p.gate_kind, act2f<DT>(gr[n]));
    float v = p.branch_scale * o;
    if (p.h) v += p.stream_scale * h_at(p.h, p.h_ld, n);
    if (F32) {
      ((float*)p.h_out)[(size_t)m * p.h_out_ld + n] = v;
    } else {
      const uint16_t b = f2act<DT>(v);
      ((uint16_t*)p.h_out)[(size_t)m * p.h_out_ld + n] = b;
      v = act2f<DT>(b);
    }
    ss += v * v;
  }
  if (!p.pre_w) return;
  const float xs = 1.f / sqrtf(block_sum(ss, red) / (float)N + p.eps);
  // each thread reads back the elements it wrote
  for (int n = tid; n < N; n += 256)
    p.x[(size_t)m * p.x_ld + n] = f2act<DT>(h_at(p.h_out, p.h_out_ld, n) * xs * (p.w_offset + act2f<DT>(p.pre_w[n])));
}

template <int DT, bool F32>
__global__ __launch_bounds__(256) void k_block_norm(BlockNormParams p) {
  __shared__ float red[4];
  for (long long m = blockIdx.x; m < p.M; m += gridDim.x) block_norm_row<DT, F32>(p, (int)m, red);
}

hipError_t SPEAR_D(launch_block_norm)(const BlockNormParams& p, hipStream_t st) {
  if (p.M <= 0 || p.N <= 0) return hipSuccess;
  const int grid = std::min(p.M, 1 << 20);  // a launch holds fewer than 2^32 threads
  if (p.f32) hipLaunchKernelGGL((k_block_norm<DTC, true>), dim3(grid), dim3(256), 0, st, p);
  else hipLaunchKernelGGL((k_block_norm<DTC, false>), dim3(grid), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace spear
