// gfx950 (MI355X) kernel of the norms around a block:
//   o = y or RMSNorm(y; post_w), h' = rho h + beta act(gate) (.) o,
//   x = RMSNorm(h'; pre_w) over the stored h'
#include "spear_device.h"

namespace spear {

// sum over a wave, the same in every lane: exchanges in registers within 16 lanes
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_add<0xB1>(v);   // pairs
  v = dpp_add<0x4E>(v);   // pairs of a four
  v = dpp_add<0x141>(v);  // fours of an eight (mirrored)
  v = dpp_add<0x140>(v);  // eights of a sixteen (mirrored)
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// sum over the workgroup (a multiple of 64 threads), the same in every thread
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
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

// 16 bytes at an address of any element (the compiler's own unaligned access)
typedef u32x4 __attribute__((aligned(2))) u32x4_a2;
typedef f32x4 __attribute__((aligned(4))) f32x4_a4;
template <bool AL>
__device__ __forceinline__ u32x4 ld8(const uint16_t* p) {
  if constexpr (AL) return *(const u32x4*)p;
  else return *(const u32x4_a2*)p;
}
template <bool AL>
__device__ __forceinline__ void st8(uint16_t* p, u32x4 v) {
  if constexpr (AL) *(u32x4*)p = v;
  else *(u32x4_a2*)p = v;
}
// eight activations from element n of a row (cnt of them, the others zero)
template <bool AL>
__device__ __forceinline__ u32x4 ld_chunk(const uint16_t* r, int n, int cnt) {
  if (cnt >= 8) return ld8<AL>(r + n);
  u32x4 v = u32x4{0, 0, 0, 0};
  if constexpr (!AL) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < cnt) v[e >> 1] |= (uint32_t)r[n + e] << (16 * (e & 1));
  }
  return v;
}
template <bool AL>
__device__ __forceinline__ void st_chunk(uint16_t* r, int n, int cnt, u32x4 v) {
  if (cnt >= 8) {
    st8<AL>(r + n, v);
  } else if constexpr (!AL) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < cnt) r[n + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
  }
}
struct f32x8 {
  f32x4 v[2];
};
template <bool AL>
__device__ __forceinline__ f32x8 ldf_chunk(const float* r, int n, int cnt) {
  f32x8 o;
  if (cnt >= 8) {
    if constexpr (AL) o.v[0] = *(const f32x4*)(r + n), o.v[1] = *(const f32x4*)(r + n + 4);
    else o.v[0] = *(const f32x4_a4*)(r + n), o.v[1] = *(const f32x4_a4*)(r + n + 4);
    return o;
  }
  o.v[0] = o.v[1] = f32x4{0.f, 0.f, 0.f, 0.f};
  if constexpr (!AL) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < cnt) o.v[e >> 2][e & 3] = r[n + e];
  }
  return o;
}
template <bool AL>
__device__ __forceinline__ void stf_chunk(float* r, int n, int cnt, const f32x8& o) {
  if (cnt >= 8) {
    if constexpr (AL) *(f32x4*)(r + n) = o.v[0], *(f32x4*)(r + n + 4) = o.v[1];
    else *(f32x4_a4*)(r + n) = o.v[0], *(f32x4_a4*)(r + n + 4) = o.v[1];
  } else if constexpr (!AL) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < cnt) r[n + e] = o.v[e >> 2][e & 3];
  }
}
template <int DT>
__device__ __forceinline__ float elem(const u32x4& v, int e) {
  return act2f<DT>((v[e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
}

// Rows whose elements fit the registers of T threads, C chunks of eight each:
// every input is read once, all of a row's loads go out before the first wait,
// and the row stays in registers through both norms. WAVE: a row per wave (T =
// 64, no barrier), else a row per workgroup. Up to two chunks the weights are
// loaded once and serve all rows that the workgroup takes. AL: rows of whole
// 16-byte aligned chunks; else any length and stride.
// Bound by memory for many rows: 4096 x 8192 fp16 with both norms and a gate row
// for each token moves 336 MB in 71 us, 4.7 TB/s (a copy of 1 GiB: 5.2); by
// latency for few: 3.4 us for one row of 4096, two dependent sums behind one load.
template <int DT, bool F32, int C, bool WAVE, bool AL>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void k_block_norm_v(BlockNormParams p) {
  __shared__ float red[2][16];
  const int N = p.N, T = WAVE ? 64 : blockDim.x;
  const int t = WAVE ? threadIdx.x & 63 : threadIdx.x;
  const int per = WAVE ? blockDim.x >> 6 : 1;  // rows a workgroup takes at a time
  constexpr bool HOLD = C <= 2;  // (four chunks and both weights exceed 128 registers)
  u32x4 pw[C], nw[C];
  auto weights = [&](u32x4 (&w)[C], const uint16_t* src) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = 8 * (c * T + t);
      w[c] = src ? ld_chunk<AL>(src, n, N - n) : u32x4{0, 0, 0, 0};
    }
  };
  if constexpr (HOLD) weights(pw, p.post_w), weights(nw, p.pre_w);
  auto row_sum = [&](float v, int k) {
    v = wave_sum(v);
    if constexpr (WAVE) return v;
    if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < T >> 6; ++i) v += red[k][i];
    return v;
  };
  const float inv_n = 1.f / (float)N;
  for (long long m0 = (long long)blockIdx.x * per; m0 < p.M; m0 += (long long)gridDim.x * per) {
    const long long m = WAVE ? m0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : m0;
    if (WAVE && m >= p.M) break;
    const uint16_t* y = p.y + (size_t)m * p.y_ld;
    u32x4 yv[C], gv[C];
    u32x4 hv[C];  // h, then h' (act dtype)
    f32x8 hf[C];  // the same, fp32
    if constexpr (!HOLD) weights(pw, p.post_w);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = 8 * (c * T + t);
      yv[c] = ld_chunk<AL>(y, n, N - n);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = 8 * (c * T + t);
      if constexpr (F32) {
        hf[c].v[0] = hf[c].v[1] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (p.h) hf[c] = ldf_chunk<AL>((const float*)p.h + (size_t)m * p.h_ld, n, N - n);
      } else {
        hv[c] = p.h ? ld_chunk<AL>((const uint16_t*)p.h + (size_t)m * p.h_ld, n, N - n) : u32x4{0, 0, 0, 0};
      }
    }
    const uint16_t* gr = gate_row(p, (int)m);
    if (gr) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int n = 8 * (c * T + t);
        gv[c] = ld_chunk<AL>(gr, n, N - n);
      }
    }
    float ps = 1.f;
    if (p.post_w) {
      float ss = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = elem<DT>(yv[c], e);
          ss += v * v;
        }
      ps = 1.f / sqrtf(row_sum(ss, 0) * inv_n + p.eps);
    }
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = 8 * (c * T + t);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float o = elem<DT>(yv[c], e);
        if (p.post_w) o = o * ps * (p.w_offset + elem<DT>(pw[c], e));
        if (gr) o *= gate_value(p.gate_kind, elem<DT>(gv[c], e));
        float r = p.branch_scale * o;
        if (p.h) r += p.stream_scale * (F32 ? hf[c].v[e >> 2][e & 3] : elem<DT>(hv[c], e));
        if constexpr (F32) {
          hf[c].v[e >> 2][e & 3] = r;
        } else {
          const uint32_t q = f2act<DT>(r);
          hv[c][e >> 1] = (e & 1) ? (hv[c][e >> 1] & 0xFFFFu) | (q << 16) : (hv[c][e >> 1] & 0xFFFF0000u) | q;
          r = act2f<DT>(q);
        }
        if (n + e < N) ss += r * r;
      }
      if (n < N) {
        if constexpr (F32) stf_chunk<AL>((float*)p.h_out + (size_t)m * p.h_out_ld, n, N - n, hf[c]);
        else st_chunk<AL>((uint16_t*)p.h_out + (size_t)m * p.h_out_ld, n, N - n, hv[c]);
      }
    }
    if (!p.pre_w) {
      if (!WAVE && p.post_w) __syncthreads();  // red[0] is written again by the next row
      continue;
    }
    if constexpr (!HOLD) weights(nw, p.pre_w);
    const float xs = 1.f / sqrtf(row_sum(ss, 1) * inv_n + p.eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = 8 * (c * T + t);
      u32x4 b;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float r = F32 ? hf[c].v[e >> 2][e & 3] : elem<DT>(hv[c], e);
        const uint16_t q = f2act<DT>(r * xs * (p.w_offset + elem<DT>(nw[c], e)));
        b[e >> 1] = (e & 1) ? b[e >> 1] | ((uint32_t)q << 16) : (uint32_t)q;
      }
      if (n < N) st_chunk<AL>(p.x + (size_t)m * p.x_ld, n, N - n, b);
    }
    // (without a norm after the block the next row's sum writes red[1] with no
    // barrier of its own in between)
    if (!WAVE && !p.post_w) __syncthreads();
  }
}

template <bool F32, bool AL>
static hipError_t norm_launch(const BlockNormParams& p, hipStream_t st) {
  const int n8 = (p.N + 7) / 8;
  const auto go = [&](auto kern, int rows, int threads) {
    const long long want = ((long long)p.M + rows - 1) / rows;
    const int grid = (int)std::min<long long>(want, 256 * 2048 / threads * 2);
    hipLaunchKernelGGL(kern, dim3(grid), dim3(threads), 0, st, p);
    return hipGetLastError();
  };
  if (n8 <= 64) return go(k_block_norm_v<DTC, F32, 1, true, AL>, 4, 256);
  if (n8 <= 128) return go(k_block_norm_v<DTC, F32, 2, true, AL>, 4, 256);
  if (n8 <= 256) return go(k_block_norm_v<DTC, F32, 1, false, AL>, 1, 256);
  // Up to a row for each CU a row's latency is all: one chunk a thread (kernel
  // times with two and with one: one row of 4096 4.1 and 3.4 us, 24 of 8192 in 32
  // bits 7.2 and 6.7). More rows share a CU, and the wider workgroups cost: 301 of
  // 5003 8.8 and 11.3.
  const bool few = p.M <= 256;
  if (few && n8 <= 512) return go(k_block_norm_v<DTC, F32, 1, false, AL>, 1, 512);
  if (few && n8 <= 1024) return go(k_block_norm_v<DTC, F32, 1, false, AL>, 1, 1024);
  if (n8 <= 512) return go(k_block_norm_v<DTC, F32, 2, false, AL>, 1, 256);
  if (n8 <= 1024) return go(k_block_norm_v<DTC, F32, 2, false, AL>, 1, 512);
  if (n8 <= 2048) return go(k_block_norm_v<DTC, F32, 2, false, AL>, 1, 1024);
  return go(k_block_norm_v<DTC, F32, 4, false, AL>, 1, 1024);
}

hipError_t SPEAR_D(launch_block_norm)(const BlockNormParams& p, hipStream_t st) {
  if (p.M <= 0 || p.N <= 0) return hipSuccess;
  if (p.N > 8 * 4096) {  // longer than the registers of a workgroup
    const int grid = std::min(p.M, 1 << 20);
    if (p.f32) hipLaunchKernelGGL((k_block_norm<DTC, true>), dim3(grid), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_block_norm<DTC, false>), dim3(grid), dim3(256), 0, st, p);
    return hipGetLastError();
  }
  const bool al = ((p.N | p.y_ld | p.gate_ld | p.h_ld | p.h_out_ld | p.x_ld) & 7) == 0;
  if (p.f32) return al ? norm_launch<true, true>(p, st) : norm_launch<true, false>(p, st);
  return al ? norm_launch<false, true>(p, st) : norm_launch<false, false>(p, st);
}

}  // namespace spear
