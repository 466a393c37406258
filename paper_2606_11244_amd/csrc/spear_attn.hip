// gfx950 (MI355X) kernels of attention over a paged cache held in 8 bits.
#include "spear_device.h"
#include "spear_kv_internal.h"

namespace spear {

template <int FMT>
__device__ __forceinline__ float code_value(uint8_t b) {
  if constexpr (FMT == KV_INT8) return (float)(int8_t)b;
  else return __builtin_amdgcn_cvt_f32_fp8((int)b, 0);
}

// One wave a row and head: 64 tokens a step, a token a lane for the scores, then
// two (or one) features a lane for the sum.
template <int DT, int FMT, int D>
__global__ __launch_bounds__(64) void k_kv_attend(KvAttendParams p) {
  const int lane = threadIdx.x, h = blockIdx.x % p.H, t = blockIdx.x / p.H, hk = h / p.group;
  if (t >= p.starts[p.R]) return;
  int r = 0, hi = p.R;
  while (hi - r > 1) {
    const int mid = (r + hi) >> 1;
    if (p.starts[mid] <= t) r = mid;
    else hi = mid;
  }
  const int rows = p.starts[r + 1] - p.starts[r], i = t - p.starts[r];
  if (i < 0 || i >= rows || i >= p.max_new) return;
  const int len = (int)min((int64_t)p.lens[r], (int64_t)p.width * p.c.P), pos = p.lens[r] - rows + i;
  const int first = p.prefix ? p.prefix[r] : 0;
  const uint16_t* q = p.q + (int64_t)t * p.q_ld + h * D;
  const float slope = p.slopes ? p.slopes[h] : 0.f;
  float m = -__builtin_inff(), l = 0.f, o[D / 64] = {};
  for (int j0 = 0; j0 < len; j0 += 64) {
    const int j = j0 + lane;
    bool seen = j < len && ((j <= pos && pos - j < p.window_tokens) || j < first);
    int page = -1;
    if (seen) page = p.table[r * p.ld + j / p.c.P];
    seen = seen && page >= 0 && page < p.c.pages;
    float s = -__builtin_inff(), vs = 0.f;
    int64_t ph = 0;
    if (seen) {
      ph = (int64_t)page * p.c.Hkv + hk;
      const uint8_t* k = p.c.k + (ph * p.c.P + j % p.c.P) * D;
      float dot = 0.f;
      for (int d = 0; d < D; ++d) dot += act2f<DT>(q[d]) * code_value<FMT>(k[d]);
      s = dot * p.c.k_scale[ph] * p.scale;
      if (p.softcap > 0.f) s = p.softcap * tanhf(s / p.softcap);
      s -= slope * (float)abs(pos - j);
      vs = p.c.v_scale[ph];
    }
    float top = s;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (top == -__builtin_inff()) continue;
    const float now = fmaxf(m, top), fade = m == now ? 1.f : expf(m - now);
    const float e = seen ? expf(s - now) : 0.f;
    m = now;
    float sum = e;
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    l = l * fade + sum;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) o[c] *= fade;
    for (int x = 0; x < 64; ++x) {
      const float w = __shfl(e, x);
      if (w == 0.f) continue;
      const int64_t at = __shfl(ph, x);
      const float sc = __shfl(vs, x);
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        o[c] += w * sc * code_value<FMT>(p.c.v[(at * D + 64 * c + lane) * p.c.P + (j0 + x) % p.c.P]);
    }
  }
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
    p.out[(int64_t)t * p.out_ld + h * D + 64 * c + lane] = f2act<DT>(l > 0.f ? o[c] / l : 0.f);
}

template <int FMT>
static hipError_t attend_launch(const KvAttendParams& p, hipStream_t st) {
  const dim3 grid((uint32_t)p.T * p.H);
  if (p.c.D == 64) hipLaunchKernelGGL((k_kv_attend<DTC, FMT, 64>), grid, dim3(64), 0, st, p);
  else hipLaunchKernelGGL((k_kv_attend<DTC, FMT, 128>), grid, dim3(64), 0, st, p);
  return hipGetLastError();
}
hipError_t SPEAR_D(launch_kv_attend)(const KvAttendParams& p, int format, hipStream_t st) {
  return format == KV_INT8 ? attend_launch<KV_INT8>(p, st) : attend_launch<KV_E4M3>(p, st);
}

}  // namespace spear
