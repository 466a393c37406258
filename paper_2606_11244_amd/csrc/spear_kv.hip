// gfx950 (MI355X) kernels of a paged cache held in 8 bits: block tables and slot
// maps from lengths, rotary positions with the cache's writing, and values back.
#include "spear_device.h"
#include "spear_kv_internal.h"

namespace spear {

#if !SPEAR_BF16_UNIT
// ---------------------------------------------------------------------------
// Block tables, slots and positions. One workgroup: two sums over the requests
// (rows, then new pages of those that can be served), kept in LDS, and then the
// new pages and the rows in flat order, each finding its request by bisection.
// Everything is latency: a few dependent loads and four barriers a sum.
// ---------------------------------------------------------------------------
constexpr int kPagesThreads = 1024, kPagesEach = kKvRequests / kPagesThreads;

// exclusive sum over the workgroup, and its total
__device__ __forceinline__ int64_t scan_block(int64_t v, int64_t* red, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int64_t s = v;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(s, d);
    if (lane >= d) s += o;
  }
  __syncthreads();
  if (lane == 63) red[wave] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int i = 0; i < waves; ++i) {
    if (i < wave) before += red[i];
    all += red[i];
  }
  *total = all;
  return before + s - v;
}

// the last i of 0..n-1 with a[i] <= x (a ascending, a[0] <= x)
__device__ __forceinline__ int last_not_above(const int32_t* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kPagesThreads) void k_kv_pages(KvPagesParams p) {
  __shared__ int32_t s_start[kKvRequests + 1], s_held[kKvRequests], s_page[kKvRequests];
  __shared__ int64_t red[kPagesThreads / 64];
  __shared__ int s_taken, s_unserved;
  const int tid = threadIdx.x, each = (p.R + blockDim.x - 1) / blockDim.x;
  if (tid == 0) s_taken = 0, s_unserved = 0;
  int held[kPagesEach], rows[kPagesEach], need[kPagesEach];
  bool ok[kPagesEach];
  int64_t sum = 0;
#pragma unroll
  for (int e = 0; e < kPagesEach; ++e) {
    const int r = tid * each + e;
    held[e] = rows[e] = need[e] = 0;
    ok[e] = false;
    if (e >= each || r >= p.R) continue;
    const int h = p.held[r], f = p.fresh[r];
    ok[e] = h >= 0 && f >= 0 && (int64_t)h + f < kKvLength;
    held[e] = h;
    rows[e] = f > 0 ? min(f, p.T + 1) : 0;
    sum += rows[e];
  }
  int64_t total;
  int64_t at = scan_block(sum, red, &total);
  if (tid == 0) s_start[p.R] = p.starts[p.R] = (int)(total < p.T ? total : p.T);
  int64_t pages = 0;
#pragma unroll
  for (int e = 0; e < kPagesEach; ++e) {
    const int r = tid * each + e;
    if (e >= each || r >= p.R) continue;
    s_start[r] = p.starts[r] = (int)(at < p.T ? at : p.T);
    at += rows[e];
    const int len = ok[e] ? held[e] + p.fresh[r] : 0;
    const int has = (len + p.P - 1) / p.P;
    ok[e] = ok[e] && at <= p.T && has <= p.width;
    need[e] = ok[e] ? has - (held[e] + p.P - 1) / p.P : 0;
    pages += need[e];
  }
  at = scan_block(pages, red, &total);
  int unserved = 0, taken = 0;
#pragma unroll
  for (int e = 0; e < kPagesEach; ++e) {
    const int r = tid * each + e;
    if (e >= each || r >= p.R) continue;
    s_page[r] = (int)(at < p.n_free ? at : p.n_free);
    at += need[e];
    ok[e] = ok[e] && (need[e] == 0 || at <= p.n_free);
    if (ok[e] && need[e]) taken = (int)at;
    unserved += !ok[e];
    s_held[r] = ok[e] ? held[e] : -1;
    p.lens[r] = ok[e] ? held[e] + p.fresh[r] : 0;
  }
  if (taken) atomicMax(&s_taken, taken);
  if (unserved) atomicAdd(&s_unserved, unserved);
  __syncthreads();
  if (tid == 0) p.taken[0] = s_taken, p.taken[1] = s_unserved;
  // the k-th page taken goes to the last request whose pages begin at or before it
  for (int k = tid; k < s_taken; k += blockDim.x) {
    const int r = last_not_above(s_page, p.R, k);
    const int j = (s_held[r] + p.P - 1) / p.P + k - s_page[r];
    p.table[r * p.ld + j] = p.free_pages[k];
  }
  for (int t = tid; t < p.T; t += blockDim.x) {
    int slot = -1, pos = 0;
    if (p.R && t < s_start[p.R]) {
      const int r = last_not_above(s_start, p.R, t);
      if (s_held[r] >= 0) {
        pos = s_held[r] + t - s_start[r];
        const int had = (s_held[r] + p.P - 1) / p.P, j = pos / p.P;
        // (a new page's entry comes from the list: the table's is being written)
        const int page = j < had ? p.table[r * p.ld + j] : p.free_pages[s_page[r] + j - had];
        const int64_t s = (int64_t)page * p.P + pos % p.P;
        slot = page < 0 || s > 0x7fffffffll ? -1 : (int)s;
      }
    }
    p.slots[t] = slot;
    p.positions[t] = pos;
  }
}

hipError_t launch_kv_pages(const KvPagesParams& p, hipStream_t st) {
  const int threads = std::min(kPagesThreads, std::max(64, (std::max(p.R, p.T) + 63) / 64 * 64));
  hipLaunchKernelGGL(k_kv_pages, dim3(1), dim3(threads), 0, st, p);
  return hipGetLastError();
}
#endif

// ---------------------------------------------------------------------------
// Codes and scales
// ---------------------------------------------------------------------------

// least power of two whose multiple by 127 or 448 reaches top, from the bits of
// top = m 2^e: 127 = 1.984375 2^6, 448 = 1.75 2^8
template <int FMT>
__device__ __forceinline__ float scale_of(float top) {
  const uint32_t b = __float_as_uint(top), m = b & 0x7FFFFFu;
  const int e = (int)(b >> 23) - 127;
  const int s = FMT == KV_INT8 ? e - 6 + (m > 0x7E0000u) : e - 8 + (m > 0x600000u);
  return __uint_as_float((uint32_t)(max(s, -100) + 127) << 23);
}
// the largest code whose value is finite in the activation type (a scale that
// its page needs is at most twice what the type's largest value needs)
template <int DT, int FMT>
__device__ __forceinline__ float top_code(float scale) {
  const float reach = DT == DT_F16 ? 65504.f : 3.38953139e38f, top = FMT == KV_INT8 ? 127.f : 448.f;
  return scale * top > reach ? (FMT == KV_INT8 ? 63.f : 240.f) : top;
}
// four values (already divided by the scale) as codes in a dword
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4]) {
  if constexpr (FMT == KV_INT8) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)rintf(x[i]) & 0xFFu) << (8 * i);
    return w;
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
  }
}
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  if constexpr (FMT == KV_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)((int)(w << (24 - 8 * i)) >> 24);
  } else {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
  }
}
// a value over its scale, NaN as zero, what passes the largest code as that
__device__ __forceinline__ float to_code(float x, float inv, float most) {
  const float c = x == x ? x * inv : 0.f;
  return fminf(fmaxf(c, -most), most);
}
__device__ __forceinline__ float finite_size(float x) {
  const float a = fabsf(x);
  return a <= 3.40282347e38f ? a : 0.f;  // (false for NaN)
}

// ---------------------------------------------------------------------------
// Rotation. The angle is a 64-bit fraction of a turn, pos * freq modulo 2^64,
// exact at every position (in fp32 radians a position of 10^5 would be off by
// 10^-2). Its upper 32 bits give the quarter and a rest of at most an eighth of a
// turn either way, where Taylor's sums to x^9 and x^8 stay within 2e-9 and 3e-8.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float2 cos_sin(uint64_t turn, float magnitude) {
  const uint32_t hi = (uint32_t)(turn >> 32), quarter = (hi + 0x20000000u) >> 30;
  const float x = (float)(int)(hi - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float y = x * x;
  const float s = x * (1.f + y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880)))));
  const float c = 1.f + y * (-1.f / 2 + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320))));
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2((quarter == 1 || quarter == 2) ? -a * magnitude : a * magnitude,
                     quarter >= 2 ? -b * magnitude : b * magnitude);
}

// The features of a head as units of two runs of W features, at p0 and p1, that
// rotate together: W = 8 where pairs of features lie rot/2 apart or side by side
// and rot is a multiple of 16, else W = 1, the two features of a pair.
struct Unit {
  int p0, p1, pair;  // pair: of the first feature (-1: passes unchanged)
};
template <int W>
__device__ __forceinline__ Unit unit_at(int u, int rot, int interleaved) {
  const int f = 2 * W * u;
  if (f >= rot) return {f, f + W, -1};
  if (interleaved) return {f, f + W, f / 2};
  return {W * u, W * u + rot / 2, W * u};
}
template <int DT, int W>
__device__ __forceinline__ void load_run(const uint16_t* p, float (&x)[W]) {
  if constexpr (W == 8) {
    const u32x4 v = ldg16(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = act2f<DT>((v[i >> 1] >> (16 * (i & 1))) & 0xFFFFu);
  } else {
    x[0] = act2f<DT>(p[0]);
  }
}
// turns both runs; cs(pair) is the cosine and sine of a pair
template <int W, class CS>
__device__ __forceinline__ void turn(const Unit& u, int interleaved, float (&a)[W], float (&b)[W], CS cs) {
  if (u.pair < 0) return;
  if (W == 8 && interleaved) {
#pragma unroll
    for (int i = 0; i < W; i += 2) {
      const float2 s = cs(u.pair + i / 2), t = cs(u.pair + W / 2 + i / 2);
      const float x = a[i], y = b[i];
      a[i] = x * s.x - a[i + 1] * s.y;
      a[i + 1] = a[i + 1] * s.x + x * s.y;
      b[i] = y * t.x - b[i + 1] * t.y;
      b[i + 1] = b[i + 1] * t.x + y * t.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float2 s = cs(u.pair + i);
      const float x = a[i];
      a[i] = x * s.x - b[i] * s.y;
      b[i] = b[i] * s.x + x * s.y;
    }
  }
}

// ---------------------------------------------------------------------------
// New tokens. A workgroup of the cache's part owns the runs of tokens (those of
// one page that follow each other) that begin in its window of rows, for one head
// and K or V: it brings the run to LDS in fp32 (K turned), takes the largest
// magnitude, settles the page's scale with the one before, divides the codes
// already there if it grew, and writes the run's. One page and head is one
// workgroup's alone: no atomics, the same codes on every run. A workgroup of the
// queries' part takes whole tokens, its cosines and sines in LDS for all heads.
// Bound: the bytes of q, k and v (long prompts), latency (decode).
// ---------------------------------------------------------------------------
template <int DT, int FMT, int W>
__device__ void append_run(const KvAppendParams& p, int t, int slot, int n, int h, bool is_v, float* x, float* red) {
  const int tid = threadIdx.x, D = p.c.D, P = p.c.P, page = slot / P, off = slot % P;
  const int pitch = is_v ? D + 1 : D;
  float top = 0.f;
  if (is_v) {
    for (int i = tid; i < n * (D / 8); i += 256) {
      const int m = i / (D / 8), d = 8 * (i % (D / 8));
      float a[8];
      load_run<DT, 8>(p.v + (int64_t)(t + m) * p.v_ld + h * D + d, a);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[m * pitch + d + e] = a[e];
        top = fmaxf(top, finite_size(a[e]));
      }
    }
  } else {
    const int units = D / (2 * W);
    for (int i = tid; i < n * units; i += 256) {
      const int m = i / units;
      const Unit u = unit_at<W>(i % units, p.r.rot, p.r.interleaved);
      const uint16_t* k = p.k + (int64_t)(t + m) * p.k_ld + h * D;
      float a[W], b[W];
      load_run<DT, W>(k + u.p0, a);
      load_run<DT, W>(k + u.p1, b);
      const uint64_t pos = p.r.rot ? (uint64_t)(int64_t)p.positions[t + m] : 0;
      turn<W>(u, p.r.interleaved, a, b, [&](int i) { return cos_sin(pos * p.r.freqs[i], p.r.magnitude); });
#pragma unroll
      for (int e = 0; e < W; ++e) {
        x[m * pitch + u.p0 + e] = a[e];
        x[m * pitch + u.p1 + e] = b[e];
        top = fmaxf(top, fmaxf(finite_size(a[e]), finite_size(b[e])));
      }
    }
  }
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if ((tid & 63) == 0) red[tid >> 6] = top;
  float* scale = (is_v ? p.c.v_scale : p.c.k_scale) + (int64_t)page * p.c.Hkv + h;
  const float before = off ? *scale : 0.f;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float s = fmaxf(before, scale_of<FMT>(top)), inv = 1.f / s, ratio = before * inv;
  const float most = top_code<DT, FMT>(s);
  const bool grew = s > before;
  if (tid == 0 && grew) *scale = s;
  uint8_t* codes = (is_v ? p.c.v : p.c.k) + ((int64_t)page * p.c.Hkv + h) * P * D;
  if (is_v) {  // [D][P]: dwords of four places
    const int g0 = grew ? 0 : off / 4, groups = (off + n + 3) / 4 - g0;
    for (int i = tid; i < D * groups; i += 256) {
      const int d = i / groups, at = 4 * (g0 + i % groups);
      uint32_t* w = (uint32_t*)(codes + d * P + at);
      uint32_t old = 0;
      float c[4];
      const bool part = at < off || at + 4 > off + n;
      if (part) old = *w;
      uint32_t kept = old;
      if (at < off && grew) {
        decode4<FMT>(old, c);
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] *= ratio;
        kept = encode4<FMT>(c);
      }
      uint32_t fresh = 0, before_run = 0, behind_run = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = at + e - off;
        c[e] = m >= 0 && m < n ? to_code(x[m * pitch + d], inv, most) : 0.f;
        before_run |= m < 0 ? 0xFFu << (8 * e) : 0u;
        behind_run |= m >= n ? 0xFFu << (8 * e) : 0u;
      }
      fresh = encode4<FMT>(c);
      *w = (kept & before_run) | (old & behind_run) | (fresh & ~(before_run | behind_run));
    }
  } else {  // [P][D]
    const int m0 = grew ? -off : 0, quads = D / 4;
    for (int i = tid; i < (n - m0) * quads; i += 256) {
      const int m = m0 + i / quads, d = 4 * (i % quads);
      uint32_t* w = (uint32_t*)(codes + (off + m) * D + d);
      float c[4];
      if (m < 0) {
        decode4<FMT>(*w, c);
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] *= ratio;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = to_code(x[m * pitch + d + e], inv, most);
      }
      *w = encode4<FMT>(c);
    }
  }
  __syncthreads();  // x and red belong to the next run
}

template <int DT, int FMT, int W>
__global__ __launch_bounds__(256) void k_kv_append(KvAppendParams p) {
  extern __shared__ float lds[];
  __shared__ float red[4];
  const int tid = threadIdx.x, D = p.c.D, P = p.c.P;
  const int64_t capacity = (int64_t)p.c.pages * P;
  if (blockIdx.x < p.kv_blocks) {
    const int is_v = blockIdx.x & 1, h = (blockIdx.x >> 1) % p.c.Hkv;
    const int t0 = (int)((blockIdx.x >> 1) / p.c.Hkv) * p.window;
    for (int t = t0; t < min(t0 + p.window, p.T); ++t) {
      const int slot = p.slots[t];
      if (slot < 0 || slot >= capacity) continue;
      if (t) {  // not the first of its page's tokens
        const int prev = p.slots[t - 1];
        if (prev >= 0 && prev < capacity && prev / P == slot / P) continue;
      }
      // how many follow: the first lane whose token does not
      const int most = min(P - slot % P, p.T - t), lane = tid & 63;
      int n = 0;
      for (int i = 0; i < most; i += 64) {
        const int m = i + lane;
        const uint64_t yes = __ballot(m < most && p.slots[t + m] == slot + m);
        const int run = yes == ~0ull ? 64 : __builtin_ctzll(~yes);
        n += run;
        if (run < 64) break;
      }
      append_run<DT, FMT, W>(p, t, slot, n, h, is_v, lds, red);
    }
    return;
  }
  // queries
  const int t0 = (int)(blockIdx.x - p.kv_blocks) * p.q_tokens, count = min(p.q_tokens, p.T - t0);
  float2* cs = (float2*)lds;
  const int half = p.r.rot / 2, units = D / (2 * W), per = p.H * units;
  for (int i = tid; i < count * half; i += 256)
    cs[i] = cos_sin((uint64_t)(int64_t)p.positions[t0 + i / half] * p.r.freqs[i % half], p.r.magnitude);
  __syncthreads();
  for (int i = tid; i < count * per; i += 256) {
    const int m = i / per, hu = i % per, h = hu / units, t = t0 + m;
    const int slot = p.slots[t];
    if (slot < 0 || slot >= capacity) continue;
    const Unit u = unit_at<W>(hu % units, p.r.rot, p.r.interleaved);
    const uint16_t* q = p.q + (int64_t)t * p.q_ld + h * D;
    uint16_t* o = p.q_out + (int64_t)t * p.qo_ld + h * D;
    float a[W], b[W];
    load_run<DT, W>(q + u.p0, a);
    load_run<DT, W>(q + u.p1, b);
    turn<W>(u, p.r.interleaved, a, b, [&](int i) { return cs[m * half + i]; });
    if constexpr (W == 8) {
      u32x4 va, vb;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        va[e] = (uint32_t)f2act<DT>(a[2 * e]) | ((uint32_t)f2act<DT>(a[2 * e + 1]) << 16);
        vb[e] = (uint32_t)f2act<DT>(b[2 * e]) | ((uint32_t)f2act<DT>(b[2 * e + 1]) << 16);
      }
      *(u32x4*)(o + u.p0) = va;
      *(u32x4*)(o + u.p1) = vb;
    } else {
      o[u.p0] = f2act<DT>(a[0]);
      o[u.p1] = f2act<DT>(b[0]);
    }
  }
}

template <int FMT>
static hipError_t append_launch(const KvAppendParams& p, hipStream_t st) {
  const uint32_t run = (uint32_t)std::min(p.c.P, p.T) * (p.c.D + 1) * 4;
  const uint32_t lds = std::max(run, (uint32_t)(p.q_tokens * p.r.rot / 2 * 8));
  const auto go = [&](auto kern) {
    const hipError_t e = allow_lds(kern, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(p.kv_blocks + p.q_blocks), dim3(256), lds, st, p);
    return hipGetLastError();
  };
  return p.r.rot % 16 == 0 ? go(k_kv_append<DTC, FMT, 8>) : go(k_kv_append<DTC, FMT, 1>);
}
hipError_t SPEAR_D(launch_kv_append)(const KvAppendParams& p, int format, hipStream_t st) {
  return format == KV_INT8 ? append_launch<KV_INT8>(p, st) : append_launch<KV_E4M3>(p, st);
}

// ---------------------------------------------------------------------------
// Values back: sixteen tokens of one head a workgroup; V, whose places of one
// feature lie side by side, changes its order through LDS.
// ---------------------------------------------------------------------------
template <int DT, int FMT>
__global__ __launch_bounds__(256) void k_kv_read(KvReadParams p) {
  __shared__ uint16_t turned[16][128 + 2];
  const int tid = threadIdx.x, D = p.c.D, P = p.c.P, h = blockIdx.x % p.c.Hkv;
  const int64_t i0 = (int64_t)(blockIdx.x / p.c.Hkv) * 16, capacity = (int64_t)p.c.pages * P;
  auto slot_of = [&](int m) {
    const int s = i0 + m < p.n ? p.slots[i0 + m] : -1;
    return s < capacity ? s : -1;
  };
  for (int i = tid; i < 16 * (D / 4); i += 256) {
    const int m = i / (D / 4), d = 4 * (i % (D / 4)), s = slot_of(m);
    if (s < 0) continue;
    const int64_t ph = (int64_t)(s / P) * p.c.Hkv + h;
    float c[4];
    decode4<FMT>(*(const uint32_t*)(p.c.k + (ph * P + s % P) * D + d), c);
    const float scale = p.c.k_scale[ph];
    uint16_t* o = p.k_out + ((i0 + m) * p.c.Hkv + h) * D + d;
    *(u32x2*)o = u32x2{(uint32_t)f2act<DT>(c[0] * scale) | ((uint32_t)f2act<DT>(c[1] * scale) << 16),
                       (uint32_t)f2act<DT>(c[2] * scale) | ((uint32_t)f2act<DT>(c[3] * scale) << 16)};
  }
  {
    const int m = tid & 15, s = slot_of(m);
    if (s >= 0) {
      const int64_t ph = (int64_t)(s / P) * p.c.Hkv + h;
      const float scale = p.c.v_scale[ph];
      for (int d = tid >> 4; d < D; d += 16) {
        float c[4];
        decode4<FMT>(p.c.v[(ph * D + d) * P + s % P], c);
        turned[m][d] = f2act<DT>(c[0] * scale);
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < 16 * (D / 2); i += 256) {
    const int m = i / (D / 2), d = 2 * (i % (D / 2));
    if (slot_of(m) < 0) continue;
    *(uint32_t*)(p.v_out + ((i0 + m) * p.c.Hkv + h) * D + d) = *(const uint32_t*)&turned[m][d];
  }
}

hipError_t SPEAR_D(launch_kv_read)(const KvReadParams& p, int format, hipStream_t st) {
  const dim3 grid((uint32_t)((p.n + 15) / 16 * p.c.Hkv));
  if (format == KV_INT8) hipLaunchKernelGGL((k_kv_read<DTC, KV_INT8>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((k_kv_read<DTC, KV_E4M3>), grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace spear
