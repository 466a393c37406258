// gfx950 (MI355X) kernels of a paged cache held in 8 bits: block tables and slot
// maps from lengths, rotary positions with the cache's writing, and values back.
#include "spear_device.h"
#include "spear_kv_internal.h"

namespace spear {

#if !SPEAR_BF16_UNIT
// ---------------------------------------------------------------------------
// Block tables, slots and positions. Two sums over the requests (rows, then new
// pages of those that can be served), kept in LDS, and then the new pages and the
// rows in flat order, each finding its request by bisection. Bound: latency, a few
// dependent loads and two barriers a sum: one request 3.4 us, 384 with 5276 rows 6.7.
// ---------------------------------------------------------------------------
constexpr int kPagesThreads = 1024;

// sum over the workgroup before this thread, and in all, held at 2^32 - 1
__device__ __forceinline__ uint32_t scan_block(uint32_t v, uint32_t* red, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(s, d);
    if (lane >= d) s = __builtin_elementwise_add_sat(s, o);
  }
  const uint32_t up = __shfl_up(s, 1);
  if (lane == 63) red[wave] = s;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int i = 0; i < waves; ++i) {
    if (i < wave) before = __builtin_elementwise_add_sat(before, red[i]);
    all = __builtin_elementwise_add_sat(all, red[i]);
  }
  __syncthreads();
  *total = all;
  return lane ? __builtin_elementwise_add_sat(before, up) : before;
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

// EACH: requests a thread. Every workgroup makes the sums; the first writes what is
// one a request, and all share the new pages and the rows.
template <int EACH>
__global__ __launch_bounds__(kPagesThreads) void k_kv_pages(KvPagesParams p) {
  __shared__ int32_t s_start[EACH * kPagesThreads + 1], s_held[EACH * kPagesThreads], s_page[EACH * kPagesThreads];
  __shared__ uint32_t red[kPagesThreads / 64];
  __shared__ int s_taken, s_unserved;
  const int tid = threadIdx.x, r0 = tid * EACH, rows_all = p.T;
  const bool first = blockIdx.x == 0;
  if (tid == 0) s_taken = 0, s_unserved = 0;
  int held[EACH], fresh[EACH], need[EACH];
  bool ok[EACH];
  uint32_t sum = 0, total;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const bool there = r0 + e < p.R;
    held[e] = there ? p.held[r0 + e] : 0;
    fresh[e] = there ? p.fresh[r0 + e] : 0;
    ok[e] = there && held[e] >= 0 && fresh[e] >= 0 && (int64_t)held[e] + fresh[e] < kKvLength;
    sum = __builtin_elementwise_add_sat(sum, (uint32_t)max(fresh[e], 0));
  }
  uint32_t at = scan_block(sum, red, &total);
  if (tid == 0) s_start[p.R] = (int)min(total, (uint32_t)rows_all);
  uint32_t pages = 0;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    if (r0 + e < p.R) s_start[r0 + e] = (int)min(at, (uint32_t)rows_all);
    at = __builtin_elementwise_add_sat(at, (uint32_t)max(fresh[e], 0));
    const int has = ok[e] ? (held[e] + fresh[e] + p.P - 1) / p.P : 0;
    ok[e] = ok[e] && at <= (uint32_t)rows_all && has <= p.width;
    need[e] = ok[e] ? has - (held[e] + p.P - 1) / p.P : 0;
    pages += need[e];
  }
  at = scan_block(pages, red, &total);
  int unserved = 0, taken = 0;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    if (r0 + e >= p.R) continue;
    s_page[r0 + e] = (int)min(at, (uint32_t)p.n_free);
    at = __builtin_elementwise_add_sat(at, (uint32_t)need[e]);
    ok[e] = ok[e] && (need[e] == 0 || at <= (uint32_t)p.n_free);
    if (ok[e] && need[e]) taken = (int)at;
    unserved += !ok[e];
    s_held[r0 + e] = ok[e] ? held[e] : -1;
    if (first) {
      p.starts[r0 + e] = s_start[r0 + e];
      p.lens[r0 + e] = ok[e] ? held[e] + fresh[e] : 0;
    }
  }
  if (taken) atomicMax(&s_taken, taken);
  if (unserved) atomicAdd(&s_unserved, unserved);
  __syncthreads();
  if (first && tid == 0) p.starts[p.R] = s_start[p.R], p.taken[0] = s_taken, p.taken[1] = s_unserved;
  const int step = gridDim.x * blockDim.x, me = blockIdx.x * blockDim.x + tid;
  // the k-th page taken goes to the last request whose pages begin at or before it
  for (int k = me; k < s_taken; k += step) {
    const int r = last_not_above(s_page, p.R, k);
    const int j = (s_held[r] + p.P - 1) / p.P + k - s_page[r];
    p.table[r * p.ld + j] = p.free_pages[k];
  }
  for (int t = me; t < p.T; t += step) {
    int slot = -1, pos = 0;
    if (p.R && t < s_start[p.R]) {
      const int r = last_not_above(s_start, p.R, t), h = s_held[r];
      if (h >= 0) {
        pos = h + t - s_start[r];
        const int had = (h + p.P - 1) / p.P, j = pos / p.P;
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
  const bool many = p.R > kPagesThreads;
  const int threads = many ? kPagesThreads : std::min(kPagesThreads, std::max(64, (std::max(p.R, p.T) + 63) / 64 * 64));
  // a row a thread: 5276 rows of 384 requests took 12.5 us in one workgroup
  const int grid = std::max(1, std::min(64, (p.T + threads - 1) / threads));
  if (many) hipLaunchKernelGGL(k_kv_pages<4>, dim3(grid), dim3(threads), 0, st, p);
  else hipLaunchKernelGGL(k_kv_pages<1>, dim3(grid), dim3(threads), 0, st, p);
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
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (DT == DT_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, h16x2));
  else return pack_bf16(a, b);
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

// The same in 64 bits (to 5e-17), for keys whose code fp32 leaves open.
struct CosSin64 {
  double x, y;
};
__device__ __forceinline__ CosSin64 cos_sin64(uint64_t turn, double magnitude) {
  const uint64_t quarter = (turn + 0x2000000000000000ull) >> 62;
  const double x = (double)(int64_t)(turn - (quarter << 62)) * 3.4061215800865545e-19;  // 2 pi / 2^64
  const double y = x * x;
  double s = 1. / 1307674368000, c = 1. / 20922789888000;  // 15!, 16!
  const double fs[] = {1. / 6227020800, 1. / 39916800, 1. / 362880, 1. / 5040, 1. / 120, 1. / 6, 1.};
  const double fc[] = {1. / 87178291200, 1. / 479001600, 1. / 3628800, 1. / 40320, 1. / 720, 1. / 24, 1. / 2, 1.};
  s = -s;
#pragma unroll
  for (int i = 0; i < 7; ++i) s = __builtin_fma(s, y, (i & 1) ? -fs[i] : fs[i]);
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_fma(c, y, (i & 1) ? fc[i] : -fc[i]);
  s *= x;
  const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return {(quarter == 1 || quarter == 2) ? -a * magnitude : a * magnitude, quarter >= 2 ? -b * magnitude : b * magnitude};
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
template <int W, class T, class CS>
__device__ __forceinline__ void turn(const Unit& u, int interleaved, T (&a)[W], T (&b)[W], CS cs) {
  if (u.pair < 0) return;
  if (W == 8 && interleaved) {
#pragma unroll
    for (int i = 0; i < W; i += 2) {
      const auto s = cs(u.pair + i / 2), t = cs(u.pair + W / 2 + i / 2);
      const T x = a[i], y = b[i];
      a[i] = x * s.x - a[i + 1] * s.y;
      a[i + 1] = a[i + 1] * s.x + x * s.y;
      b[i] = y * t.x - b[i + 1] * t.y;
      b[i + 1] = b[i + 1] * t.x + y * t.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const auto s = cs(u.pair + i);
      const T x = a[i];
      a[i] = x * s.x - b[i] * s.y;
      b[i] = b[i] * s.x + x * s.y;
    }
  }
}

// ---------------------------------------------------------------------------
// New tokens. A workgroup of the cache's part owns the runs of tokens (those of
// one page that follow each other) that begin in its share of a window of 64 rows,
// for one head and K or V: it takes the run to registers (K turned), the largest magnitude,
// settles the page's scale with the one before, divides the codes already there
// if it grew, and writes the run's. One page and head is one workgroup's alone: no
// atomics, the same codes on every run. A workgroup of the queries' part takes
// a token, its cosines and sines in LDS for all heads.
// Bound: the bytes of q, k and v (long prompts: 4096 tokens with 64 heads of queries and
// 8 of keys and values, 159 MB in 42 us, 3.8 TB/s), latency (decode: a token 5.8 us, 5.4
// without a rotation: slots, rows and the page's scale, maximum, codes one after the other).
// ---------------------------------------------------------------------------

// the scale of a page and head, from the one before and the largest magnitude given
struct PageScale {
  float scale, inv, ratio, most;  // ratio: what older codes are multiplied by
  bool grew;
};
template <int DT, int FMT>
__device__ __forceinline__ PageScale settle(float top, float before, float* red) {
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  __syncthreads();  // (red: of the run before)
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  PageScale s;
  s.scale = fmaxf(before, scale_of<FMT>(top));
  s.inv = 1.f / s.scale;
  s.ratio = before * s.inv;
  s.most = top_code<DT, FMT>(s.scale);
  s.grew = s.scale > before;
  return s;
}
// Older codes under a scale that grew. INT8's are held to the new scale's largest code: 127 at
// 2^9 would become 63.5 and round to 64 at 2^10, in fp16 an infinity. E4M3's largest, 448, is at
// most 224 under a larger scale, below the limit of 240.
template <int FMT>
__device__ __forceinline__ uint32_t divide4(uint32_t w, const PageScale& s) {
  float c[4];
  decode4<FMT>(w, c);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    c[e] *= s.ratio;
    if (FMT == KV_INT8) c[e] = fminf(fmaxf(c[e], -s.most), s.most);
  }
  return encode4<FMT>(c);
}

template <int DT, int FMT, int D, int W>
__device__ __forceinline__ void append_k(const KvAppendParams& p, int t, int slot, int n, int h, float* red) {
  constexpr int units = D / (2 * W);
  const int tid = threadIdx.x, P = p.c.P, page = slot >> p.log2_page, off = slot & (P - 1);
  const int64_t ph = (int64_t)page * p.c.Hkv + h;
  const float before = off ? p.c.k_scale[ph] : 0.f;
  uint8_t* codes = p.c.k + ph * P * D;
  typedef typename std::conditional<W == 8, u32x4, uint16_t>::type Raw;
  struct Pair {
    Raw a, b;
  };
  auto load = [&](int i) {
    const Unit u = unit_at<W>(i % units, p.r.rot, p.r.interleaved);
    const uint16_t* k = p.k + (int64_t)(t + i / units) * p.k_ld + h * D;
    return Pair{*(const Raw*)(k + u.p0), *(const Raw*)(k + u.p1)};
  };
  auto position = [&](int i) { return p.r.rot ? (uint64_t)(int64_t)p.positions[t + i / units] : 0; };
  auto widen = [&](const Raw& r, auto (&x)[W]) {
    if constexpr (W == 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = act2f<DT>((r[e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
    } else {
      x[0] = act2f<DT>(r);
    }
  };
  // the largest magnitude of a unit, turned in fp32
  auto largest = [&](int i, const Pair& r) {
    const Unit u = unit_at<W>(i % units, p.r.rot, p.r.interleaved);
    const uint64_t pos = position(i);
    float a[W], b[W], top = 0.f;
    widen(r.a, a), widen(r.b, b);
    turn<W>(u, p.r.interleaved, a, b, [&](int x) { return cos_sin(pos * p.r.freqs[x], p.r.magnitude); });
#pragma unroll
    for (int e = 0; e < W; ++e) top = fmaxf(top, fmaxf(finite_size(a[e]), finite_size(b[e])));
    return top;
  };
  // its codes, each the nearest to the rotation in 64 bits: from fp32, and the pairs one of
  // whose values then lies nearer to the border of two codes than fp32 is off once more in
  // 64 bits, one by one. 4096 tokens of 8 heads and 64 heads of queries: 45 us all in fp32
  // (one code in 10^5 the neighbour of the right one), 63 all in 64 bits, 48 this way.
  auto put = [&](int i, const Pair& r, const PageScale& s) {
    const Unit u = unit_at<W>(i % units, p.r.rot, p.r.interleaved);
    const uint64_t pos = position(i);
    float a[W], b[W], reach[W];
    widen(r.a, a), widen(r.b, b);
    const bool side_by_side = W == 8 && p.r.interleaved;
    // an fp32 rotation is off by at most 2^-21 of what it is made of
    const float part = u.pair < 0 ? 0.f : fabsf(p.r.magnitude * s.inv) * 4.76837158e-7f;
#pragma unroll
    for (int e = 0; e < W; ++e)
      reach[e] = part * (!side_by_side ? fabsf(a[e]) + fabsf(b[e])
                         : e < W / 2   ? fabsf(a[(2 * e) % W]) + fabsf(a[(2 * e + 1) % W])
                                       : fabsf(b[(2 * e) % W]) + fabsf(b[(2 * e + 1) % W]));
    turn<W>(u, p.r.interleaved, a, b, [&](int x) { return cos_sin(pos * p.r.freqs[x], p.r.magnitude); });
#pragma unroll
    for (int e = 0; e < W; ++e) a[e] = to_code(a[e], s.inv, s.most), b[e] = to_code(b[e], s.inv, s.most);
    uint8_t* row = codes + (off + i / units) * D;
    uint32_t near = 0;  // pairs
    auto check = [&](float c, float code, int pair) {
      // (half the distance of two codes at c)
      const float half = FMT == KV_INT8 ? 0.5f : __uint_as_float((max((__float_as_uint(c) >> 23) & 255u, 121u) - 4) << 23);
      near |= fabsf(fabsf(c - code) - half) <= reach[pair] ? 1u << pair : 0u;
    };
    auto eight = [&](const float (&c)[W], int run) {
      u32x2 w;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float x[4] = {c[4 * q % W], c[(4 * q + 1) % W], c[(4 * q + 2) % W], c[(4 * q + 3) % W]};
        float y[4];
        w[q] = encode4<FMT>(x);
        decode4<FMT>(w[q], y);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (4 * q + e < W) check(x[e], y[e], side_by_side ? (W * run + 4 * q + e) / 2 : (4 * q + e) % W);
      }
      return w;
    };
    const u32x2 wa = eight(a, 0), wb = eight(b, 1);
    if constexpr (W == 8) {
      *(u32x2*)(row + u.p0) = wa;
      *(u32x2*)(row + u.p1) = wb;
    } else {  // (a rotation of no multiple of 16 features: a byte a store)
      row[u.p0] = (uint8_t)wa[0];
      row[u.p1] = (uint8_t)wb[0];
    }
    if (u.pair < 0) near = 0;
    const uint16_t* k = p.k + (int64_t)(t + i / units) * p.k_ld + h * D;
    for (; near; near &= near - 1) {
      const int e = __builtin_ctz(near);
      const int fa = side_by_side ? u.p0 + 2 * e : u.p0 + e, fb = side_by_side ? fa + 1 : u.p1 + e;
      const CosSin64 cs = cos_sin64(pos * p.r.freqs[u.pair + e], p.r.magnitude);
      const double x = act2f<DT>(k[fa]), y = act2f<DT>(k[fb]);
      auto code = [&](double v) {
        const double c = v == v ? v * (double)s.inv : 0.;
        const double d = fmin(fmax(c, -(double)s.most), (double)s.most);
        float f = (float)(FMT == KV_INT8 ? rint(d) : d);
        if (FMT == KV_E4M3) {  // to fp32 with an odd last bit if inexact: the rounding to a code sees the side of a border
          f = __uint_as_float(__float_as_uint(f) - (fabs((double)f) > fabs(d)));
          f = __uint_as_float(__float_as_uint(f) | ((double)f != d));
        }
        return f;
      };
      const float c[4] = {code(x * cs.x - y * cs.y), code(y * cs.x + x * cs.y), 0.f, 0.f};
      const uint32_t w = encode4<FMT>(c);
      row[fa] = (uint8_t)w;
      row[fb] = (uint8_t)(w >> 8);
    }
  };
  // a thread's first unit is held between the two, others are read again
  const int all = n * units;
  Pair own = {};
  float top = 0.f;
  if (tid < all) own = load(tid);
  if (tid < all) top = largest(tid, own);
#pragma unroll 1
  for (int i = tid + 256; i < all; i += 256) top = fmaxf(top, largest(i, load(i)));
  const PageScale s = settle<DT, FMT>(top, before, red);
  if (s.grew) {
    if (tid == 0) p.c.k_scale[ph] = s.scale;
    for (int i = tid; i < off * D / 4; i += 256) ((uint32_t*)codes)[i] = divide4<FMT>(((uint32_t*)codes)[i], s);
  }
#pragma unroll 1
  for (int i = tid; i < all; i += 256) {
    put(i, own, s);
    if (i + 256 < all) own = load(i + 256);
  }
}

// V: a unit is four places of a page (a dword of codes) and eight features
template <int DT, int FMT, int D>
__device__ __forceinline__ void append_v(const KvAppendParams& p, int t, int slot, int n, int h, float* red) {
  const int tid = threadIdx.x, P = p.c.P, page = slot >> p.log2_page, off = slot & (P - 1);
  const int64_t ph = (int64_t)page * p.c.Hkv + h;
  const float before = off ? p.c.v_scale[ph] : 0.f;
  uint8_t* codes = p.c.v + ph * P * D;
  constexpr int U = 2;  // units a thread at most
  const int q0 = off / 4, quads = (off + n + 3) / 4 - q0, units = quads * (D / 8);
  u32x4 x[U][4];
  int quad[U], feature[U];
  float top = 0.f;
#pragma unroll
  for (int y = 0; y < U; ++y) {
    const int i = tid + 256 * y;
    quad[y] = q0 + i % quads, feature[y] = 8 * (i / quads);
    if (i >= units) continue;
    const int m0 = 4 * quad[y] - off;
    const uint16_t* v = p.v + (int64_t)t * p.v_ld + h * D + feature[y];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[y][e] = m0 + e >= 0 && m0 + e < n ? ldg16(v + (int64_t)(m0 + e) * p.v_ld) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int f = 0; f < 8; ++f) top = fmaxf(top, finite_size(act2f<DT>((x[y][e][f >> 1] >> (16 * (f & 1))) & 0xFFFFu)));
  }
  const PageScale s = settle<DT, FMT>(top, before, red);
  if (tid == 0 && s.grew) p.c.v_scale[ph] = s.scale;
  if (s.grew)
    for (int i = tid; i < D * q0; i += 256) {
      uint32_t* w = (uint32_t*)(codes + i / q0 * P + 4 * (i % q0));
      *w = divide4<FMT>(*w, s);
    }
#pragma unroll
  for (int y = 0; y < U; ++y) {
    const int i = tid + 256 * y;
    if (i >= units) continue;
    const int m0 = 4 * quad[y] - off;
    uint32_t before_run = 0, behind_run = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      before_run |= m0 + e < 0 ? 0xFFu << (8 * e) : 0u;
      behind_run |= m0 + e >= n ? 0xFFu << (8 * e) : 0u;
    }
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      uint32_t* w = (uint32_t*)(codes + (feature[y] + f) * P + 4 * quad[y]);
      float c[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = to_code(act2f<DT>((x[y][e][f >> 1] >> (16 * (f & 1))) & 0xFFFFu), s.inv, s.most);
      uint32_t fresh = encode4<FMT>(c);
      if (before_run | behind_run) {
        const uint32_t old = *w, kept = before_run && s.grew ? divide4<FMT>(old, s) : old;
        fresh = (kept & before_run) | (old & behind_run) | (fresh & ~(before_run | behind_run));
      }
      *w = fresh;
    }
  }
}

// (four workgroups a CU: at the 137 registers that INT8 took without it, three fit, and
// the queries of a prompt came at 3560 GB/s, 3800 with it)
template <int DT, int FMT, int D, int W>
__global__ __launch_bounds__(256, 4) void k_kv_append(KvAppendParams p) {
  __shared__ float2 cs[64];
  __shared__ float red[4];
  const int tid = threadIdx.x, P = p.c.P, capacity = p.c.pages << p.log2_page;
  if (blockIdx.x < p.kv_blocks) {
    // (sub, window of 64 tokens, head, K or V): the sub-th of every p.subs runs that begin in the window.
    // The subs that find none in a prompt come last: side by side with the others they would leave the
    // work to the same few CUs (4096 tokens, 8 heads: 47 us, 35 this way).
    uint32_t b = blockIdx.x;
    const int is_v = b & 1, h = (b >>= 1) % p.c.Hkv, windows = (p.T + 63) / 64;
    const int t0 = (int)((b /= p.c.Hkv) % windows) * 64, sub = (int)(b / windows);
    const int lane = tid & 63, own = t0 + lane < p.T ? p.slots[t0 + lane] : -1;
    const int prev = t0 + lane > 0 && t0 + lane <= p.T ? p.slots[t0 + lane - 1] : -1;
    const bool first = own >= 0 && own < capacity && !(prev >= 0 && prev < capacity && (prev ^ own) < P);
    uint64_t starts = __ballot(first);
    for (int run = 0; starts; ++run, starts &= starts - 1) {
      if (run % p.subs != sub) continue;
      const int x = __builtin_ctzll(starts), t = t0 + x, slot = __builtin_amdgcn_readlane(own, x);
      // how many follow: the first lane whose token does not
      const int most = min(P - (slot & (P - 1)), p.T - t);
      int n = 0;
      for (int i = 0; i < most; i += 64) {
        const int m = i + lane;
        const uint64_t yes = __ballot(m < most && p.slots[t + m] == slot + m);
        const int more = yes == ~0ull ? 64 : __builtin_ctzll(~yes);
        n += more;
        if (more < 64) break;
      }
      if (is_v) append_v<DT, FMT, D>(p, t, slot, n, h, red);
      else append_k<DT, FMT, D, W>(p, t, slot, n, h, red);
    }
    return;
  }
  // queries: a token, N units a thread at a time, all requested before the first is turned
  const int t = (int)(blockIdx.x - p.kv_blocks), slot = p.slots[t];
  if (slot < 0 || slot >= capacity) return;
  constexpr int units = D / (2 * W), N = 2;
  const int half = p.r.rot / 2, all = p.H * units;
  const uint64_t pos = half ? (uint64_t)(int64_t)p.positions[t] : 0;
  const uint16_t* q = p.q + (int64_t)t * p.q_ld;
  uint16_t* out = p.q_out + (int64_t)t * p.qo_ld;
  typedef typename std::conditional<W == 8, u32x4, uint16_t>::type Raw;
  Raw ra[N], rb[N];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int i = min(i0 + 256 * x, all - 1);
      const Unit u = unit_at<W>(i % units, p.r.rot, p.r.interleaved);
      ra[x] = *(const Raw*)(q + i / units * D + u.p0);
      rb[x] = *(const Raw*)(q + i / units * D + u.p1);
    }
  };
  auto put = [&](int i0) {
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int i = i0 + 256 * x;
      if (i >= all) continue;
      const Unit u = unit_at<W>(i % units, p.r.rot, p.r.interleaved);
      uint16_t* o = out + i / units * D;
      float a[W], b[W];
      if constexpr (W == 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          a[e] = act2f<DT>((ra[x][e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
          b[e] = act2f<DT>((rb[x][e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
        }
      } else {
        a[0] = act2f<DT>(ra[x]), b[0] = act2f<DT>(rb[x]);
      }
      turn<W>(u, p.r.interleaved, a, b, [&](int y) { return cs[y]; });
      if constexpr (W == 8) {
        *(u32x4*)(o + u.p0) = u32x4{pack2<DT>(a[0], a[1]), pack2<DT>(a[2], a[3]), pack2<DT>(a[4], a[5]), pack2<DT>(a[6], a[7])};
        *(u32x4*)(o + u.p1) = u32x4{pack2<DT>(b[0], b[1]), pack2<DT>(b[2], b[3]), pack2<DT>(b[4], b[5]), pack2<DT>(b[6], b[7])};
      } else {
        o[u.p0] = f2act<DT>(a[0]);
        o[u.p1] = f2act<DT>(b[0]);
      }
    }
  };
  fetch(tid);
  if (tid < half) cs[tid] = cos_sin(pos * p.r.freqs[tid], p.r.magnitude);
  __syncthreads();
  put(tid);
  for (int i0 = tid + 256 * N; i0 < all; i0 += 256 * N) {
    fetch(i0);
    put(i0);
  }
}

template <int FMT, int D>
static hipError_t append_launch(const KvAppendParams& p, hipStream_t st) {
  const dim3 grid(p.kv_blocks + p.q_blocks);
  if (p.r.rot % 16 == 0) hipLaunchKernelGGL((k_kv_append<DTC, FMT, D, 8>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((k_kv_append<DTC, FMT, D, 1>), grid, dim3(256), 0, st, p);
  return hipGetLastError();
}
hipError_t SPEAR_D(launch_kv_append)(const KvAppendParams& p, int format, hipStream_t st) {
  if (p.c.D == 64) return format == KV_INT8 ? append_launch<KV_INT8, 64>(p, st) : append_launch<KV_E4M3, 64>(p, st);
  return format == KV_INT8 ? append_launch<KV_INT8, 128>(p, st) : append_launch<KV_E4M3, 128>(p, st);
}

// ---------------------------------------------------------------------------
// Values back: sixteen tokens of one head a workgroup; V, whose places of one
// feature lie side by side, changes its order through LDS. Bound: bytes (4096 tokens of
// 8 heads, 25 MB in 6.9 us, 3.6 TB/s), latency (a few tokens 3 us).
// ---------------------------------------------------------------------------
template <int DT, int FMT, int D>
__global__ __launch_bounds__(256) void k_kv_read(KvReadParams p) {
  __shared__ uint16_t turned[16][D + 2];
  const int tid = threadIdx.x, P = p.c.P, h = blockIdx.x % p.c.Hkv, capacity = p.c.pages << p.log2_page;
  const int64_t i0 = (int64_t)(blockIdx.x / p.c.Hkv) * 16;
  auto slot_of = [&](int m) {
    const int s = i0 + m < p.n ? p.slots[i0 + m] : -1;
    return s < capacity ? s : -1;
  };
  // all loads before the first value: K's dwords of four features, V's bytes
  constexpr int U = D / 64, V = D / 16;
  uint32_t k[U], v[V];
  float k_scale[U];
  int k_slot[U];
#pragma unroll
  for (int x = 0; x < U; ++x) {
    const int i = tid + 256 * x, m = i / (D / 4), d = 4 * (i % (D / 4)), s = k_slot[x] = slot_of(m), at = max(s, 0);
    const int64_t ph = (int64_t)(at >> p.log2_page) * p.c.Hkv + h;
    k[x] = *(const uint32_t*)(p.c.k + (ph * P + (at & (P - 1))) * D + d);
    k_scale[x] = p.c.k_scale[ph];
  }
  const int m = tid & 15, d0 = tid >> 4, s = slot_of(m), at = max(s, 0);
  const int64_t ph = (int64_t)(at >> p.log2_page) * p.c.Hkv + h;
#pragma unroll
  for (int x = 0; x < V; ++x) v[x] = p.c.v[(ph * D + d0 + 16 * x) * P + (at & (P - 1))];
  const float v_scale = p.c.v_scale[ph];
#pragma unroll
  for (int x = 0; x < U; ++x) {
    const int i = tid + 256 * x;
    float c[4];
    decode4<FMT>(k[x], c);
    uint16_t* o = p.k_out + ((i0 + i / (D / 4)) * p.c.Hkv + h) * D + 4 * (i % (D / 4));
    if (k_slot[x] >= 0) *(u32x2*)o = u32x2{pack2<DT>(c[0] * k_scale[x], c[1] * k_scale[x]), pack2<DT>(c[2] * k_scale[x], c[3] * k_scale[x])};
  }
#pragma unroll
  for (int x = 0; x < V; ++x) {
    float c[4];
    decode4<FMT>(v[x], c);
    turned[m][d0 + 16 * x] = f2act<DT>(c[0] * v_scale);
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < U; ++x) {
    const int i = tid + 256 * x, m = i / (D / 4), d = 4 * (i % (D / 4));
    const uint32_t* t = (const uint32_t*)&turned[m][d];
    if (k_slot[x] >= 0) *(u32x2*)(p.v_out + ((i0 + m) * p.c.Hkv + h) * D + d) = u32x2{t[0], t[1]};
  }
}

template <int FMT, int D>
static hipError_t read_launch(const KvReadParams& p, hipStream_t st) {
  hipLaunchKernelGGL((k_kv_read<DTC, FMT, D>), dim3((uint32_t)((p.n + 15) / 16 * p.c.Hkv)), dim3(256), 0, st, p);
  return hipGetLastError();
}
hipError_t SPEAR_D(launch_kv_read)(const KvReadParams& p, int format, hipStream_t st) {
  if (p.c.D == 64) return format == KV_INT8 ? read_launch<KV_INT8, 64>(p, st) : read_launch<KV_E4M3, 64>(p, st);
  return format == KV_INT8 ? read_launch<KV_INT8, 128>(p, st) : read_launch<KV_E4M3, 128>(p, st);
}

}  // namespace spear
