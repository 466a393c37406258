// gfx950 (MI355X) kernels of attention over a paged cache held in 8 bits.
#include "spear_device.h"
#include "spear_kv_internal.h"

namespace spear {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;  // running maximum of a row that has seen nothing
// Weights are the second product's operand and held in the activation type as its MFMA takes
// it: in two parts they would take V's MFMAs twice. Error against 64 bits of ordinary calls,
// with the output's own rounding: fp16 2.1e-4 with exact weights, 2.2e-4 to 2.6e-4 with these,
// bf16 1.7e-3 and 1.9e-3 to 2.2e-3. Tiles sum them as rounded, two an instruction: what rounding
// puts on all of a row's weights alike is then not in the quotient. fp16 has nothing below
// 2^-25, where a long context's tail may have its weight (131000 tokens: up to 0.4 % of the
// largest's): weights are made against a maximum kLift powers of two lower, so that the largest is
// 2^7, in tiles 2^3, and 2^-32 or 2^-28 of it still counts (bf16 has fp32's range).
template <int DT> constexpr float kLift = DT == DT_F16 ? 7.f : 0.f;
template <int DT> constexpr float kTileLift = DT == DT_F16 ? 3.f : 0.f;
// How far scores may pass a row's maximum, in powers of two, before it is moved and
// what was summed is scaled: weights up to 2^(kLift + 8), in fp16's range.
constexpr float kSlack = 8.f;
// Where the maximum costs more than the weights: a step's weights are made against the
// maximum so far, and once more against a new one only where a row's sum of them (half
// a row's, a lane's) passes 2^12, in fp16 2^15: each weight is in its range. (With the largest
// at 2^7 that comes more often: a prompt of 4096 314 us instead of 307, 309 with 2^4.)
template <int DT> constexpr float kMostSum = DT == DT_F16 ? 32768.f : 4096.f;

#if !SPEAR_BF16_UNIT
// ---------------------------------------------------------------------------
// The plan. One workgroup: requests are told apart by their rows, all steps are
// summed, and each request's (or tile's) steps are cut into stretches of equal
// length near all steps / goal, so that workgroups have like shares whatever the
// lengths; heavy tiles (late positions) come first. Bound: latency, once for all layers:
// one request 3.6 us, 24 or 64 requests 4.2, the 128 tiles of a prompt of 4096 9.6.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024, kSizes = 32;

// sum over the workgroup before this thread, and in all
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t* red, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = v;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t o = __shfl_up(s, d);
    if (lane >= d) s += o;
  }
  __syncthreads();
  if (lane == 63) red[wave] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int i = 0; i < (int)(blockDim.x >> 6); ++i) {
    if (i < wave) before += red[i];
    all += red[i];
  }
  *total = all;
  return before + s - v;
}

__device__ __forceinline__ int plan_find(const int32_t* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// request r: its rows and positions; whatever the arrays hold, rows lie within the step
__device__ __forceinline__ AttnItem plan_request(const AttnPlanParams& p, int r) {
  AttnItem it = {};
  it.key = p.key;
  const int a = min(max(p.starts[r], 0), p.T), b = min(max(p.starts[r + 1], a), p.T);
  const int len = max(p.lens[r], 0);
  it.r = r;
  it.row0 = a;
  it.rows = min(b - a, p.max_new);
  it.pos0 = len - (b - a);
  it.end = p.pages ? (int)min(min((int64_t)len, (int64_t)p.width * p.P), (int64_t)kKvLength) : 0;  // (tokens that have a place)
  it.prefix = p.prefix ? min(max(p.prefix[r], 0), it.end) : 0;
  return it;
}
// the tokens and steps that rows i0..i1-1 of the request see; the steps' count
__device__ __forceinline__ int plan_range(const AttnPlanParams& p, AttnItem& it, int i0, int i1) {
  const int lo = it.pos0 + i0, hi = it.pos0 + i1;
  it.first = max(0, min(lo, kKvLength) - p.window + 1);
  it.end = min(it.end, max(min(hi, kKvLength), it.prefix));
  it.s0 = it.prefix > 0 ? 0 : it.first / kStep;
  it.s1 = max(it.s0, (it.end + kStep - 1) / kStep);
  return it.s1 - it.s0;
}
// the least steps of a stretch, so that `total` steps make about `goal` of them (no request has
// more steps than kKvLength's, and a sum over all of them passes 32 bits)
__device__ __forceinline__ int plan_least(int64_t total, int goal, int least) {
  return max(least, (int)min((total + goal - 1) / goal, (int64_t)(kKvLength / kStep)));
}
__device__ __forceinline__ int plan_splits(int steps, int c) { return steps > c ? (steps + c - 1) / c : 1; }
// the same of few rows, whose stretches have at least the square root of a fifth of the
// request's steps, in fours (the waves' turns): one workgroup joins them all, and a long
// request of few heads would be all joining (120000 tokens, one head: 35 us in stretches
// of 8 steps, 26 of 20)
__device__ __forceinline__ int plan_row_splits(int steps, int c) {
  return plan_splits(steps, max(c, 4 * (int)ceilf(__builtin_amdgcn_sqrtf((float)steps * 0.0125f))));
}
// stretch x of it's splits
__device__ __forceinline__ AttnItem plan_stretch(AttnItem it, int splits, int x, int part) {
  const int s0 = it.s0, n = it.s1 - it.s0;
  it.splits = splits, it.split = x, it.part = part;
  it.s0 = s0 + (int)((int64_t)n * x / splits);
  it.s1 = s0 + (int)((int64_t)n * (x + 1) / splits);
  return it;
}

// EACH: requests a thread
template <int EACH>
__global__ __launch_bounds__(kPlanThreads) void k_attention_plan(AttnPlanParams p) {
  constexpr int R = EACH * kPlanThreads;
  __shared__ int32_t s_item[R + 1], s_part[R], s_place[R], s_tile[R + 1];
  __shared__ int64_t red[kPlanThreads / 64];
  __shared__ int s_size[kSizes];
  const int tid = threadIdx.x, r0 = tid * EACH;
  // requests: steps of those of few rows, tiles of the others
  int steps[EACH], tiles[EACH];
  int64_t sum = 0, tile_sum = 0, total;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    steps[e] = -1, tiles[e] = 0;
    if (r0 + e >= p.R) continue;
    AttnItem it = plan_request(p, r0 + e);
    if (it.rows == 0) continue;
    const int64_t rows = (int64_t)it.rows * p.group;
    if (rows <= kRows) sum += steps[e] = plan_range(p, it, 0, it.rows);
    else tile_sum += tiles[e] = (int)((rows + p.z.tile_rows - 1) / p.z.tile_rows);
  }
  if (tid < kSizes) s_size[tid] = 0;
  plan_scan(sum, red, &total);
  const int c = plan_least(total, p.z.goal_rows, p.z.least_rows);
  // their stretches, long ones first: by size in kSizes classes (where a request stands
  // in its class is left to chance, and makes no difference to what is computed)
  int64_t counts = 0;  // items, and partial results in the upper half
  int place[EACH], size[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    place[e] = size[e] = 0;
    if (steps[e] < 0) continue;
    const int k = plan_row_splits(steps[e], c);
    counts += k + ((int64_t)(k > 1 ? k : 0) << 32);
    size[e] = kSizes - 1 - min((int)((int64_t)steps[e] * (kSizes - 1) / ((int64_t)c * k)), kSizes - 1);
    place[e] = atomicAdd(&s_size[size[e]], k);
  }
  int64_t at = plan_scan(counts, red, &total), tile_at = 0, n_tiles = 0;
  const int n_items = (int)(total & 0xFFFFFFFF);  // at most R + goal_rows
  if (p.z.max_tile) tile_at = plan_scan(tile_sum, red, &n_tiles);  // (uniform)
  // (more than the step's rows make: starts that contradict themselves, and no tile is
  // taken rather than some, whose counters would be left over)
  if (n_tiles > p.z.max_tile - p.z.goal_tile) n_tiles = 0;
  int before[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) before[e] = 0;
  for (int i = 0; i < kSizes; ++i) {
    const int n = s_size[i];
#pragma unroll
    for (int e = 0; e < EACH; ++e) before[e] += i < size[e] ? n : 0;
  }
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    if (r0 + e >= p.R) continue;
    s_item[r0 + e] = (int)(at & 0xFFFFFFFF);
    s_part[r0 + e] = (int)(at >> 32);
    s_place[r0 + e] = before[e] + place[e];
    s_tile[r0 + e] = (int)min(tile_at, n_tiles);
    tile_at += tiles[e];
    if (steps[e] >= 0) {
      const int k = plan_row_splits(steps[e], c);
      at += k + ((int64_t)(k > 1 ? k : 0) << 32);
    }
  }
  if (tid == 0) s_item[p.R] = n_items, s_tile[p.R] = (int)n_tiles;
  __syncthreads();
  for (int i = tid; i < n_items; i += blockDim.x) {
    const int r = plan_find(s_item, p.R, i), x = i - s_item[r];
    AttnItem it = plan_request(p, r);
    int k = plan_row_splits(plan_range(p, it, 0, it.rows), c);
    if (k > 1 && s_part[r] + k > p.z.part_rows) it.s1 = it.s0, k = 1;  // (arrays that contradict themselves)
    const int at = s_place[r];
    if (at + k > p.z.max_rows) it.key = 0;  // (more than the sizes allow: none of it)
    if (at + x < p.z.max_rows) p.items_rows[at + x] = plan_stretch(it, k, k > 1 ? x : 0, s_part[r]);
  }
  for (int i = n_items + tid; i < p.z.max_rows; i += blockDim.x) p.items_rows[i].key = 0;
  if (!p.z.max_tile) return;
  // tiles, the last first
  auto tile_of = [&](int t, AttnItem& it) {
    const int r = plan_find(s_tile, p.R, t);
    it = plan_request(p, r);
    it.tile = t - s_tile[r];
    const int64_t row = (int64_t)it.tile * p.z.tile_rows;
    if (row >= (int64_t)it.rows * p.group) it.key = 0, it.tile = 0;  // (arrays that contradict themselves)
    const int i0 = it.tile * p.z.tile_rows / p.group;
    return plan_range(p, it, i0, min(it.rows, (it.tile * p.z.tile_rows + p.z.tile_rows - 1) / p.group + 1));
  };
  sum = 0;
  AttnItem it;
  int k = 0;
  for (int t = tid; t < n_tiles; t += blockDim.x) sum += tile_of((int)n_tiles - 1 - t, it);
  plan_scan(sum, red, &total);
  const int ct = plan_least(total, p.z.goal_tile, p.z.least_tile);
  int64_t base = 0;  // as counts
  for (int t0 = 0; t0 < n_tiles; t0 += blockDim.x) {
    const int t = (int)n_tiles - 1 - t0 - tid;
    k = 0;
    if (t >= 0) k = plan_splits(n_tiles <= blockDim.x ? it.s1 - it.s0 : tile_of(t, it), ct);
    int64_t all;
    const int64_t before_me = base + plan_scan(k + ((int64_t)(k > 1 ? k : 0) << 32), red, &all);
    base += all;
    int i = (int)(before_me & 0xFFFFFFFF);
    const int part = (int)(before_me >> 32);
    const bool room = k <= 1 || part + k <= p.z.part_tile;
    if (!room) it.s1 = it.s0;
    if (k > p.z.max_tile - i) it.key = 0;  // (more than the sizes allow: none of it)
    for (int x = 0; x < k && i < p.z.max_tile; ++x, ++i)
      p.items_tile[i] = plan_stretch(it, room ? k : 1, room ? x : 0, part);
  }
  for (int i = (int)(base & 0xFFFFFFFF) + tid; i < p.z.max_tile; i += blockDim.x) p.items_tile[i].key = 0;
}

hipError_t launch_attention_plan(const AttnPlanParams& p, hipStream_t st) {
  const int want = std::min(kPlanThreads, std::max({p.R, p.z.max_rows, p.z.max_tile, kSizes}));
  const dim3 threads((want + 63) / 64 * 64);
  if (p.R > kPlanThreads) hipLaunchKernelGGL(k_attention_plan<4>, dim3(1), threads, 0, st, p);
  else hipLaunchKernelGGL(k_attention_plan<1>, dim3(1), threads, 0, st, p);
  return hipGetLastError();
}
#endif

// ---------------------------------------------------------------------------
// Codes as operands: eight codes in the activation type. K's scale goes on the
// fp32 score. V's goes on V (exact: a power of two; of INT8 codes in fp16 a scale
// from 2^-14 on, what is below on the weight) or, where a code of INT8 becomes bf16
// and a product more would be an instruction for two codes, on the weight.
// ---------------------------------------------------------------------------
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));

template <int DT, int FMT>
__device__ __forceinline__ u32x4 operand8(uint32_t w0, uint32_t w1, float scale) {
  if constexpr (FMT == KV_E4M3) {
    if constexpr (DT == DT_F16)
      return u32x4{__builtin_bit_cast(uint32_t, (h16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, scale, false)),
                   __builtin_bit_cast(uint32_t, (h16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, scale, true)),
                   __builtin_bit_cast(uint32_t, (h16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, scale, false)),
                   __builtin_bit_cast(uint32_t, (h16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, scale, true))};
    else
      return u32x4{__builtin_bit_cast(uint32_t, (b16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false)),
                   __builtin_bit_cast(uint32_t, (b16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true)),
                   __builtin_bit_cast(uint32_t, (b16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false)),
                   __builtin_bit_cast(uint32_t, (b16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true))};
  } else {
    return i8x8_exact<DT>(w0, w1);
  }
}
template <int DT, int FMT>
__device__ __forceinline__ u32x4 v_operand8(uint32_t w0, uint32_t w1, float scale) {
  u32x4 x = operand8<DT, FMT>(w0, w1, scale);
  if constexpr (DT == DT_F16 && FMT == KV_INT8) {
    const h16x2 s = h16x2{(_Float16)scale, (_Float16)scale};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t e = x[i];  // (this clang's bit_cast of an element of a vector takes the first one)
      x[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2, e) * s);
    }
  }
  return x;
}
// V's scale as (factor of V, factor of the weight)
template <int DT, int FMT>
__device__ __forceinline__ float2 v_factors(float s) {
  if constexpr (FMT == KV_E4M3) return make_float2(s, 1.f);  // (one rounding to the activation type, with the code's)
  else if constexpr (DT == DT_F16) return make_float2(fmaxf(s, 6.103515625e-5f), fminf(s * 16384.f, 1.f));
  else return make_float2(1.f, s);
}

template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (DT == DT_F16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, h16x2));
  else
    return pack_bf16(a, b);
}

// the larger of the two halves of a wave, and of its four sixteens
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_sixteens(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// c plus both weights of a pair, as they are held
template <int DT>
__device__ __forceinline__ float add2(uint32_t pair, float c) {
  if constexpr (DT == DT_F16)
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(h16x2, pair), h16x2{(_Float16)1.f, (_Float16)1.f}, c, false);
  else
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b16x2, pair), b16x2{(__bf16)1.f, (__bf16)1.f}, c, false);
}

// a pair of fp16 weights times a power of two of at most one
__device__ __forceinline__ uint32_t scaled2(uint32_t pair, float f) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2, pair) * h16x2{(_Float16)f, (_Float16)f});
}

// A score in powers of two. OPT: capped, or biased by distance.
struct ScoreOptions {
  float scale, cap, inv_cap, slope2;  // slope2: slope times log2 e
};
// (of a plain score all but the dot product is one factor: at least the least float,
// which makes no difference to a score of scale zero, and keeps what is masked, minus
// infinity, from a product with zero and from a page's scale that is no number)
__device__ __forceinline__ float dot_factor(float k_scale, const ScoreOptions& o) {
  return fmaxf(k_scale * (o.scale * kLog2e), 1.17549435e-38f);
}
// cap tanh(z), z = t / cap: cap (1 - 2 / (e^2z + 1)), off by some 2^-23 cap (the reciprocal
// instruction's last place with it), which leaves nothing of a score far below the cap (at a cap
// of 10^4 a score was off by 10^-3, at 10^8 it was gone). Below a quarter of the cap Taylor's
// sum t (1 - z^2/3 + 2 z^4/15 - 17 z^6/315 + 62 z^8/2835), whose next term is 10^-8 at most.
__device__ __forceinline__ float capped(float t, const ScoreOptions& o) {
  const float z = t * o.inv_cap, y = z * z;
  const float near = t * (1.f + y * (-1.f / 3 + y * (2.f / 15 + y * (-17.f / 315 + y * (62.f / 2835)))));
  const float far = o.cap * (1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * (2.f * kLog2e)) + 1.f));
  return fabsf(z) < 0.25f ? near : far;
}
__device__ __forceinline__ float score2(float dot, float k_scale, const ScoreOptions& o, int pos, int j) {
  float t = dot * (k_scale * o.scale);
  if (o.cap > 0.f) t = capped(t, o);
  return t * kLog2e - o.slope2 * (float)abs(pos - j);
}

// Kernel arguments are read where the compiler first needs them, and a line of them
// not yet read is another trip to memory: what is used late is asked for at the start,
// with the rest (one request of 500 tokens 5.84 us, 5.68 this way).
__device__ __forceinline__ void early(const AttnParams& p) {
  asm volatile("" ::"s"(p.window), "s"(p.out), "s"(p.out_ld), "s"(p.slopes), "s"(p.softcap), "s"(p.inv_cap), "s"(p.scale));
  asm volatile("" ::"s"(p.counters_rows), "s"(p.counters_tile), "s"(p.parts_rows), "s"(p.parts_tile));
}

// an item of the plan, by scalar loads (a launch only reads plans)
__device__ __forceinline__ AttnItem item_at(const AttnItem* items, int idx) {
  typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
  static_assert(sizeof(AttnItem) == sizeof(u32x16), "one load");
  return __builtin_bit_cast(AttnItem, *(const __attribute__((address_space(4))) u32x16*)(uintptr_t)(items + idx));
}

// Masks of tokens as bits, bit e of token j + e. (Compact code counts here: a call of
// few steps spends its time on fetching what it runs once, and the last step of every
// row is a masked one; compared and selected one by one this cost 3 us a call.)
__device__ __forceinline__ uint32_t below(int x) { return (uint32_t)((1ull << min(max(x, 0), 32)) - 1); }
// tokens that some row of the item sees
__device__ __forceinline__ uint32_t live_tokens(int j, const AttnItem& it) {
  return (below(it.end - j) & ~below(it.first - j)) | below(it.prefix - j);
}
// tokens that the row at pos sees
__device__ __forceinline__ uint32_t seen_tokens(int j, const AttnItem& it, int pos, int window) {
  return ((below(pos + 1 - j) & ~below(pos - window + 1 - j)) | below(it.prefix - j)) & below(it.end - j);
}
// x where bit e of the mask is set, else minus infinity
__device__ __forceinline__ float where_seen(float x, uint32_t mask, int e) {
  const uint32_t m = (uint32_t)((int)(mask << (31 - e)) >> 31);
  return __uint_as_float((__float_as_uint(x) & m) | (0xFF800000u & ~m));
}
// sixteen bits as bytes of four dwords
__device__ __forceinline__ u32x4 byte_mask(uint32_t bits) {
  u32x4 m;
#pragma unroll
  for (int w = 0; w < 4; ++w) m[w] = ((((bits >> (4 * w)) & 15u) * 0x00204081u) & 0x01010101u) * 0xFFu;
  return m;
}

// ---------------------------------------------------------------------------
// At most 16 rows (decode): four waves, each a step of 64 tokens in turn, its
// codes in registers and those of the next step in flight. S^T = K Q^T and
// O^T = V^T P^T on 16 x 16 x 32 MFMAs: with the tokens as rows of S^T a lane holds
// 16 scores of one row, of 16 tokens that lie side by side, so that the weights
// are V's operand as they are, a page's scale is one number a lane, and K and V
// come in pieces of 16 bytes. The waves' and then the stretches' results are
// joined in order, the latter by the stretch that ends last.
// Bound: the codes' bytes (long caches: one request of 131000 tokens, 8 heads of 128,
// 268 MB in 52 us, 5.1 TB/s, in replays of a graph 55, where the loads alone take as long;
// 64 requests of up to 8192 tokens, 155 MB in 31 us, 5.0 TB/s, and 34), latency (one request
// of 500 tokens: 5.7 us in a graph).
// K goes through LDS so that V has the registers to be a step ahead (with both in
// registers, and stretches in the requests' order, these 64 took 45 us).
// ---------------------------------------------------------------------------
constexpr int kWaves = 4;  // of a workgroup of k_attend_rows and k_attend_mid
// LDS of either: K of each wave's step, then each wave's O
template <int D, int ROWS>
constexpr int few_lds() { return kWaves * std::max(kStep * D, ROWS * (D + 4) * 4); }

template <int DT, int FMT, int D, bool OPT>
__device__ __forceinline__ void attend_rows(const AttnParams& p, uint32_t block, char* lds, float* s_m, float* s_l, int* s_last) {
  constexpr int W = kWaves, KS = D / 64, DTILES = D / 16, PITCH = D + 4, KBYTES = kStep * D;
  float* s_o = (float*)lds;
  const int head = block % p.c.Hkv, idx = block / p.c.Hkv;
  AttnItem it = item_at(p.items_rows, idx);
  if (it.key != p.key) return;
  if (p.c.pages == 0) it.s1 = it.s0;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int P = p.c.P, live_rows = it.rows * p.group;
  const bool mine = c < live_rows;
  const int i = mine ? c / p.group : 0, hq = head * p.group + (mine ? c % p.group : 0);
  const uint32_t sign = p.scale < 0.f ? 0x80008000u : 0u;  // (a scale below zero: of q)
  u32x4 q[2 * KS];
  {
    const uint16_t* qp = p.q + (int64_t)(it.row0 + i) * p.q_ld + hq * D + 16 * g;
#pragma unroll
    for (int s = 0; s < 2 * KS; ++s) q[s] = ldg16(qp + 64 * (s >> 1) + 8 * (s & 1)) ^ sign;
    if (!mine)
#pragma unroll
      for (int s = 0; s < 2 * KS; ++s) q[s] = u32x4{0, 0, 0, 0};
  }
  const int pos = it.pos0 + i, pos_max = it.pos0 + it.rows - 1;
  const ScoreOptions opt{fabsf(p.scale), p.softcap, p.inv_cap, OPT && p.slopes ? p.slopes[hq] * kLog2e : 0.f};
  const int32_t* table = p.table + it.r * p.ld;
  const uint32_t page_bytes = P * D, pool_bytes = p.c.Hkv * page_bytes;
  const uint8_t *k_head = p.c.k + (int64_t)head * page_bytes, *v_head = p.c.v + (int64_t)head * page_bytes;

  // the table's entry of the lane's run of 16 tokens, run g, and whether it is a page
  // (looked at only where it is used: a comparison here would wait for the load)
  auto entry_at = [&](int s) {
    const int j = s * kStep + 16 * g;
    int page = -1;
    if (s < it.s1 && j < it.end) page = table[j >> p.log2_page];
    return page;
  };
  auto page_of = [&](int entry) { return (uint32_t)entry < (uint32_t)p.c.pages ? entry : -1; };
  // K straight to LDS, a KB an instruction from tokens that lie side by side; the
  // pieces of token t stand in the order piece ^ turn(t), so that the sixteen tokens
  // that a sixteen of lanes reads lie in different banks
  auto turn = [](int t) { return D == 128 ? ((t >> 4) & 3) | ((t >> 1) & 1) << 2 : (t >> 4) & 3; };
  char* const s_k = lds + wave * KBYTES;
  constexpr int PIECES = D / 16, TOKENS = 64 / PIECES;  // of a token; tokens an instruction
  auto load_k = [&](int s, int page) {
#pragma unroll
    for (int x = 0; x < kStep / TOKENS; ++x) {
      const int run = x * TOKENS / 16, in_run = x * TOKENS % 16 + lane / PIECES;
      const int pg = max(__builtin_amdgcn_readlane(page, 16 * run), 0);
      const uint8_t* k = k_head + (uint64_t)pg * pool_bytes + ((s * kStep + 16 * run) & (P - 1)) * D;
      const uint8_t* from = k + (in_run * D + 16 * ((lane % PIECES) ^ turn(16 * run + in_run)));
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                       (__attribute__((address_space(3))) void*)(s_k + 1024 * x), 16, 0, 2);
    }
  };
  u32x4 vr[DTILES], vn[DTILES];  // V of this step, and of the next
  auto load_v = [&](u32x4 (&vr)[DTILES], int s, int page) {
    const int at = (s * kStep + 16 * g) & (P - 1);
    const uint8_t* v = v_head + (uint64_t)(uint32_t)max(page, 0) * pool_bytes + (c * P + at);
#pragma unroll
    for (int d = 0; d < DTILES; ++d) vr[d] = __builtin_nontemporal_load((const u32x4*)(v + d * 16 * P));
  };
  auto scales = [&](int page) {
    const int64_t ph = (int64_t)max(page, 0) * p.c.Hkv + head;
    return make_float2(p.c.k_scale[ph], p.c.v_scale[ph]);
  };

  f32x4 o[DTILES] = {};
  float m = kLowest, l = 0.f;
  int s = it.s0 + wave;
  if (s < it.s1) {
    int page = page_of(entry_at(s)), next, entry;
    float2 sn = {};
    load_k(s, page);
    float2 sc = scales(page);
    load_v(vr, s, page);
    next = page;
    entry = entry_at(s + W);
    for (; s < it.s1; s += W) {
      f32x4 st[4] = {};
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int token = 16 * (c >> 2) + 4 * t + (c & 3);
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          const u32x4 k = *(const u32x4*)(s_k + token * D + 16 * ((g + 4 * x) ^ turn(token)));
          st[t] = mfma16<DT>(operand8<DT, FMT>(k[0], k[1], 1.f), q[2 * x], st[t]);
          st[t] = mfma16<DT>(operand8<DT, FMT>(k[2], k[3], 1.f), q[2 * x + 1], st[t]);
        }
      }
      const bool more = s + W < it.s1;
      if (more) {
        __builtin_amdgcn_s_waitcnt(0xC07F);  // this wave's reads of K have left LDS (lgkmcnt 0)
        next = page_of(entry);
        load_k(s + W, next);
        load_v(vn, s + W, next);
        sn = scales(next);
        entry = entry_at(s + 2 * W);
      }
      const int j0 = s * kStep + 16 * g;
      // every row sees every token of the step, all pages are there
      const bool whole = s * kStep + kStep <= min(it.end, it.pos0 + 1) && pos_max - s * kStep < p.window &&
                         __all(page >= 0);
      float2 f = v_factors<DT, FMT>(sc.y);
      const float fk = OPT ? 1.f : dot_factor(sc.x, opt);  // what st is of a score
      if constexpr (OPT) {
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e >> 2][e & 3] = score2(st[e >> 2][e & 3], sc.x, opt, pos, j0 + e);
      }
      if (!whole) {
        const uint32_t there = page >= 0 ? 0xFFFFu : 0u, live = live_tokens(j0, it) & there;
        const uint32_t sees = seen_tokens(j0, it, pos, p.window) & there;
        if (!live) f = make_float2(1.f, 1.f);
        const u32x4 bytes = byte_mask(live);
#pragma unroll
        for (int d = 0; d < DTILES; ++d) vr[d] &= bytes;
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e >> 2][e & 3] = where_seen(st[e >> 2][e & 3], sees, e);
      }
      float top = st[0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, st[e >> 2][e & 3]);
      top *= fk;
      top = max_sixteens(top);
      if (__any(top > m + (kLift<DT> + kSlack))) {
        const float now = fmaxf(m, top - kLift<DT>), fade = __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= fade;
#pragma unroll
        for (int d = 0; d < DTILES; ++d) o[d] *= fade;
      }
      float w[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e >> 2][e & 3], fk, -m));
        l += w[e];
      }
      if (FMT == KV_INT8 && (DT != DT_F16 || __any(f.y != 1.f))) {
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] *= f.y;
      }
      u32x4 pw[2];
#pragma unroll
      for (int e = 0; e < 8; ++e) pw[e >> 2][e & 3] = pack2<DT>(w[2 * e], w[2 * e + 1]);
#pragma unroll
      for (int d = 0; d < DTILES; ++d) {
        o[d] = mfma16<DT>(v_operand8<DT, FMT>(vr[d][0], vr[d][1], f.x), pw[0], o[d]);
        o[d] = mfma16<DT>(v_operand8<DT, FMT>(vr[d][2], vr[d][3], f.x), pw[1], o[d]);
      }
      page = next, sc = sn;
#pragma unroll
      for (int d = 0; d < DTILES; ++d) vr[d] = vn[d];
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  __syncthreads();
#pragma unroll
  for (int d = 0; d < DTILES; ++d) *(f32x4*)&s_o[(wave * kRows + c) * PITCH + 16 * d + 4 * g] = o[d];
  if (g == 0) s_m[wave * kRows + c] = m, s_l[wave * kRows + c] = l;
  __syncthreads();
  // Eight features a thread: D / 8 threads a row, the rows that are there, and so
  // many groups of threads as the workgroup holds, which share the partial results.
  constexpr int F = 8, CHUNKS = D / F;
  const int per = live_rows * CHUNKS, groups = 64 * W / per, part = tid / per;
  const int row = tid % per / CHUNKS, d0 = tid % CHUNKS * F;
  float top = kLowest, x[F] = {}, total = 0.f;
  // one more result of maximum pm and sum pl, its features v
  auto add = [&](float pm, float pl, const float (&v)[F]) {
    const float now = fmaxf(top, pm), f0 = __builtin_amdgcn_exp2f(top - now), f1 = __builtin_amdgcn_exp2f(pm - now);
    top = now;
    total = total * f0 + pl * f1;
#pragma unroll
    for (int e = 0; e < F; ++e) x[e] = x[e] * f0 + v[e] * f1;
  };
  if (part == 0) {
#pragma unroll
    for (int v = 0; v < W; ++v) {
      float y[F];
#pragma unroll
      for (int e = 0; e < F; ++e) y[e] = s_o[(v * kRows + row) * PITCH + d0 + e];
      add(s_m[v * kRows + row], s_l[v * kRows + row], y);
    }
  }
  if (it.splits > 1) {
    const uint32_t size = kRows * (D + 2) * 4, slot = (uint32_t)it.part * p.c.Hkv + head;
    const rsrc_t r = make_rsrc((const char*)p.parts_rows + (size_t)slot * size, (uint32_t)((it.splits - 1) * p.c.Hkv + 1) * size);
    const uint32_t at = (uint32_t)it.split * p.c.Hkv * size;
    if (part == 0) {
#pragma unroll
      for (int e = 0; e < F; e += 4) bst128c(r, at + (row * D + d0 + e) * 4, f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]});
      float* ml = p.parts_rows + ((size_t)slot * size + at) / 4 + kRows * D;
      if (d0 == 0) st_agent(ml + row, top), st_agent(ml + kRows + row, total);
    }
    complete_and_sync();
    if (tid == 0) *s_last = arrive_last(p.counters_rows + slot, it.splits);
    __syncthreads();
    if (!*s_last) return;
    // group `part` takes every groups-th stretch in order, N in flight; then the groups in order
    constexpr int N = 8;
    total = 0.f;
    top = kLowest;
#pragma unroll
    for (int e = 0; e < F; ++e) x[e] = 0.f;
    const uint32_t stride = p.c.Hkv * size, own = (row * D + d0) * 4, own_m = (kRows * D + row) * 4;
    for (int b = part < groups ? part : it.splits; b < it.splits; b += N * groups) {
      f32x4 v[N][F / 4];
      float pm[N], pl[N];
#pragma unroll
      for (int y = 0; y < N; ++y) {
        const uint32_t off = b + y * groups < it.splits ? (b + y * groups) * stride : kOOB;
        pm[y] = __uint_as_float(bld32c(r, off + own_m));
        pl[y] = __uint_as_float(bld32c(r, off + own_m + kRows * 4));
#pragma unroll
        for (int e = 0; e < F / 4; ++e) v[y][e] = bld128cf(r, off + own + 16 * e);
      }
#pragma unroll
      for (int y = 0; y < N; ++y) {
        if (b + y * groups >= it.splits) continue;
        const float z[F] = {v[y][0][0], v[y][0][1], v[y][0][2], v[y][0][3], v[y][1][0], v[y][1][1], v[y][1][2], v[y][1][3]};
        add(pm[y], pl[y], z);
      }
    }
    static_assert(64 * W / CHUNKS <= W * kRows, "a place in s_o for each row of each group");
    if (part < groups) {
#pragma unroll
      for (int e = 0; e < F; ++e) s_o[(part * live_rows + row) * PITCH + d0 + e] = x[e];
      if (d0 == 0) s_m[part * live_rows + row] = top, s_l[part * live_rows + row] = total;
    }
    __syncthreads();
    if (part == 0) {
      total = 0.f;
      top = kLowest;
#pragma unroll
      for (int e = 0; e < F; ++e) x[e] = 0.f;
      for (int b = 0; b < groups; ++b) {
        float y[F];
#pragma unroll
        for (int e = 0; e < F; ++e) y[e] = s_o[(b * live_rows + row) * PITCH + d0 + e];
        add(s_m[b * live_rows + row], s_l[b * live_rows + row], y);
      }
    }
  }
  if (part) return;
  const float inv = total > 0.f ? 1.f / total : 0.f;
  uint16_t* out = p.out + (int64_t)(it.row0 + row / p.group) * p.out_ld + (head * p.group + row % p.group) * D + d0;
  *(u32x4*)out = u32x4{pack2<DT>(x[0] * inv, x[1] * inv), pack2<DT>(x[2] * inv, x[3] * inv),
                       pack2<DT>(x[4] * inv, x[5] * inv), pack2<DT>(x[6] * inv, x[7] * inv)};
}

// ---------------------------------------------------------------------------
// Tiles of 32 rows (some new tokens, chunks too few to fill the GPU in tiles of
// 256): as attend_rows, four waves with a step each in turn, K by way of LDS, V in
// registers, on 32 x 32 x 16 MFMAs. The order in which K's tokens are read from LDS is that which
// leaves a lane the scores of sixteen tokens side by side, run 2t + h of the step.
// Tiles of 32 rows and not more: more workgroups, and two of them to a SIMD's registers
// (a chunk of 512 beside 8 requests 31 us, 45 in tiles of 64).
// Bound: the conversions and exponentials beside the MFMAs; that chunk, 12.6 GFLOP, 8
// heads on one: 28.3 us, 445 TFLOP/s.
// ---------------------------------------------------------------------------
template <int DT, int FMT, int D, bool OPT>
__device__ __forceinline__ void attend_mid(const AttnParams& p, uint32_t block, char* lds, float* s_m, float* s_l, int* s_last) {
  constexpr int W = kWaves, Y = kMidRows / 32, DTILES = D / 32, KX = D / 32, PITCH = D + 4, KBYTES = kStep * D;
  float* s_o = (float*)lds;
  const int head = block % p.c.Hkv, idx = block / p.c.Hkv;
  AttnItem it = item_at(p.items_tile, idx);
  if (it.key != p.key) return;
  if (p.c.pages == 0) it.s1 = it.s0;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const int P = p.c.P, tile_row = it.tile * kMidRows, live_rows = min(it.rows * p.group - tile_row, kMidRows);
  const uint32_t sign = p.scale < 0.f ? 0x80008000u : 0u;  // (a scale below zero: of q)
  const float scale = fabsf(p.scale);
  u32x4 q[Y][2 * KX];
  int pos[Y];
  float slope2[Y];
#pragma unroll
  for (int y = 0; y < Y; ++y) {
    const bool mine = 32 * y + c < live_rows;
    const int row = tile_row + (mine ? 32 * y + c : 0), i = row / p.group, hq = head * p.group + row % p.group;
    const uint16_t* qp = p.q + (int64_t)(it.row0 + i) * p.q_ld + hq * D + 16 * h;
#pragma unroll
    for (int x = 0; x < 2 * KX; ++x) {
      q[y][x] = ldg16(qp + 32 * (x >> 1) + 8 * (x & 1)) ^ sign;
      if (!mine) q[y][x] = u32x4{0, 0, 0, 0};
    }
    pos[y] = it.pos0 + i;
    slope2[y] = OPT && p.slopes ? p.slopes[hq] * kLog2e : 0.f;
  }
  const int pos_lo = it.pos0 + tile_row / p.group, pos_hi = it.pos0 + (tile_row + live_rows - 1) / p.group;
  const int32_t* table = p.table + it.r * p.ld;
  const uint32_t page_bytes = P * D, pool_bytes = p.c.Hkv * page_bytes;
  const uint8_t *k_head = p.c.k + (int64_t)head * page_bytes, *v_head = p.c.v + (int64_t)head * page_bytes;

  // table entry of run lane / 16; pages of all four runs, uniform
  auto entry_at = [&](int s) {
    const int j = s * kStep + 16 * (lane >> 4);
    int page = -1;
    if (s < it.s1 && j < it.end) page = table[j >> p.log2_page];
    return page;
  };
  typedef int Pages __attribute__((ext_vector_type(4)));
  auto pages_of = [&](int entry) {
    auto page = [&](int e) { return (uint32_t)e < (uint32_t)p.c.pages ? e : -1; };
    return Pages{page(__builtin_amdgcn_readlane(entry, 0)), page(__builtin_amdgcn_readlane(entry, 16)),
                 page(__builtin_amdgcn_readlane(entry, 32)), page(__builtin_amdgcn_readlane(entry, 48))};
  };
  // the lane's run 2t + h. (As an array indexed by h the pages went to LDS by way of the
  // workgroup's size, which is read from host memory: 19 us instead of 5 at 64 x 64 tokens.)
  auto mine_of = [&](const Pages& pg, int t) {
    const int a = t ? pg.z : pg.x, b = t ? pg.w : pg.y;
    return h ? b : a;
  };
  // K to LDS as in k_attend_rows; here the sixteen tokens that a sixteen of lanes reads
  // are four times four, 4 and 16 apart
  auto turn = [](int t) { return D == 128 ? ((t >> 1) & 3) | ((t >> 4) & 1) << 2 : ((t >> 2) & 1) | ((t >> 4) & 1) << 1; };
  char* const s_k = lds + wave * KBYTES;
  constexpr int PIECES = D / 16, TOKENS = 64 / PIECES;
  auto load_k = [&](int s, const Pages& pg) {
#pragma unroll
    for (int x = 0; x < kStep / TOKENS; ++x) {
      const int run = x * TOKENS / 16, in_run = x * TOKENS % 16 + lane / PIECES;
      const uint8_t* k = k_head + (uint64_t)(uint32_t)max(pg[run], 0) * pool_bytes + ((s * kStep + 16 * run) & (P - 1)) * D;
      const uint8_t* from = k + (in_run * D + 16 * ((lane % PIECES) ^ turn(16 * run + in_run)));
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                       (__attribute__((address_space(3))) void*)(s_k + 1024 * x), 16, 0, 0);
    }
  };
  u32x4 vr[2][DTILES];  // V of this step, run 2t + h
  auto load_v = [&](int s, const Pages& pg) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int page = max(mine_of(pg, t), 0), at = (s * kStep + 32 * t + 16 * h) & (P - 1);
      const uint8_t* from = v_head + (uint64_t)(uint32_t)page * pool_bytes + (c * P + at);
#pragma unroll
      for (int d = 0; d < DTILES; ++d) vr[t][d] = ldg16(from + d * 32 * P);
    }
  };
  struct Scales {
    float2 at[2];
  };
  auto scales = [&](const Pages& pg) {
    Scales r;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint64_t ph = (uint64_t)(uint32_t)max(mine_of(pg, t), 0) * p.c.Hkv + head;
      r.at[t] = make_float2(p.c.k_scale[ph], p.c.v_scale[ph]);
    }
    return r;
  };

  f32x16 o[Y][DTILES] = {};
  float m[Y], l[Y];
#pragma unroll
  for (int y = 0; y < Y; ++y) m[y] = kLowest, l[y] = 0.f;
  int s = it.s0 + wave;
  if (s < it.s1) {
    Pages page = pages_of(entry_at(s)), next = page;
    load_k(s, page);
    Scales sc = scales(page), sn = sc;
    int entry = entry_at(s + W);
    for (; s < it.s1; s += W) {
      f32x16 st[Y][2] = {};  // [32 rows][32 tokens]
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int token = 32 * t + 16 * ((c >> 2) & 1) + 4 * (c >> 3) + (c & 3);
#pragma unroll
        for (int x = 0; x < KX; ++x) {
          const u32x4 k = *(const u32x4*)(s_k + token * D + 16 * ((2 * x + h) ^ turn(token)));
          const u32x4 a = operand8<DT, FMT>(k[0], k[1], 1.f), b = operand8<DT, FMT>(k[2], k[3], 1.f);
#pragma unroll
          for (int y = 0; y < Y; ++y) st[y][t] = mfma32<DT>(a, q[y][2 * x], st[y][t]);
#pragma unroll
          for (int y = 0; y < Y; ++y) st[y][t] = mfma32<DT>(b, q[y][2 * x + 1], st[y][t]);
        }
      }
      load_v(s, page);
      const bool more = s + W < it.s1;
      if (more) {
        __builtin_amdgcn_s_waitcnt(0xC07F);  // this wave's reads of K have left LDS (lgkmcnt 0)
        next = pages_of(entry);
        load_k(s + W, next);
        sn = scales(next);
        entry = entry_at(s + 2 * W);
      }
      const int j0 = s * kStep;
      const bool whole = j0 + kStep <= min(it.end, pos_lo + 1) && pos_hi - j0 < p.window &&
                         (page.x | page.y | page.z | page.w) >= 0;
      float2 f[2] = {v_factors<DT, FMT>(sc.at[0].y), v_factors<DT, FMT>(sc.at[1].y)};
      uint32_t there[2];
      if (!whole) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          there[t] = mine_of(page, t) >= 0 ? 0xFFFFu : 0u;
          const uint32_t live = live_tokens(j0 + 32 * t + 16 * h, it) & there[t];
          if (!live) f[t] = make_float2(1.f, 1.f);
          const u32x4 bytes = byte_mask(live);
#pragma unroll
          for (int d = 0; d < DTILES; ++d) vr[t][d] &= bytes;
        }
      }
      u32x4 pw[Y][4];  // weights: [32 rows][eight tokens of either run]
#pragma unroll
      for (int y = 0; y < Y; ++y) {
        const ScoreOptions opt{scale, p.softcap, p.inv_cap, slope2[y]};
        float g[2];  // what st is of a score
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          g[t] = OPT ? 1.f : dot_factor(sc.at[t].x, opt);
          if constexpr (OPT) {
#pragma unroll
            for (int e = 0; e < 16; ++e) st[y][t][e] = score2(st[y][t][e], sc.at[t].x, opt, pos[y], j0 + 32 * t + 16 * h + e);
          }
          if (!whole) {
            const uint32_t sees = seen_tokens(j0 + 32 * t + 16 * h, it, pos[y], p.window) & there[t];
#pragma unroll
            for (int e = 0; e < 16; ++e) st[y][t][e] = where_seen(st[y][t][e], sees, e);
          }
        }
        // a step's weights against the maximum so far, and once more where a sum passes
        float sum;
        for (int pass = 0;; ++pass) {
          sum = 0.f;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float u = __builtin_amdgcn_exp2f(__builtin_fmaf(st[y][t][2 * e], g[t], -m[y]));
              const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(st[y][t][2 * e + 1], g[t], -m[y]));
              if constexpr (DT != DT_F16 && FMT == KV_INT8) {
                sum += u + v;
                pw[y][2 * t + (e >> 2)][e & 3] = pack2<DT>(u * f[t].y, v * f[t].y);
              } else {
                const uint32_t w = pack2<DT>(u, v);
                sum = add2<DT>(w, sum);
                pw[y][2 * t + (e >> 2)][e & 3] = DT == DT_F16 && FMT == KV_INT8 ? scaled2(w, f[t].y) : w;
              }
            }
          if (pass || !__any(!(sum <= kMostSum<DT>))) break;
          float top = kLowest;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            float x = st[y][t][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) x = fmaxf(x, st[y][t][e]);
            top = fmaxf(top, x * g[t]);
          }
          const float now = fmaxf(m[y], max_halves(top) - kTileLift<DT>), fade = __builtin_amdgcn_exp2f(m[y] - now);
          m[y] = now;
          l[y] *= fade;
#pragma unroll
          for (int d = 0; d < DTILES; ++d) o[y][d] *= fade;
        }
        l[y] += sum;
      }
      __builtin_amdgcn_sched_barrier(0);  // (V's operands made ahead of the softmax would not fit the registers)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < DTILES; ++d) {
          const u32x4 a = v_operand8<DT, FMT>(vr[t][d][0], vr[t][d][1], f[t].x), b = v_operand8<DT, FMT>(vr[t][d][2], vr[t][d][3], f[t].x);
#pragma unroll
          for (int y = 0; y < Y; ++y) o[y][d] = mfma32<DT>(a, pw[y][2 * t], o[y][d]);
#pragma unroll
          for (int y = 0; y < Y; ++y) o[y][d] = mfma32<DT>(b, pw[y][2 * t + 1], o[y][d]);
        }
      page = next, sc = sn;
    }
  }
  __syncthreads();
#pragma unroll
  for (int y = 0; y < Y; ++y) {
    l[y] += __shfl_xor(l[y], 32);
    const int at = wave * kMidRows + 32 * y + c;
#pragma unroll
    for (int d = 0; d < DTILES; ++d)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *(f32x4*)&s_o[at * PITCH + 32 * d + 8 * x + 4 * h] = f32x4{o[y][d][4 * x], o[y][d][4 * x + 1], o[y][d][4 * x + 2], o[y][d][4 * x + 3]};
    if (h == 0) s_m[at] = m[y], s_l[at] = l[y];
  }
  __syncthreads();
  // a thread: a row, every EACH-th of its runs of four features
  constexpr int EACH = 256 / kMidRows, F = D / 4 / EACH;
  const int row = tid / EACH, own = tid % EACH;
  f32x4 x[F] = {};
  float top = kLowest, total = 0.f;
  auto add = [&](float pm, float pl, const f32x4 (&v)[F]) {
    const float now = fmaxf(top, pm), f0 = __builtin_amdgcn_exp2f(top - now), f1 = __builtin_amdgcn_exp2f(pm - now);
    top = now;
    total = total * f0 + pl * f1;
#pragma unroll
    for (int e = 0; e < F; ++e) x[e] = x[e] * f0 + v[e] * f1;
  };
#pragma unroll
  for (int v = 0; v < W; ++v) {
    f32x4 y[F];
#pragma unroll
    for (int e = 0; e < F; ++e) y[e] = *(const f32x4*)&s_o[(v * kMidRows + row) * PITCH + 4 * (EACH * e + own)];
    add(s_m[v * kMidRows + row], s_l[v * kMidRows + row], y);
  }
  if (it.splits > 1) {
    const uint32_t size = kMidRows * (D + 2) * 4, slot = (uint32_t)it.part * p.c.Hkv + head, stride = p.c.Hkv * size;
    const rsrc_t r = make_rsrc((const char*)p.parts_tile + (size_t)slot * size, (uint32_t)((it.splits - 1) * p.c.Hkv + 1) * size);
    const uint32_t at = (uint32_t)it.split * stride, mine = (row * D + 4 * own) * 4, mine_m = (kMidRows * D + row) * 4;
    if (row < live_rows) {
#pragma unroll
      for (int e = 0; e < F; ++e) bst128c(r, at + mine + 16 * EACH * e, x[e]);
      float* ml = p.parts_tile + ((size_t)slot * size + at + mine_m) / 4;
      if (own == 0) st_agent(ml, top), st_agent(ml + kMidRows, total);
    }
    complete_and_sync();
    if (tid == 0) *s_last = arrive_last(p.counters_tile + slot, it.splits);
    __syncthreads();
    if (!*s_last) return;
    top = kLowest, total = 0.f;
#pragma unroll
    for (int e = 0; e < F; ++e) x[e] = f32x4{};
    constexpr int N = 4;  // stretches in flight, joined in order
    for (int b = 0; b < it.splits; b += N) {
      f32x4 v[N][F];
      float pm[N], pl[N];
#pragma unroll
      for (int y = 0; y < N; ++y) {
        const uint32_t off = b + y < it.splits && row < live_rows ? (b + y) * stride : kOOB;
        pm[y] = __uint_as_float(bld32c(r, off + mine_m));
        pl[y] = __uint_as_float(bld32c(r, off + mine_m + kMidRows * 4));
#pragma unroll
        for (int e = 0; e < F; ++e) v[y][e] = bld128cf(r, off + mine + 16 * EACH * e);
      }
#pragma unroll
      for (int y = 0; y < N; ++y)
        if (b + y < it.splits) add(pm[y], pl[y], v[y]);
    }
  }
  if (row >= live_rows) return;
  const float inv = total > 0.f ? 1.f / total : 0.f;
  const int i = (tile_row + row) / p.group, hq = head * p.group + (tile_row + row) % p.group;
  uint16_t* out = p.out + (int64_t)(it.row0 + i) * p.out_ld + hq * D + 4 * own;
#pragma unroll
  for (int e = 0; e < F; ++e) *(u32x2*)(out + 4 * EACH * e) = u32x2{pack2<DT>(x[e][0] * inv, x[e][1] * inv), pack2<DT>(x[e][2] * inv, x[e][3] * inv)};
}

template <int DT, int FMT, int D, bool OPT>
__global__ __launch_bounds__(64 * kWaves, 2) void k_attend_rows(AttnParams p) {
  __shared__ __attribute__((aligned(16))) char lds[few_lds<D, kRows>()];
  __shared__ float s_m[kWaves * kRows], s_l[kWaves * kRows];
  __shared__ int s_last;
  early(p);
  attend_rows<DT, FMT, D, OPT>(p, blockIdx.x, lds, s_m, s_l, &s_last);
}
// both kinds in one launch, side by side on the GPU: those of 32 rows first
template <int DT, int FMT, int D, bool OPT>
__global__ __launch_bounds__(64 * kWaves, 2) void k_attend_mid(AttnParams p) {
  __shared__ __attribute__((aligned(16))) char lds[few_lds<D, kMidRows>()];
  __shared__ float s_m[kWaves * kMidRows], s_l[kWaves * kMidRows];
  __shared__ int s_last;
  early(p);
  if (blockIdx.x < p.mid_blocks) attend_mid<DT, FMT, D, OPT>(p, blockIdx.x, lds, s_m, s_l, &s_last);
  else attend_rows<DT, FMT, D, OPT>(p, blockIdx.x - p.mid_blocks, lds, s_m, s_l, &s_last);
}

// ---------------------------------------------------------------------------
// Tiles of 256 rows (prompts, chunks): eight waves of 32 rows. All waves bring a
// step's codes to LDS as operands (each code converted once for 256 rows), two
// steps in LDS and one in registers, and multiply on 32 x 32 x 16 MFMAs, again
// S^T = K Q^T and O^T = V^T P^T: a lane holds half the scores of one row, and its
// weights are V's operand once V's tokens stand in LDS in the order in which the
// MFMA leaves the scores (the middle quads of every sixteen exchanged).
// Bound: the MFMAs and the exponentials beside them: a prompt of 4096, 64 heads, 275 GFLOP
// in 309 us, 890 TFLOP/s; its loads and MFMAs without a softmax take 200. Tried in its
// place, same prompt: the weights of a step made beside the next step's scores 322, tiles
// of 128 rows at two workgroups a CU 367, four buffers and a barrier each two steps 319.
// ---------------------------------------------------------------------------
template <int DT, int FMT, int D, bool OPT>
__global__ __launch_bounds__(2 * tile_rows(D), 2) void k_attend_tile(AttnParams p) {
  constexpr int KP = D * 2 + 16, VP = kStep * 2 + 16, PIECES = D / 16;  // pitches in bytes; pieces of a row of K
  constexpr int KBYTES = kStep * KP, BUF = KBYTES + D * VP, ROWS = tile_rows(D), THREADS = 2 * ROWS;
  __shared__ __attribute__((aligned(16))) char lds[2 * BUF];
  __shared__ __attribute__((aligned(16))) float s_ks[2][4];
  // tokens of the four runs that stand in a page. (Words of their own: as the sign of s_ks, taken
  // off in the steps that are masked, the compiler moved that |x| to one of the two branches into
  // them, and rows of pages outside the pool were NaN.)
  __shared__ __attribute__((aligned(16))) uint32_t s_there[2][4];
  __shared__ int s_last;
  early(p);
  const int head = blockIdx.x % p.c.Hkv, idx = blockIdx.x / p.c.Hkv;
  AttnItem it = item_at(p.items_tile, idx);
  if (it.key != p.key) return;
  if (p.c.pages == 0) it.s1 = it.s0;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, h = lane >> 5;
  const int P = p.c.P, live_rows = it.rows * p.group, wave_row = it.tile * ROWS + 32 * wave;
  const int row = wave_row + c;
  const bool active = wave_row < live_rows, mine = row < live_rows;
  const int i = mine ? row / p.group : it.rows - 1, hq = head * p.group + (mine ? row % p.group : 0);
  const uint32_t sign = p.scale < 0.f ? 0x80008000u : 0u;  // (a scale below zero: of q)
  u32x4 q[D / 16];
  {
    const uint16_t* qp = p.q + (int64_t)(it.row0 + i) * p.q_ld + hq * D + 8 * h;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) q[s] = ldg16(qp + 16 * s) ^ sign;
    if (!mine)
#pragma unroll
      for (int s = 0; s < D / 16; ++s) q[s] = u32x4{0, 0, 0, 0};
  }
  const int pos = it.pos0 + i;
  // positions of the wave's first and last row
  const int pos_lo = it.pos0 + min(wave_row / p.group, it.rows - 1), pos_hi = it.pos0 + min((wave_row + 31) / p.group, it.rows - 1);
  const ScoreOptions opt{fabsf(p.scale), p.softcap, p.inv_cap, OPT && p.slopes ? p.slopes[hq] * kLog2e : 0.f};
  const int32_t* table = p.table + it.r * p.ld;
  const uint32_t page_bytes = P * D, pool_bytes = p.c.Hkv * page_bytes;

  // staging: a thread's pieces are N of K, TOKENS apart, and N of V, FEATURES apart, of one run
  constexpr int N = kStep * PIECES / THREADS, TOKENS = THREADS / PIECES, FEATURES = THREADS / 4;
  static_assert(N >= 1 && TOKENS % 16 == 0 && N * FEATURES == D, "whole pieces");
  const int k_token = tid / PIECES, k_piece = tid % PIECES, v_feature = tid >> 2, v_run = tid & 3;
  const uint8_t* k_head = p.c.k + (int64_t)head * page_bytes + 16 * k_piece;
  const uint8_t* v_head = p.c.v + (int64_t)head * page_bytes + v_feature * P;
  // table entries of a step's runs; whether they are pages is looked at where they are
  // used (a comparison here would wait for the load)
  auto entry_at = [&](int s, int run) {
    const int j = s * kStep + 16 * run;
    int page = -1;
    if (s < it.s1 && j < it.end) page = table[j >> p.log2_page];
    return page;
  };
  auto page_of = [&](int entry) { return (uint32_t)entry < (uint32_t)p.c.pages ? entry : -1; };
  u32x4 kr[N], vr[N];
  float2 sc;  // scales of this thread's run of V
  int entry_k[N], entry_v, held_v = 0;
  auto entries = [&](int s) {
#pragma unroll
    for (int x = 0; x < N; ++x) entry_k[x] = entry_at(s, (k_token + TOKENS * x) >> 4);
    entry_v = entry_at(s, v_run);
  };
  auto fetch = [&](int s) {  // entries of s are there; those of s + 1 follow
#pragma unroll
    for (int x = 0; x < N; ++x)
      kr[x] = ldg16(k_head + (uint64_t)(uint32_t)max(page_of(entry_k[x]), 0) * pool_bytes + ((s * kStep + k_token + TOKENS * x) & (P - 1)) * D);
    const uint32_t page_v = max(held_v = page_of(entry_v), 0);
    const uint8_t* v = v_head + (uint64_t)page_v * pool_bytes + ((s * kStep + 16 * v_run) & (P - 1));
#pragma unroll
    for (int x = 0; x < N; ++x) vr[x] = ldg16(v + FEATURES * x * P);
    const uint64_t ph = (uint64_t)page_v * p.c.Hkv + head;
    sc = make_float2(p.c.k_scale[ph], p.c.v_scale[ph]);
    entries(s + 1);
  };
  auto stage = [&](int s) {
    char* buf = lds + (s & 1) * BUF;
#pragma unroll
    for (int x = 0; x < N; ++x) {
      u32x4* k = (u32x4*)(buf + (k_token + TOKENS * x) * KP + 32 * k_piece);
      k[0] = operand8<DT, FMT>(kr[x][0], kr[x][1], 1.f);
      k[1] = operand8<DT, FMT>(kr[x][2], kr[x][3], 1.f);
    }
    float f = sc.y;
    const int j0 = s * kStep + 16 * v_run;
    if (held_v < 0 || j0 + 16 > it.end || j0 < it.first) {
      const uint32_t live = held_v >= 0 ? live_tokens(j0, it) & 0xFFFFu : 0u;
      const u32x4 bytes = byte_mask(live);
#pragma unroll
      for (int x = 0; x < N; ++x) vr[x] &= bytes;
      if (!live) f = 1.f;
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
      u32x4* v = (u32x4*)(buf + KBYTES + (v_feature + FEATURES * x) * VP + 32 * v_run);
      if (FMT == KV_INT8 && (DT != DT_F16 || f < 6.103515625e-5f)) {  // (fp16: a scale below its normal range)
        v[0] = i8x8_to_act<DT>(vr[x][0], vr[x][2], f);
        v[1] = i8x8_to_act<DT>(vr[x][1], vr[x][3], f);
      } else {
        v[0] = v_operand8<DT, FMT>(vr[x][0], vr[x][2], f);
        v[1] = v_operand8<DT, FMT>(vr[x][1], vr[x][3], f);
      }
    }
    // (runs 0..3) what a dot product is of a score
    if (tid < 4) s_ks[s & 1][tid] = OPT ? sc.x : dot_factor(sc.x, opt), s_there[s & 1][tid] = held_v < 0 ? 0u : 0xFFFFu;
  };

  f32x16 o[D / 32] = {};
  float m = kLowest, l = 0.f;
  if (it.s0 < it.s1) {
    entries(it.s0);
    fetch(it.s0);
    stage(it.s0);
    if (it.s0 + 1 < it.s1) fetch(it.s0 + 1);
    __syncthreads();
  }
  for (int s = it.s0; s < it.s1; ++s) {
    // (the other buffer's readers have passed the last barrier)
    if (s + 1 < it.s1) {
      stage(s + 1);
      if (s + 2 < it.s1) fetch(s + 2);
    }
    const int j0 = s * kStep;
    const bool sees_any = active && ((j0 <= pos_hi && j0 + kStep > pos_lo - p.window + 1) || j0 < it.prefix);
    if (sees_any) {
      const char* buf = lds + (s & 1) * BUF;
      f32x16 st[2] = {};
#pragma unroll
      for (int x = 0; x < D / 16; ++x)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          st[t] = mfma32<DT>(*(const u32x4*)(buf + (32 * t + c) * KP + 32 * x + 16 * h), q[x], st[t]);
      const f32x4 ks = *(const f32x4*)s_ks[s & 1];
      const u32x4 there = *(const u32x4*)s_there[s & 1];
      const bool pages_there = __builtin_amdgcn_readfirstlane(there[0] & there[1] & there[2] & there[3]) != 0;
      const bool whole = j0 + kStep <= min(it.end, pos_lo + 1) && pos_hi - j0 < p.window && pages_there;
      f32x4 f = ks;  // what st is of a score
      if constexpr (OPT) {
        f = f32x4{1.f, 1.f, 1.f, 1.f};
#pragma unroll
        for (int e = 0; e < 32; ++e)
          st[e >> 4][e & 15] = score2(st[e >> 4][e & 15], ks[e >> 3], opt, pos, j0 + 8 * (e >> 2) + 4 * h + (e & 3));
      }
      if (!whole) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          uint32_t sees = seen_tokens(j0 + 32 * t, it, pos, p.window);
          sees &= there[2 * t] | there[2 * t + 1] << 16;
          sees >>= 4 * h;
#pragma unroll
          for (int e = 0; e < 16; ++e) st[t][e] = where_seen(st[t][e], sees, 8 * (e >> 2) + (e & 3));
        }
      }
      u32x4 pw[4];  // sixteen tokens each
      float sum;
      for (int pass = 0;; ++pass) {
        sum = 0.f;
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int x = 8 * (y & 1) + 2 * e;
            pw[y][e] = pack2<DT>(__builtin_amdgcn_exp2f(__builtin_fmaf(st[y >> 1][x], f[y], -m)),
                                 __builtin_amdgcn_exp2f(__builtin_fmaf(st[y >> 1][x + 1], f[y], -m)));
            sum = add2<DT>(pw[y][e], sum);
          }
        if (pass || !__any(!(sum <= kMostSum<DT>))) break;
        float top = kLowest;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = st[r >> 1][8 * (r & 1)];
#pragma unroll
          for (int e = 1; e < 8; ++e) x = fmaxf(x, st[r >> 1][8 * (r & 1) + e]);
          top = fmaxf(top, x * f[r]);
        }
        const float now = fmaxf(m, max_halves(top) - kTileLift<DT>), fade = __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= fade;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[d] *= fade;
      }
      l += sum;
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
          o[d] = mfma32<DT>(*(const u32x4*)(buf + KBYTES + (32 * d + c) * VP + 32 * y + 16 * h), pw[y], o[d]);
    }
    __syncthreads();
  }
  l += __shfl_xor(l, 32);
  if (it.splits > 1) {
    const uint32_t size = ROWS * (D + 2) * 4, slot = (uint32_t)it.part * p.c.Hkv + head;
    const rsrc_t r = make_rsrc((const char*)p.parts_tile + (size_t)slot * size, (uint32_t)((it.splits - 1) * p.c.Hkv + 1) * size);
    const uint32_t at = (uint32_t)it.split * p.c.Hkv * size, own = ((32 * wave + c) * D + 4 * h) * 4;
    const uint32_t own_m = (ROWS * D + 32 * wave + c) * 4;
    if (active) {
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          bst128c(r, at + own + (32 * d + 8 * x) * 4, f32x4{o[d][4 * x], o[d][4 * x + 1], o[d][4 * x + 2], o[d][4 * x + 3]});
      float* ml = p.parts_tile + ((size_t)slot * size + at + own_m) / 4;
      if (h == 0) st_agent(ml, m), st_agent(ml + ROWS, l);
    }
    complete_and_sync();
    if (tid == 0) s_last = arrive_last(p.counters_tile + slot, it.splits);
    __syncthreads();
    if (!s_last) return;
    if (active) {
      m = kLowest, l = 0.f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d] = f32x16{};
      for (int b = 0; b < it.splits; ++b) {
        const uint32_t off = b * p.c.Hkv * size;
        const float pm = __uint_as_float(bld32c(r, off + own_m)), pl = __uint_as_float(bld32c(r, off + own_m + ROWS * 4));
        const float now = fmaxf(m, pm), f0 = __builtin_amdgcn_exp2f(m - now), f1 = __builtin_amdgcn_exp2f(pm - now);
        m = now;
        l = l * f0 + pl * f1;
        f32x4 v[D / 8];
#pragma unroll
        for (int x = 0; x < D / 8; ++x) v[x] = bld128cf(r, off + own + 8 * x * 4);
#pragma unroll
        for (int x = 0; x < D / 8; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[x >> 2][4 * (x & 3) + e] = o[x >> 2][4 * (x & 3) + e] * f0 + v[x][e] * f1;
      }
    }
  }
  if (!mine) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  uint16_t* out = p.out + (int64_t)(it.row0 + i) * p.out_ld + hq * D + 4 * h;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *(u32x2*)(out + 32 * d + 8 * x) = u32x2{pack2<DT>(o[d][4 * x] * inv, o[d][4 * x + 1] * inv),
                                              pack2<DT>(o[d][4 * x + 2] * inv, o[d][4 * x + 3] * inv)};
}

template <int FMT, int D, bool OPT>
static hipError_t attend_launch(const AttnParams& p, const AttnShape& z, hipStream_t st) {
  const uint32_t rows = (uint32_t)z.max_rows * p.c.Hkv, tiles = (uint32_t)z.max_tile * p.c.Hkv;
  if (tiles && z.tile_rows == kMidRows) {
    hipLaunchKernelGGL((k_attend_mid<DTC, FMT, D, OPT>), dim3(tiles + rows), dim3(64 * kWaves), 0, st, p);
    return hipGetLastError();
  }
  if (tiles) {
    hipLaunchKernelGGL((k_attend_tile<DTC, FMT, D, OPT>), dim3(tiles), dim3(2 * tile_rows(D)), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (rows) hipLaunchKernelGGL((k_attend_rows<DTC, FMT, D, OPT>), dim3(rows), dim3(64 * kWaves), 0, st, p);
  return hipGetLastError();
}
template <int FMT, int D>
static hipError_t attend_options(const AttnParams& p, const AttnShape& z, hipStream_t st) {
  return p.slopes || p.softcap > 0.f ? attend_launch<FMT, D, true>(p, z, st) : attend_launch<FMT, D, false>(p, z, st);
}
hipError_t SPEAR_D(launch_attend)(const AttnParams& p, const AttnShape& z, int format, hipStream_t st) {
  if (p.c.D == 64) return format == KV_INT8 ? attend_options<KV_INT8, 64>(p, z, st) : attend_options<KV_E4M3, 64>(p, z, st);
  return format == KV_INT8 ? attend_options<KV_INT8, 128>(p, z, st) : attend_options<KV_E4M3, 128>(p, z, st);
}

}  // namespace spear
