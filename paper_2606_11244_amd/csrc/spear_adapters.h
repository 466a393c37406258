// What other kernels share with the adapters' own (spear_adapters.hip): tokens and
// slots, the decode coordinates, which a GEMV launch may carry along as further
// workgroups, and the two parts in which the coordinates enter an MFMA.
#pragma once

#include "spear_device.h"

namespace spear {

// ---------------------------------------------------------------------------
// tokens and slots
// ---------------------------------------------------------------------------

// the slot of token m, or -1 (none) for any id outside [0, L)
__device__ __forceinline__ int slot_of(const AdapterParams& p, int m) {
  const int a = p.ids[m];
  return a >= 0 && a < p.L ? a : -1;
}
__device__ __forceinline__ int rank_of(const AdapterParams& p, int a) {
  if (a < 0) return 0;
  return p.ranks ? min(max(p.ranks[a], 0), p.R) : p.R;
}

// The tokens of one slot that a leader's workgroups own.
struct TokenGroup {
  int a, r;    // slot (-1: none) and its rank
  int cnt;     // tokens, 0: this token leads none
  int tok;     // this lane's: token lane % 16 of the group (past cnt: the leader)
};
// Among the 64 tokens around m; every wave of the workgroup calls it. stok: 16
// ints of LDS.
__device__ __forceinline__ TokenGroup token_group(const AdapterParams& p, int m, int* stok) {
  const int lane = threadIdx.x & 63, ml = m & 63, m0 = m - ml;
  const int id = m0 + lane < p.M ? slot_of(p, m0 + lane) : -2;
  TokenGroup g;
  g.a = __builtin_amdgcn_readlane(id, ml);
  const uint64_t same = __ballot(id == g.a);
  const int before = __popcll(same & ((1ull << ml) - 1));
  g.cnt = 0;
  g.r = 0;
  g.tok = m;
  if (before & 15) return g;  // uniform
  const uint64_t mine = same & ~((1ull << ml) - 1);
  g.cnt = min(16, (int)__popcll(mine));
  const int pos = __popcll(mine & ((1ull << lane) - 1));
  if (((mine >> lane) & 1) && pos < 16) stok[pos] = m0 + lane;  // every wave writes the same
  __syncthreads();
  g.tok = stok[min(lane & 15, g.cnt - 1)];
  g.r = rank_of(p, g.a);
  return g;
}

// ---------------------------------------------------------------------------
// u, up to 16 tokens of one slot
// ---------------------------------------------------------------------------

// acc[t] += rows j0 + 16 t .. +16 of A_a times the group's tokens, over the
// wave's share (wave, wave + NW, ..) of the nit iterations of 128 K from it0,
// rotated by rot. K order within an iteration: MFMA jj,
// lane group lg takes K [8 lg + 32 jj, +8) for both operands (64 contiguous
// bytes per row and load). Rows from r on are not read.
//
// In the MFMA's layout (lane: column lane % 16) the tokens cost 16 loads for
// 512 K however few they are, as many as 16 rows of the slot, and the loads'
// rate is the bound. So up to four tokens (the usual case at decode) come in
// whole, one load each, and through the wave's own part of the LDS, xs
// [4][kXRow].
//
// The wave's iterations lie NW apart, from one that differs between the slots:
// the slot's rows are a multiple of 4 KB apart on the usual layers, so that a
// load's 16 rows lie in one L2 channel, and waves that walked K in step would
// queue at a few channels at a time. (Between the slots, not the leaders: a
// token's sums are in the order that its own slot gives, whichever tokens share
// the slot and whichever row is the first of them.)
//
// At these sizes a workgroup's time is its instructions as much as its loads (a
// SIMD issues one every four cycles): every load takes its place in K from a
// scalar and a constant, and nothing is masked lane by lane.
constexpr int kXRow = 512 + 8;  // halves
template <int DT, int RT, bool FEW>
__device__ __forceinline__ void project_part(rsrc_t rx, const TokenGroup& g, const int* stok, uint16_t* xs, rsrc_t ra,
                                             int K, int j0, int r, int it0, int nit, int rot, int wave, int NW,
                                             f32x4 (&acc)[RT]) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  uint32_t aoff[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int j = j0 + 16 * t + lr;
    aoff[t] = j < r ? (uint32_t)j * K * 2 + 16 * lg : kOOB;
  }
  const uint16_t* xr = xs + min(lr, g.cnt - 1) * kXRow + 8 * lg;
  const uint32_t xo = (uint32_t)g.tok * K * 2 + 16 * lg;
  uint32_t xw[4];  // FEW: this lane's 16 bytes of each token's iterations
#pragma unroll
  for (int t = 0; t < 4; ++t) xw[t] = FEW ? (uint32_t)stok[min(t, g.cnt - 1)] * K * 2 + 16 * lr : 0u;
  int i = wave;
  auto at = [&](int j) {  // iteration j of the walk, its place in a row (bytes)
    const int v = j + rot;
    return (uint32_t)(it0 + (v >= nit ? v - nit : v)) * (kIterK * 2);
  };
  // I iterations, all of their loads in flight together
  auto pass = [&](auto ic) {
    constexpr int I = decltype(ic)::value;
    u32x4 av[I][RT][4], xv[FEW ? 1 : I][4];
    uint32_t kb[I];  // uniform
#pragma unroll
    for (int h = 0; h < I; ++h) kb[h] = at(i + h * NW);
    if constexpr (FEW) {
      // lane group h brings iteration h
      const uint32_t kl = at(i + min(lg, I - 1) * NW);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t == 0 || t < g.cnt) xv[0][t] = bld128(rx, xw[t] + kl);  // (uniform)
    } else {
#pragma unroll
      for (int h = 0; h < I; ++h)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) xv[h][jj] = bld128s(rx, xo + 64 * jj, kb[h]);
    }
#pragma unroll
    for (int h = 0; h < I; ++h)
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) av[h][t][jj] = bld128s(ra, aoff[t] + 64 * jj, kb[h]);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (FEW) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t == 0 || t < g.cnt) *(u32x4*)(xs + t * kXRow + 8 * lane) = xv[0][t];
      __builtin_amdgcn_wave_barrier();  // the wave's own LDS, in program order
    }
#pragma unroll
    for (int h = 0; h < I; ++h)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        u32x4 xf;
        if constexpr (FEW) xf = *(const u32x4*)(xr + 128 * h + 32 * jj);
        else xf = xv[h][jj];
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = mfma16<DT>(av[h][t][jj], xf, acc[t]);
      }
    if constexpr (FEW) __builtin_amdgcn_wave_barrier();
    i += I * NW;
  };
  constexpr int I = RT == 1 && FEW ? 4 : 2;
  while (i + (I - 1) * NW < nit) pass(std::integral_constant<int, I>());
  if (I == 4 && i + NW < nit) pass(std::integral_constant<int, 2>());
  while (i < nit) pass(std::integral_constant<int, 1>());
}
// (the second half of acc stays as it is where the ranks fit one row tile)
template <int DT>
__device__ __forceinline__ void project(rsrc_t rx, const TokenGroup& g, const int* stok, uint16_t* xs, rsrc_t ra, int K,
                                        int j0, int r, int it0, int nit, int rot, int wave, int NW, f32x4 (&acc)[2]) {
  if (r - j0 > 16) {
    if (g.cnt <= 4) project_part<DT, 2, true>(rx, g, stok, xs, ra, K, j0, r, it0, nit, rot, wave, NW, acc);
    else project_part<DT, 2, false>(rx, g, stok, xs, ra, K, j0, r, it0, nit, rot, wave, NW, acc);
  } else {
    f32x4 a1[1] = {acc[0]};
    if (g.cnt <= 4) project_part<DT, 1, true>(rx, g, stok, xs, ra, K, j0, r, it0, nit, rot, wave, NW, a1);
    else project_part<DT, 1, false>(rx, g, stok, xs, ra, K, j0, r, it0, nit, rot, wave, NW, a1);
    acc[0] = a1[0];
  }
}

// ---------------------------------------------------------------------------
// few tokens: u in slices over K
// ---------------------------------------------------------------------------

// Workgroup b of a member: the sums of one token's slot over a K-slice for one
// rank group, by any number NW of waves; smem: shrink_slot_lds(NW) bytes.
inline size_t shrink_slot_lds(int NW) { return 64 + (size_t)NW * (2048 + 8 * kXRow); }
template <int DT>
__device__ __forceinline__ void shrink_slot(const AdapterParams& p, int b, char* smem) {
  const int NW = blockDim.x >> 6;
  int* stok = (int*)smem;                            // [16]
  float* red = (float*)(smem + 64);                  // [NW][2][256]
  uint16_t* xs = (uint16_t*)(smem + 64 + NW * 2048); // [NW][4 kXRow]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = p.P * p.RG, m = b / per, rem = b - m * per, rg = rem / p.P, ks = rem - rg * p.P;
  const TokenGroup g = token_group(p, m, stok);
  if (g.cnt == 0 || 32 * rg >= g.r) return;
  const rsrc_t rx = make_rsrc(p.x, (uint32_t)p.M * p.K * 2);
  const rsrc_t ra = make_rsrc(p.A + (size_t)g.a * p.a_stride, (uint32_t)p.R * p.K * 2);
  f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  const int it0 = ks * p.ips, nit = min(p.K / kIterK - it0, p.ips);
  project<DT>(rx, g, stok, xs + wave * 4 * kXRow, ra, p.K, 32 * rg, g.r, it0, nit, g.a % nit, wave, NW, acc);
#pragma unroll
  for (int t = 0; t < 2; ++t) *(f32x4*)(red + (2 * wave + t) * 256 + 4 * lane) = acc[t];
  __syncthreads();
  // lane l of a tile holds token l % 16, ranks 4 (l / 16) .. +4
  for (int i = wave; i < 2; i += NW) {
    const int tok = lane & 15, j = 32 * rg + 16 * i + 4 * (lane >> 4);
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < NW; ++w) s += *(const f32x4*)(red + (2 * w + i) * 256 + 4 * lane);
    if (tok < g.cnt) *(f32x4*)(p.upart + ((size_t)ks * p.M + stok[tok]) * (32 * p.RG) + j) = s;
  }
}

// ---------------------------------------------------------------------------
// the parts of u
// ---------------------------------------------------------------------------

// The two activation-dtype parts of a coordinate. fp16 has neither the range
// nor, for small values, the precision: where the largest of the 32 coordinates
// of a token and rank group is not between 1/2 and 2^15, they are first scaled
// by a power of two that brings it near 2^14, undone on the fp32 result of
// their MFMA.
template <int DT>
__device__ __forceinline__ void split_parts(float v, uint16_t* hi, uint16_t* lo) {
  *hi = f2act<DT>(v);
  const float h = act2f<DT>(*hi);
  *lo = __builtin_fabsf(h) < __builtin_inff() ? f2act<DT>(v - h) : (uint16_t)0;
}
__device__ __forceinline__ int scale_exp(float maxabs) {  // k: the values times 2^k
  const int e = (int)((__float_as_uint(maxabs) >> 23) & 255) - 127;
  return e == 128 || (e >= -1 && e <= 14) ? 0 : min(max(14 - e, -113), 100);
}
__device__ __forceinline__ float exp2i(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

}  // namespace spear
