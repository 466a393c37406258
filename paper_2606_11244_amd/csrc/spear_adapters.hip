// gfx950 (MI355X) kernels of the low-rank adapters of many requests: the term
//   d[m] = res[m] + s_a B_a (A_a x[m]),   a = ids[m] (d[m] = res[m] without one)
// that the 4-bit product's final store adds in place of a residual.
//
// Two steps, the coordinates u[m] = s_a A_a x[m] (bound by reading x and the
// slots' A) and the term B_a u[m] (bound by reading B and writing d). Both are
// MFMAs of up to 16 tokens by 16 rows of a slot (rows as the A operand, tokens
// as the columns of the B operand, so that a lane's results belong to one
// token), over the slots that the tokens at hand name; a result is kept only
// for the tokens of the slot it was formed with, by selection and not by a
// product with zero, so that no token meets another's values. u is held in
// fp32 and enters the second MFMA as two activation-dtype parts.
//
// Decode (up to 64 tokens): the tokens of one slot, up to 16 of them, belong
// to the workgroups of the first of them ("leader"); the other tokens'
// workgroups end at once. Nothing needs sorting, and the ids are read on the
// device. Beyond, a workgroup owns 64 consecutive tokens and walks the slots
// they name.
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
__device__ __forceinline__ int rank_of(const AdapterParams& p, int a) {  // a uniform
  if (a < 0) return 0;
  return p.ranks ? min(max(p.ranks[a], 0), p.R) : p.R;
}

// The tokens of one slot that a leader's workgroups own.
struct TokenGroup {
  int a, r;    // slot (-1: none) and its rank
  int cnt;     // tokens, 0: this token leads none
  int tok;     // this lane's: token lane % 16 of the group (past cnt: the leader)
};
// M <= 64; every wave of the workgroup calls it. stok: 16 ints of LDS.
__device__ __forceinline__ TokenGroup token_group(const AdapterParams& p, int m, int* stok) {
  const int lane = threadIdx.x & 63;
  const int id = lane < p.M ? slot_of(p, lane) : -2;
  TokenGroup g;
  g.a = __builtin_amdgcn_readlane(id, m);
  const uint64_t same = __ballot(id == g.a);
  const int before = __popcll(same & ((1ull << m) - 1));
  g.cnt = 0;
  g.r = 0;
  g.tok = m;
  if (before & 15) return g;  // uniform
  const uint64_t mine = same & ~((1ull << m) - 1);
  g.cnt = min(16, (int)__popcll(mine));
  const int pos = __popcll(mine & ((1ull << lane) - 1));
  if (((mine >> lane) & 1) && pos < 16) stok[pos] = lane;  // every wave writes the same
  __syncthreads();
  g.tok = stok[min(lane & 15, g.cnt - 1)];
  g.r = rank_of(p, g.a);
  return g;
}

// ---------------------------------------------------------------------------
// u, up to 16 tokens of one slot
// ---------------------------------------------------------------------------

// acc[t] += rows j0 + 16 t .. +16 of A_a times the tokens at xoff (per lane: byte
// offset of its token's row), over the wave's share of iterations [it_beg,
// it_end) of 128 K. K order within an iteration: MFMA jj, lane group lg takes
// K [8 lg + 32 jj, +8) for both operands (64 contiguous bytes per row and
// load). Rows from r on are not read.
template <int DT, int RT>
__device__ __forceinline__ void project(rsrc_t rx, uint32_t xoff, rsrc_t ra, int K, int j0, int r, int it_beg,
                                        int it_end, int wave, int NW, f32x4 (&acc)[RT]) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  constexpr int IPP = 2;  // iterations whose loads are in flight together
  uint32_t aoff[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int j = j0 + 16 * t + lr;
    aoff[t] = j < r ? (uint32_t)j * K * 2 + 16 * lg : kOOB;
  }
  const uint32_t xo = xoff + 16 * lg;
  for (int it0 = it_beg + wave * IPP; it0 < it_end; it0 += NW * IPP) {
    u32x4 xv[IPP][4], av[IPP][RT][4];
#pragma unroll
    for (int h = 0; h < IPP; ++h) {
      const bool ok = it0 + h < it_end;  // uniform
      const uint32_t kb = (uint32_t)(it0 + h) * (kIterK * 2);
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) xv[h][jj] = bld128(rx, ok ? xo + kb + 64 * jj : kOOB);
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
          av[h][t][jj] = bld128(ra, ok && aoff[t] != kOOB ? aoff[t] + kb + 64 * jj : kOOB);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int h = 0; h < IPP; ++h)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = mfma16<DT>(av[h][t][jj], xv[h][jj], acc[t]);
  }
}

// The two activation-dtype parts of a coordinate. fp16 has neither the range
// nor, for small values, the precision: there the 32 coordinates of a token and
// rank group are first scaled by a power of two that brings the largest near
// 2^14, undone on the fp32 result of their MFMA.
template <int DT>
__device__ __forceinline__ void split_parts(float v, uint16_t* hi, uint16_t* lo) {
  *hi = f2act<DT>(v);
  const float h = act2f<DT>(*hi);
  *lo = __builtin_fabsf(h) < __builtin_inff() ? f2act<DT>(v - h) : (uint16_t)0;
}
__device__ __forceinline__ int scale_exp(float maxabs) {  // k: the values times 2^k
  const int e = (int)((__float_as_uint(maxabs) >> 23) & 255) - 127;
  return e == 128 ? 0 : min(max(14 - e, -113), 100);
}
__device__ __forceinline__ float exp2i(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// u [cnt][32] of a rank group in LDS (row stride us) to parts at hi, lo (row
// stride hs) and the scale of each token to undo at sc (stride ss); 32 lanes
// per token. tok(t): where token t's row goes (negative: nowhere).
template <int DT, class Row>
__device__ __forceinline__ void store_parts(int cnt, const float* u, int us, uint16_t* hi, uint16_t* lo, int hs,
                                            float* sc, int ss, Row row) {
  for (int i = threadIdx.x; i < cnt * 32; i += blockDim.x) {  // (whole waves stay together: cnt * 32 in steps of 64 or a half wave)
    const int t = i >> 5, j = i & 31;
    float v = u[t * us + j];
    const int m = row(t);
    if constexpr (DT == DT_F16) {
      float mx = __builtin_fabsf(v);
#pragma unroll
      for (int h = 16; h > 0; h >>= 1) mx = fmaxf(mx, __shfl_xor(mx, h));
      const int k = scale_exp(mx);
      v *= exp2i(k);
      if (j == 0 && m >= 0) sc[(size_t)m * ss] = exp2i(-k);
    }
    uint16_t h, l;
    split_parts<DT>(v, &h, &l);
    if (m >= 0) {
      hi[(size_t)m * hs + j] = h;
      lo[(size_t)m * hs + j] = l;
    }
  }
}

// ---------------------------------------------------------------------------
// the term
// ---------------------------------------------------------------------------

// Row pair: 32 rows of B_a as two MFMA row tiles whose row q of tile t is row 8
// (q / 4) + 4 t + q % 4, so that a lane's eight results are consecutive rows.
// Its fragments of rank group kk; ranks from r on read as zero.
template <int DT>
__device__ __forceinline__ void load_pair(const AdapterParams& p, rsrc_t rb, int n0, int kk, int r, bool vec,
                                          u32x4 (&bf)[2]) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int j0 = 32 * kk + 8 * lg;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int n = n0 + 8 * (lr >> 2) + 4 * t + (lr & 3);
    const uint32_t off = ((uint32_t)n * p.R + j0) * 2;
    if (vec) {
      bf[t] = bld128(rb, n < p.N && j0 < r ? off : kOOB);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = j0 + 2 * q;
        bf[t][q] = bld16(rb, n < p.N && j < r ? off + 4 * q : kOOB) |
                   (bld16(rb, n < p.N && j + 1 < r ? off + 4 * q + 2 : kOOB) << 16);
      }
    }
  }
}
// (the ranks past r of a whole chunk of eight, read with it: to zero)
__device__ __forceinline__ void mask_pair(int kk, int r, u32x4 (&bf)[2]) {
  const int j0 = 32 * kk + 8 * ((threadIdx.x & 63) >> 4);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t keep = (j0 + 2 * q < r ? 0xFFFFu : 0u) | (j0 + 2 * q + 1 < r ? 0xFFFF0000u : 0u);
    bf[0][q] &= keep;
    bf[1][q] &= keep;
  }
}

// A lane's eight rows n .. n + 8 of token m: v plus the residual, rounded once.
template <int DT>
__device__ __forceinline__ void store_term(const AdapterParams& p, int m, int n, const f32x4 (&v)[2]) {
  const size_t o = (size_t)m * p.N + n;
  if ((p.N & 7) == 0) {
    if (n >= p.N) return;
    u32x4 rv = u32x4{0, 0, 0, 0}, w;
    if (p.res) rv = ldg16(p.res + o);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float a = v[q >> 1][2 * (q & 1)] + act2f<DT>(rv[q] & 0xFFFFu);
      const float b = v[q >> 1][2 * (q & 1) + 1] + act2f<DT>(rv[q] >> 16);
      w[q] = (uint32_t)f2act<DT>(a) | ((uint32_t)f2act<DT>(b) << 16);
    }
    *(u32x4*)(p.d + o) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (n + e < p.N) p.d[o + e] = f2act<DT>(v[e >> 2][e & 3] + (p.res ? act2f<DT>(p.res[o + e]) : 0.f));
  }
}

// The rows [n0, n1) of the term for a group of up to 16 tokens of one slot, by
// the workgroup; part(kk, hi, lo, sc): this lane's fragments of u (token lane %
// 16, ranks 32 kk + 8 (lane / 16) .. +8) and its scale.
template <int DT, class Part>
__device__ __forceinline__ void expand_group(const AdapterParams& p, const TokenGroup& g, int n0, int n1, Part part) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), NW = blockDim.x >> 6;
  const rsrc_t rb = make_rsrc(p.B + (size_t)max(g.a, 0) * p.b_stride, (uint32_t)p.N * p.R * 2);
  const int nkk = (g.r + 31) >> 5;
  const bool vec = (p.R & 7) == 0 && (p.b_stride & 7) == 0;
  const bool cut = vec && (g.r & 7) != 0;
  for (int n = n0 + 32 * wave; n < n1; n += 32 * NW) {
    f32x4 v[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
    for (int kk = 0; kk < nkk; ++kk) {
      u32x4 bf[2], hi, lo;
      float sc = 1.f;
      load_pair<DT>(p, rb, n, kk, g.r, vec, bf);
      part(kk, hi, lo, sc);
      if (cut) mask_pair(kk, g.r, bf);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if constexpr (DT == DT_F16) {
          f32x4 q = f32x4{0.f, 0.f, 0.f, 0.f};
          q = mfma16<DT>(bf[t], hi, q);
          q = mfma16<DT>(bf[t], lo, q);
          v[t] += sc * q;
        } else {
          v[t] = mfma16<DT>(bf[t], hi, v[t]);
          v[t] = mfma16<DT>(bf[t], lo, v[t]);
        }
      }
    }
    if (lr < g.cnt) store_term<DT>(p, g.tok, n + 8 * lg, v);
  }
}

// ---------------------------------------------------------------------------
// decode: u in slices over K, then the term
// ---------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ void shrink_group(const AdapterParams& p, int b) {
  __shared__ float red[4][2][256];
  __shared__ float u[16][33];
  __shared__ int stok[16], s_last;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = p.P * p.RG, m = b / per, rem = b - m * per, rg = rem / p.P, ks = rem - rg * p.P;
  const TokenGroup g = token_group(p, m, stok);
  if (g.cnt == 0 || 32 * rg >= g.r) return;
  const rsrc_t rx = make_rsrc(p.x, (uint32_t)p.M * p.K * 2);
  const rsrc_t ra = make_rsrc(p.A + (size_t)g.a * p.a_stride, (uint32_t)p.R * p.K * 2);
  f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  const int it0 = ks * p.ips, it1 = min(p.K / kIterK, it0 + p.ips);
  if (g.r - 32 * rg > 16) {
    project<DT, 2>(rx, (uint32_t)g.tok * p.K * 2, ra, p.K, 32 * rg, g.r, it0, it1, wave, 4, acc);
  } else {
    f32x4 a1[1] = {acc[0]};
    project<DT, 1>(rx, (uint32_t)g.tok * p.K * 2, ra, p.K, 32 * rg, g.r, it0, it1, wave, 4, a1);
    acc[0] = a1[0];
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) *(f32x4*)(red[wave][t] + 4 * lane) = acc[t];
  __syncthreads();
  // lane l of a tile holds token l % 16, ranks 4 (l / 16) .. +4
  const float sc = p.scale ? p.scale[g.a] : 1.f;
  float* part = p.upart + (size_t)ks * p.M * (32 * p.RG);
  for (int i = threadIdx.x; i < 512; i += 256) {
    const int t = i >> 8, l = (i & 255) >> 2, e = i & 3, tok = l & 15, j = 16 * t + 4 * (l >> 4) + e;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) s += red[w][t][4 * l + e];
    s = 32 * rg + j < g.r ? s : 0.f;
    if (p.P == 1) u[tok][j] = sc * s;
    else if (tok < g.cnt) st_agent(part + (size_t)stok[tok] * (32 * p.RG) + 32 * rg + j, s);
  }
  if (p.P > 1) {
    complete_and_sync();
    if (threadIdx.x == 0) s_last = arrive_last(p.ctr + m * p.RG + rg, (uint32_t)p.P) ? 1 : 0;
    __syncthreads();
    if (!s_last) return;
    const int W = 32 * p.RG;
    const rsrc_t rp = make_rsrc(p.upart, (uint32_t)p.P * p.M * W * 4);
    sum_slices(rp, p.P, g.cnt * 32,
               [&](int q, int i) { return (uint32_t)((q * p.M + stok[i >> 5]) * W + 32 * rg + (i & 31)) * 4u; },
               [&](int i, float v) { u[i >> 5][i & 31] = sc * v; });
  }
  __syncthreads();
  const int W = 32 * p.RG;
  store_parts<DT>(g.cnt, &u[0][0], 33, p.uh + 32 * rg, p.ul + 32 * rg, W, p.us + rg, p.RG,
                  [&](int t) { return stok[t]; });
}

// ---------------------------------------------------------------------------
// beyond: 64 consecutive tokens
// ---------------------------------------------------------------------------

// The slots that the 64 tokens from m0 name, one after another: next() gives the
// tokens of the next one this part owns (the i-th with i % PA == pa).
struct TileSlots {
  int id;         // this lane's token's slot (-1: none, -2: no token)
  uint64_t left;  // tokens of slots not yet given
  int i, pa, PA;
  __device__ __forceinline__ TileSlots(const AdapterParams& p, int m0, int pa_, int PA_) : i(0), pa(pa_), PA(PA_) {
    const int m = m0 + (threadIdx.x & 63);
    id = m < p.M ? slot_of(p, m) : -2;
    left = __ballot(id >= 0);
  }
  __device__ __forceinline__ bool next(int* a, uint64_t* toks) {
    while (left) {
      *a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
      *toks = __ballot(id == *a);
      left &= ~*toks;
      if (i++ % PA == pa) return true;
    }
    return false;
  }
};

template <int DT>
__device__ __forceinline__ void shrink_tile(const AdapterParams& p, int b) {
  __shared__ float red[4][2][4][256];
  __shared__ float u[64][33];
  __shared__ int s_last;
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = p.P * p.RG * p.PA, tb = b / per;
  int rem = b - tb * per;
  const int rg = rem / (p.P * p.PA);
  rem -= rg * p.P * p.PA;
  const int ks = rem / p.PA, pa = rem - ks * p.PA;
  const int m0 = 64 * tb, cnt = min(64, p.M - m0), W = 32 * p.RG;
  const rsrc_t rx = make_rsrc(p.x, (uint32_t)p.M * p.K * 2);
  const int it_beg = ks * p.ips, it_end = min(p.K / kIterK, it_beg + p.ips);
  f32x4 acc[2][4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < 4; ++s) acc[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint64_t owned = 0;  // tokens of this part's slots
  const TileSlots slots0(p, m0, pa, p.PA);
  uint32_t xoff[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) xoff[s] = (uint32_t)min(m0 + 16 * s + lr, p.M - 1) * p.K * 2 + 16 * lg;
  for (int it = it_beg + wave; it < it_end; it += 4) {
    const uint32_t kb = (uint32_t)it * (kIterK * 2);
    u32x4 xv[4][4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) xv[s][jj] = bld128(rx, xoff[s] + kb + 64 * jj);
    TileSlots slots = slots0;
    int a;
    uint64_t toks;
    while (slots.next(&a, &toks)) {
      const int r = rank_of(p, a) - 32 * rg;  // ranks of this group
      if (r <= 0) continue;
      const rsrc_t ra = make_rsrc(p.A + (size_t)a * p.a_stride, (uint32_t)p.R * p.K * 2);
      u32x4 av[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
          av[t][jj] = bld128(ra, 16 * t + lr < r ? (uint32_t)(32 * rg + 16 * t + lr) * p.K * 2 + 16 * lg + kb + 64 * jj : kOOB);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const uint32_t st = (uint32_t)(toks >> (16 * s)) & 0xFFFFu;
        if (st == 0) continue;  // uniform
        const bool in = (st >> lr) & 1;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4 q = acc[t][s];
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) q = mfma16<DT>(av[t][jj], xv[s][jj], q);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][s][e] = in ? q[e] : acc[t][s][e];
        }
      }
    }
  }
  {
    TileSlots slots = slots0;
    int a;
    uint64_t toks;
    while (slots.next(&a, &toks)) owned |= toks;
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < 4; ++s) *(f32x4*)(red[wave][t][s] + 4 * lane) = acc[t][s];
  __syncthreads();
  const auto scale_of = [&](int tok) {
    const int a = slot_of(p, m0 + tok);
    return p.scale && a >= 0 ? p.scale[a] : 1.f;
  };
  for (int i = threadIdx.x; i < 2048; i += 256) {
    const int ts = i >> 8, t = ts >> 2, s = ts & 3, l = (i & 255) >> 2, e = i & 3;
    const int tok = 16 * s + (l & 15), j = 16 * t + 4 * (l >> 4) + e;
    if (!((owned >> tok) & 1)) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) v += red[w][t][s][4 * l + e];
    // (ranks past the slot's: zero even where the token holds an infinity)
    if (32 * rg + j >= rank_of(p, slot_of(p, m0 + tok))) v = 0.f;
    if (p.P == 1) u[tok][j] = scale_of(tok) * v;
    else st_agent(p.upart + ((size_t)ks * p.M + m0 + tok) * W + 32 * rg + j, v);
  }
  if (p.P > 1) {
    complete_and_sync();
    if (threadIdx.x == 0) s_last = arrive_last(p.ctr + tb * p.RG + rg, (uint32_t)(p.P * p.PA)) ? 1 : 0;
    __syncthreads();
    if (!s_last) return;
    // (tokens without a slot: whatever lies there, never used)
    const rsrc_t rp = make_rsrc(p.upart, (uint32_t)p.P * p.M * W * 4);
    sum_slices(rp, p.P, cnt * 32,
               [&](int q, int i) { return (uint32_t)((q * p.M + m0 + (i >> 5)) * W + 32 * rg + (i & 31)) * 4u; },
               [&](int i, float v) { u[i >> 5][i & 31] = scale_of(i >> 5) * v; });
    owned = ~0ull;
  }
  __syncthreads();
  store_parts<DT>(cnt, &u[0][0], 33, p.uh + 32 * rg, p.ul + 32 * rg, W, p.us + rg, p.RG,
                  [&](int t) { return (owned >> t) & 1 ? m0 + t : -1; });
}

// The term of 64 tokens and 32 rpw rows a wave, part pa of PA (the tokens
// without a slot belong to part 0). NKK: rank groups whose parts of u stay in
// registers (0: read again for each slot and row pair).
template <int DT, int NKK>
__device__ __forceinline__ void expand_tile(const AdapterParams& p, int b) {
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = p.chunks * p.PA, tb = b / per, rem = b - tb * per, chunk = rem / p.PA, pa = rem - chunk * p.PA;
  const int m0 = 64 * tb, W = 32 * p.RG;
  const TileSlots slots0(p, m0, pa, p.PA);
  const bool vec = (p.R & 7) == 0 && (p.b_stride & 7) == 0;
  uint64_t owned = pa == 0 ? __ballot(slots0.id == -1) : 0;
  {
    TileSlots slots = slots0;
    int a;
    uint64_t toks;
    while (slots.next(&a, &toks)) owned |= toks;
  }
  if (!owned) return;
  auto part = [&](int s, int kk, u32x4& hi, u32x4& lo, float& sc) {
    const size_t m = (size_t)min(m0 + 16 * s + lr, p.M - 1);
    hi = ldg16(p.uh + m * W + 32 * kk + 8 * lg);
    lo = ldg16(p.ul + m * W + 32 * kk + 8 * lg);
    sc = DT == DT_F16 ? p.us[m * p.RG + kk] : 1.f;
  };
  constexpr int H = NKK > 0 ? NKK : 1;
  u32x4 hi[H][4], lo[H][4];
  float sc[H][4];
  if constexpr (NKK > 0) {
#pragma unroll
    for (int kk = 0; kk < H; ++kk)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (kk < p.RG) part(s, kk, hi[kk][s], lo[kk][s], sc[kk][s]);
  }
  const int rows = 128 * p.rpw;
  for (int n = chunk * rows + 32 * wave; n < min(p.N, (chunk + 1) * rows); n += 128) {
    f32x4 acc[4][2];
#pragma unroll
    for (int s = 0; s < 4; ++s) acc[s][0] = acc[s][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    TileSlots slots = slots0;
    int a;
    uint64_t toks;
    while (slots.next(&a, &toks)) {
      const int r = rank_of(p, a), nkk = (r + 31) >> 5;
      const rsrc_t rb = make_rsrc(p.B + (size_t)a * p.b_stride, (uint32_t)p.N * p.R * 2);
      f32x4 v[4][2];
#pragma unroll
      for (int s = 0; s < 4; ++s) v[s][0] = v[s][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      auto group = [&](int kk, const u32x4 (&h)[4], const u32x4 (&l)[4], const float (&c)[4]) {
        u32x4 bf[2];
        load_pair<DT>(p, rb, n, kk, r, vec, bf);
        if (vec && (r & 7)) mask_pair(kk, r, bf);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          if (((toks >> (16 * s)) & 0xFFFFu) == 0) continue;  // uniform
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if constexpr (DT == DT_F16) {
              f32x4 q = f32x4{0.f, 0.f, 0.f, 0.f};
              q = mfma16<DT>(bf[t], h[s], q);
              q = mfma16<DT>(bf[t], l[s], q);
              v[s][t] += c[s] * q;
            } else {
              v[s][t] = mfma16<DT>(bf[t], h[s], v[s][t]);
              v[s][t] = mfma16<DT>(bf[t], l[s], v[s][t]);
            }
          }
        }
      };
      if constexpr (NKK > 0) {
#pragma unroll
        for (int kk = 0; kk < H; ++kk)
          if (kk < nkk) group(kk, hi[kk], lo[kk], sc[kk]);
      } else {
        for (int kk = 0; kk < nkk; ++kk) {
#pragma unroll
          for (int s = 0; s < 4; ++s) part(s, kk, hi[0][s], lo[0][s], sc[0][s]);
          group(kk, hi[0], lo[0], sc[0]);
        }
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const bool in = (toks >> (16 * s + lr)) & 1;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[s][t][e] = in ? v[s][t][e] : acc[s][t][e];
      }
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if ((owned >> (16 * s + lr)) & 1) store_term<DT>(p, m0 + 16 * s + lr, n + 8 * lg, acc[s]);
  }
}

// ---------------------------------------------------------------------------
// kernels: up to kGroupMax layers a launch, each with workgroups of its own
// ---------------------------------------------------------------------------
__device__ __forceinline__ int member(const int (&start)[kGroupMax + 1], int n, int b) {
  int i = 0;
#pragma unroll
  for (int j = 1; j < kGroupMax; ++j)
    if (j < n && b >= start[j]) i = j;
  return i;
}

template <int DT, bool TILE>
__global__ __launch_bounds__(256) void k_adapter_shrink(AdapterGroup g) {
  const int i = member(g.shrink_start, g.n, blockIdx.x), b = blockIdx.x - g.shrink_start[i];
  if constexpr (TILE) shrink_tile<DT>(g.p[i], b);
  else shrink_group<DT>(g.p[i], b);
}

template <int DT, int NKK>
__global__ __launch_bounds__(256) void k_adapter_expand_tile(AdapterGroup g) {
  const int i = member(g.expand_start, g.n, blockIdx.x);
  expand_tile<DT, NKK>(g.p[i], blockIdx.x - g.expand_start[i]);
}

template <int DT>
__global__ __launch_bounds__(256) void k_adapter_expand(AdapterGroup g) {
  __shared__ int stok[16];
  const int i = member(g.expand_start, g.n, blockIdx.x), b = blockIdx.x - g.expand_start[i];
  const AdapterParams& p = g.p[i];
  const int m = b / p.chunks, chunk = b - m * p.chunks;
  const TokenGroup t = token_group(p, m, stok);
  if (t.cnt == 0) return;
  const int lg = (threadIdx.x & 63) >> 4, W = 32 * p.RG, rows = 128 * p.rpw;
  expand_group<DT>(p, t, chunk * rows, min(p.N, (chunk + 1) * rows), [&](int kk, u32x4& hi, u32x4& lo, float& sc) {
    hi = ldg16(p.uh + (size_t)t.tok * W + 32 * kk + 8 * lg);
    lo = ldg16(p.ul + (size_t)t.tok * W + 32 * kk + 8 * lg);
    sc = DT == DT_F16 ? p.us[(size_t)t.tok * p.RG + kk] : 1.f;
  });
}

// ---------------------------------------------------------------------------
// launcher
// ---------------------------------------------------------------------------
hipError_t SPEAR_D(launch_adapters)(const AdapterGroup& all, hipStream_t st) {
  // members of the decode kind and of the other kind in launches of their own
  for (int tile = 0; tile < 2; ++tile) {
    AdapterGroup g;
    g.n = 0;
    g.shrink_start[0] = g.expand_start[0] = 0;
    int rg = 0;
    for (int i = 0; i < all.n; ++i) {
      const AdapterParams& p = all.p[i];
      if (p.tile != tile) continue;
      const int units = tile ? (p.M + 63) / 64 * p.PA : p.M;
      g.p[g.n] = p;
      g.shrink_start[g.n + 1] = g.shrink_start[g.n] + units * p.P * p.RG;
      g.expand_start[g.n + 1] = g.expand_start[g.n] + units * p.chunks;
      rg = std::max(rg, p.RG);
      ++g.n;
    }
    if (g.n == 0) continue;
    const auto go = [&](auto kern, int grid) {
      hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, st, g);
      return hipGetLastError();
    };
    const int gs = g.shrink_start[g.n], ge = g.expand_start[g.n];
    hipError_t err = tile ? go(k_adapter_shrink<DTC, true>, gs) : go(k_adapter_shrink<DTC, false>, gs);
    if (err != hipSuccess) return err;
    if (!tile) err = go(k_adapter_expand<DTC>, ge);
    else if (rg == 1) err = go(k_adapter_expand_tile<DTC, 1>, ge);
    else if (rg == 2) err = go(k_adapter_expand_tile<DTC, 2>, ge);
    else err = go(k_adapter_expand_tile<DTC, 0>, ge);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace spear
