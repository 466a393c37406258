// gfx950 (MI355X) kernels of the low-rank adapters of many requests: the term
//   d[m] = res[m] + s_a B_a (A_a x[m]),   a = ids[m] (d[m] = res[m] without one)
// that the 4-bit product's final store adds in place of a residual, or that
// takes the product's sums (yf, fp32) up and is the layer's output.
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
// Up to 128 tokens (their coordinates in spear_adapters.h) the tokens of one slot
// among 64, up to 16 of them, belong to the workgroups of the first of them
// ("leader"); the other tokens' workgroups end at once. Nothing needs sorting,
// and the ids are read on the device. Beyond, a workgroup owns 64 consecutive
// tokens and walks the slots they name.
//
// The coordinates leave as sums over K-slices, which every workgroup of the
// second step adds up for its own tokens: a few KB from L2 each, in place of a
// last arriver that sums them alone (8B down, K = 14336, 300 tokens: 32 us for
// the first step that way, 18 and 3 more in the second this way, as both were
// built then; now 8.3 and 8.1). One launch
// that forms u anew in each workgroup of the term was slower wherever A is not
// tiny: a CU draws about 12 bytes a cycle from its L2 (8B gate and up at eight
// requests 17.8 us against 12.0 for the two, o 14.0 against 10.2; 8B q, k, v at 16
// requests 9.4 against 10.1; 1B q at one token, rank 8, 6.1 against 8.2).
#include "spear_adapters.h"

namespace spear {

// ---------------------------------------------------------------------------
// u for the term
// ---------------------------------------------------------------------------

// The parts of u for the term, in LDS: [T tokens][32 RG + 8] high, the same low,
// [T][RG] scales.
struct Parts {
  uint16_t *hi, *lo;
  float* sc;
  int ld, RG;
  __device__ __forceinline__ Parts(char* lds, int T, int RG_) : ld(32 * RG_ + 8), RG(RG_) {
    hi = (uint16_t*)lds;
    lo = hi + T * ld;
    sc = (float*)(lo + T * ld);
  }
  // the parts of token t's ranks j .. j + 4
  template <int DT>
  __device__ __forceinline__ void put(int t, int j, const f32x4& v) const {
    uint16_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) split_parts<DT>(v[e], &h[e], &l[e]);
    *(u32x2*)(hi + t * ld + j) = u32x2{h[0] | ((uint32_t)h[1] << 16), h[2] | ((uint32_t)h[3] << 16)};
    *(u32x2*)(lo + t * ld + j) = u32x2{l[0] | ((uint32_t)l[1] << 16), l[2] | ((uint32_t)l[3] << 16)};
  }
  // this lane's fragment of token t, rank group kk
  __device__ __forceinline__ void get(int t, int kk, u32x4& h, u32x4& l, float& f) const {
    const int o = t * ld + 32 * kk + 8 * ((threadIdx.x & 63) >> 4);
    h = *(const u32x4*)(hi + o);
    l = *(const u32x4*)(lo + o);
    f = sc[t * RG + kk];
  }
};
// Fills them for T tokens: val(t, j) gives u of token t, ranks j .. j + 4. Eight
// threads hold a token's rank group. Ends with a barrier.
template <int DT, class Val>
__device__ __forceinline__ void build_parts(const Parts& o, int T, Val val) {
  const int G = 8 * o.RG;  // threads a token
  for (int i = threadIdx.x; i < T * G; i += blockDim.x) {  // (T G is a multiple of 64)
    const int t = i / G, q = i - t * G;
    f32x4 v = val(t, 4 * q);
    if constexpr (DT == DT_F16) {
      float mx = fmaxf(fmaxf(__builtin_fabsf(v[0]), __builtin_fabsf(v[1])), fmaxf(__builtin_fabsf(v[2]), __builtin_fabsf(v[3])));
#pragma unroll
      for (int h = 4; h > 0; h >>= 1) mx = fmaxf(mx, __shfl_xor(mx, h));
      const int k = scale_exp(mx);
      v *= exp2i(k);
      if ((q & 7) == 0) o.sc[t * o.RG + (q >> 3)] = exp2i(-k);
    }
    o.template put<DT>(t, 4 * q, v);
  }
  __syncthreads();
}
// u of token m, ranks j .. j + 4, from the K-slices' sums: scaled, zero from
// rank r on (whose sums were never written)
__device__ __forceinline__ f32x4 sum_u(const AdapterParams& p, int m, int j, int r, float scale) {
  const int W = 32 * p.RG;
  const rsrc_t ru = make_rsrc(p.upart, (uint32_t)p.P * p.M * W * 4);
  f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int q0 = 0; q0 < p.P; q0 += 8) {
    f32x4 w[8];
#pragma unroll
    for (int q = 0; q < 8; ++q)
      w[q] = __builtin_bit_cast(f32x4, bld128(ru, q0 + q < p.P ? (uint32_t)(((q0 + q) * p.M + m) * W + j) * 4u : kOOB));
#pragma unroll
    for (int q = 0; q < 8; ++q) s += w[q];  // (slices past the last read as zero)
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = j + e < r ? scale * s[e] : 0.f;
  return s;
}

// ---------------------------------------------------------------------------
// the term
// ---------------------------------------------------------------------------

// 64 rows of B_a from n0, rank group kk, as four MFMA row tiles: row q of tile
// t is row 32 (t / 2) + 8 (q / 4) + 4 (t % 2) + q % 4, so that a lane's results
// are two runs of eight consecutive rows. Ranks from r on are not used (of a
// whole chunk of eight they are read and put to zero).
struct RowLanes {
  uint32_t off[4];  // this lane's row of each tile at n0 = 0, ranks 8 lg
  bool vec;         // rows of whole, aligned chunks of eight ranks
  __device__ __forceinline__ explicit RowLanes(const AdapterParams& p) {
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      off[t] = (uint32_t)((32 * (t >> 1) + 8 * (lr >> 2) + 4 * (t & 1) + (lr & 3)) * p.R + 8 * lg) * 2;
    vec = (p.R & 7) == 0 && (p.b_stride & 7) == 0;
  }
};
// (rows from N on lie past the buffer rb of the slot's N R values: zero)
__device__ __forceinline__ void load_rows(const AdapterParams& p, const RowLanes& o, rsrc_t rb, int n0, int kk, int r,
                                          u32x4 (&bf)[4]) {
  const int lg = (threadIdx.x & 63) >> 4, j0 = 32 * kk + 8 * lg;
  const uint32_t base = ((uint32_t)n0 * p.R + 32 * kk) * 2;  // (past the slot where n0 >= N: not a scalar offset)
  if (o.vec) {
    const bool ok = j0 < r;
#pragma unroll
    for (int t = 0; t < 4; ++t) bf[t] = bld128(rb, ok ? o.off[t] + base : kOOB);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = j0 + 2 * q;
        bf[t][q] = bld16(rb, j < r ? o.off[t] + base + 4 * q : kOOB) |
                   (bld16(rb, j + 1 < r ? o.off[t] + base + 4 * q + 2 : kOOB) << 16);
      }
  }
}
// ranks from r on to zero (where they were read: of the slot's R)
__device__ __forceinline__ void mask_rows(int kk, int r, u32x4 (&bf)[4]) {
  const int j0 = 32 * kk + 8 * ((threadIdx.x & 63) >> 4);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t keep = (j0 + 2 * q < r ? 0xFFFFu : 0u) | (j0 + 2 * q + 1 < r ? 0xFFFF0000u : 0u);
#pragma unroll
    for (int t = 0; t < 4; ++t) bf[t][q] &= keep;
  }
}
// v += the rank group's product with the parts of u at hi, lo (undone by sc)
template <int DT>
__device__ __forceinline__ void add_product(const u32x4 (&bf)[4], u32x4 hi, u32x4 lo, float sc, f32x4 (&v)[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
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

// What the term of a lane's token is added to, its rows n + 8 lg and n + 32 + 8
// lg (eight each): the residual and the layer's sums.
struct Base {
  u32x4 res[2];
  f32x4 yf[4];
};
__device__ __forceinline__ void load_base(const AdapterParams& p, bool live, int m, int n, Base& b) {
  const int lg = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int nn = n + 32 * h + 8 * lg;
    if ((p.N & 7) == 0 && live && nn < p.N) {
      if (p.res) b.res[h] = ldg16(p.res + (size_t)m * p.N + nn);
      if (p.yf) {
        const f32x4* y = (const f32x4*)(p.yf + (size_t)m * p.N + nn);
        b.yf[2 * h] = y[0], b.yf[2 * h + 1] = y[1];
      }
    }
  }
}
// d of those rows: one rounding of the sum
template <int DT>
__device__ __forceinline__ void store_term(const AdapterParams& p, bool live, int m, int n, const Base& b,
                                           const f32x4 (&v)[4]) {
  const int lg = (threadIdx.x & 63) >> 4;
  if (!live) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int nn = n + 32 * h + 8 * lg;
    if (nn >= p.N) continue;
    const size_t o = (size_t)m * p.N + nn;
    if ((p.N & 7) == 0) {
      f32x4 f[2] = {v[2 * h], v[2 * h + 1]};
      if (p.yf) f[0] += b.yf[2 * h], f[1] += b.yf[2 * h + 1];  // (uniform)
      if (p.res) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e >> 2][e & 3] += act2f<DT>((b.res[h][e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
      }
      u32x4 w;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float x = f[q >> 1][2 * (q & 1)], y = f[q >> 1][2 * (q & 1) + 1];
        if constexpr (DT == DT_BF16) w[q] = pack_bf16(x, y);
        else w[q] = (uint32_t)f2act<DT>(x) | ((uint32_t)f2act<DT>(y) << 16);
      }
      *(u32x4*)(p.d + o) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (nn + e < p.N)
          p.d[o + e] = f2act<DT>(v[2 * h + (e >> 2)][e & 3] + (p.res ? act2f<DT>(p.res[o + e]) : 0.f) +
                                 (p.yf ? p.yf[o + e] : 0.f));
    }
  }
}

// Rows [n0, n1) of the term of up to 16 tokens of one slot (lane's token tok,
// live), 64 at a time, every `step` from the wave's first; the first 64 rows'
// operands are requested by the constructor, before u is there.
template <int DT>
struct SlotTerm {
  const AdapterParams& p;
  const RowLanes lanes;
  rsrc_t rb;
  int tok, n0;
  bool live;
  u32x4 bf[4];
  Base base;
  // (columns past the slot's rank are read and dropped: nothing waits for it)
  __device__ __forceinline__ SlotTerm(const AdapterParams& p_, int a, bool live_, int tok_, int n)
      : p(p_), lanes(p_), tok(tok_), n0(n), live(live_) {
    rb = make_rsrc(p.B + (size_t)max(a, 0) * p.b_stride, a < 0 ? 0u : (uint32_t)p.N * p.R * 2);
    load_rows(p, lanes, rb, n, 0, p.R, bf);
    load_base(p, live, tok, n, base);
  }
  __device__ __forceinline__ void rows(int n1, int step, int r, const Parts& parts) {
    const int nkk = (r + 31) >> 5;
    for (int n = n0; n < n1; n += step) {
      f32x4 v[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (n != n0) load_base(p, live, tok, n, base);
      for (int kk = 0; kk < nkk; ++kk) {
        if (n != n0 || kk > 0) load_rows(p, lanes, rb, n, kk, p.R, bf);
        u32x4 hi, lo;
        float f;
        parts.get(threadIdx.x & 15, kk, hi, lo, f);
        if (r < min(p.R, 32 * kk + 32)) mask_rows(kk, r, bf);
        add_product<DT>(bf, hi, lo, f, v);
      }
      store_term<DT>(p, live, tok, n, base, v);
    }
  }
};

// ---------------------------------------------------------------------------
// beyond: 64 consecutive tokens
// ---------------------------------------------------------------------------

// The slots that consecutive tokens name, one after another: each lane holds
// one token's slot and rank (-1: none, and ranks of zero, count as none).
// next() gives the tokens of the next slot, of those left in `left`.
struct TileSlots {
  int id, rank;
  uint64_t left;
  __device__ __forceinline__ bool next(int* a, int* r, uint64_t* toks) {
    if (!left) return false;
    const int l = __builtin_ctzll(left);
    *a = __builtin_amdgcn_readlane(id, l);
    *r = __builtin_amdgcn_readlane(rank, l);
    *toks = __ballot(id == *a) & left;
    left &= ~*toks;
    return true;
  }
};
__device__ __forceinline__ TileSlots tile_slots(const AdapterParams& p, int m0) {
  TileSlots t;
  const int m = m0 + (threadIdx.x & 63);
  t.id = m < p.M ? slot_of(p, m) : -1;
  t.rank = rank_of(p, t.id);
  t.left = __ballot(t.rank > 0);
  return t;
}

// The activations come into LDS by direct loads of whole 256-byte pieces of four
// rows each (in the MFMA's layout a load takes 64 bytes of each of 16 rows, twice
// the requests, and the requests in flight are the bound), each wave's own 16 KB,
// chunk c of row t at c ^ (t % 16).
template <int DT>
__device__ __forceinline__ void shrink_tile(const AdapterParams& p, int b) {
  __shared__ __attribute__((aligned(16))) uint16_t xs[4][64 * kIterK];
  float (*red)[2][4][256] = (float (*)[2][4][256])&xs[0][0];  // (after the last iteration)
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = p.P * p.RG * p.PA, tb = b / per;
  int rem = b - tb * per;
  const int rg = rem / (p.P * p.PA);
  rem -= rg * p.P * p.PA;
  const int ks = rem / p.PA, pa = rem - ks * p.PA;
  const int m0 = 64 * tb, W = 32 * p.RG;
  const rsrc_t rx = make_rsrc(p.x, (uint32_t)p.M * p.K * 2);
  const int it_beg = ks * p.ips, it_end = min(p.K / kIterK, it_beg + p.ips);
  TileSlots slots = tile_slots(p, m0);
  // this part's slots: the i-th with i % PA == pa, of those that reach the rank group
  uint64_t owned = slots.left;
  if (p.PA > 1) {
    TileSlots t = slots;
    owned = 0;
    int a, r;
    uint64_t toks;
    for (int i = 0; t.next(&a, &r, &toks); ++i)
      if (i % p.PA == pa) owned |= toks;
  }
  owned &= __ballot(slots.rank > 32 * rg);
  if (!owned) return;
  f32x4 acc[2][4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < 4; ++s) acc[t][s] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t xoff[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) xoff[u] = (uint32_t)(m0 + 4 * u + lg) * p.K * 2 + 16 * (lr ^ (4 * u + lg));
  const uint32_t xlast = (uint32_t)(p.M - 1) * p.K * 2 + 240;  // (for tokens past the last: no slot owns them)
  uint16_t* xw = xs[wave];
  const uint32_t aoff = (uint32_t)(32 * rg + lr) * p.K * 2 + 16 * lg;
  for (int it = it_beg + wave; it < it_end; it += 4) {
    const uint32_t kb = (uint32_t)it * (kIterK * 2);
#pragma unroll
    for (int u = 0; u < 16; ++u)
      bld128_lds(rx, xw + u * 512, min(xoff[u & 3] + (uint32_t)(16 * (u >> 2)) * p.K * 2, xlast) + kb);
    // a slot's rows of A, requested one slot ahead
    TileSlots t0 = slots;
    t0.left = owned;
    int r = 0, rn = 0;
    uint64_t toks = 0, tn = 0;
    u32x4 av[2][4], nv[2][4];
    auto request = [&]() {
      int a;
      if (!t0.next(&a, &rn, &tn)) {
        tn = 0;
        return;
      }
      rn -= 32 * rg;
      const rsrc_t ra = make_rsrc(p.A + (size_t)a * p.a_stride, (uint32_t)p.R * p.K * 2);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t ao = 16 * t + lr < rn ? aoff + (uint32_t)t * 32 * p.K : kOOB;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) nv[t][jj] = bld128s(ra, ao + 64 * jj, kb);
      }
    };
    request();
    // the activations, with the first slot's rows
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    while (tn) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) av[t][jj] = nv[t][jj];
      r = rn, toks = tn;
      request();
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const uint32_t st = (uint32_t)(toks >> (16 * s)) & 0xFFFFu;
        if (st == 0) continue;  // uniform
        const bool in = (st >> lr) & 1;
        u32x4 xv[4];
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
          xv[jj] = *(const u32x4*)(xw + (16 * s + lr) * kIterK + 8 * ((lg + 4 * jj) ^ lr));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (16 * t >= r) continue;  // uniform
          f32x4 q = acc[t][s];
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) q = mfma16<DT>(av[t][jj], xv[jj], q);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][s][e] = in ? q[e] : acc[t][s][e];
        }
      }
    }
    // the reads are done before the next iteration's loads write there
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < 4; ++s) *(f32x4*)(red[wave][t][s] + 4 * lane) = acc[t][s];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {  // eight tiles of results, 64 threads each
    const int ts = 4 * i + wave, t = ts >> 2, s = ts & 3, tok = 16 * s + lr;
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) v += *(const f32x4*)(red[w][t][s] + 4 * lane);
    if ((owned >> tok) & 1)
      *(f32x4*)(p.upart + ((size_t)ks * p.M + m0 + tok) * W + 32 * rg + 16 * t + 4 * lg) = v;
  }
}

// The term of 64 tokens, 16 a wave (the waves walk the same rows, so that B
// comes from memory once for the four), over 64 rpw rows. A wave walks (64
// rows, slot, rank group) with the fragments of B one item ahead.
template <int DT>
__device__ __forceinline__ void expand_tile(const AdapterParams& p, int b, char* smem) {
  const int lane = threadIdx.x & 63, lr = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tb = b / p.chunks, chunk = b - tb * p.chunks;
  const int m0 = 64 * tb + 16 * wave;
  const Parts parts(smem, 64, p.RG);
  build_parts<DT>(parts, 64, [&](int t, int j) {
    const int m = 64 * tb + t, mm = min(m, p.M - 1), a = m < p.M ? slot_of(p, mm) : -1;
    return sum_u(p, mm, j, rank_of(p, a), p.scale && a >= 0 ? p.scale[a] : 1.f);
  });
  if (m0 >= p.M) return;
  TileSlots all;
  {
    const int m = m0 + lr;  // (four lanes a token; lanes 0 to 15 count)
    all.id = m < p.M ? slot_of(p, m) : -1;
    all.rank = rank_of(p, all.id);
    all.left = __ballot(all.rank > 0) & 0xFFFFu;
  }
  const int m = min(m0 + lr, p.M - 1);
  const bool live = m0 + lr < p.M;
  const RowLanes lanes(p);
  const int n_beg = chunk * 64 * p.rpw, n_end = min(p.N, n_beg + 64 * p.rpw);

  struct Item {
    int n, a, r, kk;
    uint32_t toks;
  };
  TileSlots left = all;
  auto first_slot = [&](Item& t) {
    left.left = all.left;
    uint64_t m64 = 0;
    t.kk = 0;
    t.r = 0;
    t.a = 0;
    left.next(&t.a, &t.r, &m64);
    t.toks = (uint32_t)m64;
  };
  auto advance = [&](Item& t) {
    if (32 * (t.kk + 1) < t.r) {
      ++t.kk;
      return;
    }
    uint64_t m64 = 0;
    if (left.next(&t.a, &t.r, &m64)) {
      t.toks = (uint32_t)m64;
      t.kk = 0;
      return;
    }
    t.n += 64;
    first_slot(t);
  };
  auto load = [&](const Item& t, u32x4 (&bf)[4]) {
    const rsrc_t rb = make_rsrc(p.B + (size_t)t.a * p.b_stride, t.r > 0 ? (uint32_t)p.N * p.R * 2 : 0u);
    load_rows(p, lanes, rb, t.n, t.kk, t.r, bf);
  };
  Item cur;
  cur.n = n_beg;
  first_slot(cur);
  u32x4 bf[4], nx[4];
  load(cur, bf);
  f32x4 acc[4], v[4];
  Base base;
#pragma unroll
  for (int t = 0; t < 4; ++t) acc[t] = v[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  load_base(p, live, m, cur.n, base);
  while (cur.n < n_end) {
    Item nxt = cur;
    advance(nxt);
    if (nxt.n < n_end) load(nxt, nx);
    if (cur.r > 0) {
      if (lanes.vec && (cur.r & 7)) mask_rows(cur.kk, cur.r, bf);
      u32x4 hi, lo;
      float sc;
      parts.get(16 * wave + lr, cur.kk, hi, lo, sc);
      add_product<DT>(bf, hi, lo, sc, v);
    }
    if (nxt.kk == 0) {  // the slot's last rank group
      const bool in = (cur.toks >> lr) & 1;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] = in ? v[t][e] : acc[t][e];
        v[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    if (nxt.n != cur.n) {
      store_term<DT>(p, live, m, cur.n, base, acc);
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (nxt.n < n_end) load_base(p, live, m, nxt.n, base);
    }
    cur = nxt;
#pragma unroll
    for (int t = 0; t < 4; ++t) bf[t] = nx[t];
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

// The parts of u once, for a GEMM whose tiles each read them: 16 threads a token,
// four ranks of each 64. The GEMM adds them to the product's own sums, so that
// small coordinates need no scaling (a part is off by at most 2^-25); those past
// fp16's range are divided by a power of two that its weight tile is multiplied by.
template <int DT>
__global__ __launch_bounds__(256) void k_adapter_parts(AdapterGroup g) {
  const int b = member(g.expand_start, g.n, blockIdx.x);
  const AdapterParams& p = g.p[b];
  const int m = (blockIdx.x - g.expand_start[b]) * 16 + (threadIdx.x >> 4), q = threadIdx.x & 15, W = 32 * p.RG;
  const int mm = min(m, p.M - 1), a = slot_of(p, mm), r = rank_of(p, a);
  const float sc = p.scale && a >= 0 ? p.scale[a] : 1.f;
  int k = 0;
  f32x4 v = sum_u(p, mm, min(4 * q, W - 4), r, sc);
  if constexpr (DT == DT_F16) {
    float mx = 0.f;
    f32x4 w = v;
    for (int j = 4 * q;;) {
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = __builtin_fabsf(w[e]) < __builtin_inff() ? fmaxf(mx, __builtin_fabsf(w[e])) : mx;
      j += 64;
      if (j >= W) break;
      w = sum_u(p, mm, j, r, sc);
    }
#pragma unroll
    for (int h = 8; h > 0; h >>= 1) mx = fmaxf(mx, __shfl_xor(mx, h));
    k = mx > 65504.f ? (int)(__float_as_uint(mx) >> 23) - 127 - 14 : 0;
  }
  if (m >= p.M) return;
  if (q == 0) p.ukx[m] = k;
  for (int j = 4 * q; j < W; j += 64) {
    if (j >= 64) v = sum_u(p, mm, j, r, sc);
    uint16_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) split_parts<DT>(v[e] * exp2i(-k), &h[e], &l[e]);
    const size_t at = (size_t)m * W + j;
    *(u32x2*)(p.uh + at) = u32x2{h[0] | ((uint32_t)h[1] << 16), h[2] | ((uint32_t)h[3] << 16)};
    *(u32x2*)(p.ul + at) = u32x2{l[0] | ((uint32_t)l[1] << 16), l[2] | ((uint32_t)l[3] << 16)};
  }
}

// (a single member's call passes its parameters alone: the table's lookup is a
// dependent load ahead of everything else)
template <int DT, int KIND>
__device__ __forceinline__ void shrink_body(const AdapterParams& p, int b) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  if constexpr (KIND == ADAPT_TILES) shrink_tile<DT>(p, b);
  else shrink_slot<DT>(p, b, smem);
}
template <int DT, int KIND>
__device__ __forceinline__ void expand_body(const AdapterParams& p, int b, char* smem) {
  if constexpr (KIND == ADAPT_TILES) {
    expand_tile<DT>(p, b, smem);
  } else {
    __shared__ int stok[16];
    const int m = b / p.chunks, chunk = b - m * p.chunks;
    const TokenGroup t = token_group(p, m, stok);
    if (t.cnt == 0) return;
    const int rows = 256 * p.rpw, n0 = chunk * rows;
    SlotTerm<DT> term(p, t.a, (threadIdx.x & 15) < t.cnt, t.tok, n0 + 64 * (threadIdx.x >> 6));
    const Parts parts(smem, 16, p.RG);
    if (t.r > 0) {
      const float sc = p.scale ? p.scale[t.a] : 1.f;
      build_parts<DT>(parts, 16, [&](int i, int j) { return sum_u(p, stok[min(i, t.cnt - 1)], j, t.r, sc); });
    }
    term.rows(min(p.N, n0 + rows), 256, t.r, parts);
  }
}
template <int DT, int KIND>
__global__ __launch_bounds__(256) void k_adapter_shrink(AdapterParams p) {
  shrink_body<DT, KIND>(p, blockIdx.x);
}
template <int DT, int KIND>
__global__ __launch_bounds__(256) void k_adapter_shrink_group(AdapterGroup g) {
  const int i = member(g.shrink_start, g.n, blockIdx.x);
  shrink_body<DT, KIND>(g.p[i], blockIdx.x - g.shrink_start[i]);
}
template <int DT, int KIND>
__global__ __launch_bounds__(256) void k_adapter_expand(AdapterParams p) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  expand_body<DT, KIND>(p, blockIdx.x, smem);
}
template <int DT, int KIND>
__global__ __launch_bounds__(256) void k_adapter_expand_group(AdapterGroup g) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int i = member(g.expand_start, g.n, blockIdx.x);
  expand_body<DT, KIND>(g.p[i], blockIdx.x - g.expand_start[i], smem);
}

// ---------------------------------------------------------------------------
// launcher
// ---------------------------------------------------------------------------
// the members of one kind (they share its launches), their workgroups placed
template <int KIND>
static AdapterGroup of_kind(const AdapterGroup& all, size_t* parts_lds) {
  AdapterGroup g;
  g.n = 0;
  g.shrink_start[0] = g.expand_start[0] = 0;
  *parts_lds = 0;
  for (int i = 0; i < all.n; ++i) {
    const AdapterParams& p = all.p[i];
    if (p.kind != KIND) continue;
    const int units = KIND == ADAPT_TILES ? (p.M + 63) / 64 : p.M, T = KIND == ADAPT_TILES ? 64 : 16;
    g.p[g.n] = p;
    g.shrink_start[g.n + 1] = g.shrink_start[g.n] + units * p.PA * p.P * p.RG;
    g.expand_start[g.n + 1] = g.expand_start[g.n] + units * p.chunks;
    *parts_lds = std::max(*parts_lds, (size_t)T * ((32 * p.RG + 8) * 4 + p.RG * 4));
    ++g.n;
  }
  return g;
}
template <class F, class P>
static hipError_t go(F kern, const P& p, int grid, size_t lds, hipStream_t st) {
  hipError_t err = allow_lds(kern, lds);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, st, p);
  return hipGetLastError();
}
template <int KIND>
static hipError_t shrink_kind(const AdapterGroup& all, hipStream_t st) {
  size_t lds;
  const AdapterGroup g = of_kind<KIND>(all, &lds);
  if (g.n == 0) return hipSuccess;
  lds = KIND == ADAPT_TILES ? 0 : shrink_slot_lds(4);
  return g.n == 1 ? go(k_adapter_shrink<DTC, KIND>, g.p[0], g.shrink_start[1], lds, st)
                  : go(k_adapter_shrink_group<DTC, KIND>, g, g.shrink_start[g.n], lds, st);
}
template <int KIND>
static hipError_t expand_kind(const AdapterGroup& all, hipStream_t st) {
  size_t lds;
  const AdapterGroup g = of_kind<KIND>(all, &lds);
  if (g.n == 0) return hipSuccess;
  return g.n == 1 ? go(k_adapter_expand<DTC, KIND>, g.p[0], g.expand_start[1], lds, st)
                  : go(k_adapter_expand_group<DTC, KIND>, g, g.expand_start[g.n], lds, st);
}

hipError_t SPEAR_D(launch_adapter_shrink)(const AdapterGroup& all, hipStream_t st) {
  const hipError_t err = shrink_kind<ADAPT_SLOTS>(all, st);
  return err != hipSuccess ? err : shrink_kind<ADAPT_TILES>(all, st);
}
hipError_t SPEAR_D(launch_adapter_parts)(const AdapterGroup& all, hipStream_t st) {
  AdapterGroup g = all;
  g.expand_start[0] = 0;
  for (int i = 0; i < g.n; ++i) g.expand_start[i + 1] = g.expand_start[i] + (g.p[i].M + 15) / 16;
  return go(k_adapter_parts<DTC>, g, g.expand_start[g.n], 0, st);
}
hipError_t SPEAR_D(launch_adapter_expand)(const AdapterGroup& all, hipStream_t st) {
  const hipError_t err = expand_kind<ADAPT_SLOTS>(all, st);
  return err != hipSuccess ? err : expand_kind<ADAPT_TILES>(all, st);
}

}  // namespace spear
