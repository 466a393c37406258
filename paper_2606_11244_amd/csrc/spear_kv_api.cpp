// Host side of spear_kv.h: checks of the arguments, launch shapes.
#include "spear_kv_internal.h"

#include <algorithm>
#include <cmath>
#include <cstring>

#include "spear_kv.h"

using namespace spear;

namespace {

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || na == 0 || nb == 0) return false;
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}
spear_status_t hip_status(hipError_t e) { return e == hipSuccess ? SPEAR_OK : SPEAR_E_HIP; }
// a launch of fewer than 2^32 threads
bool launches(int64_t blocks, int threads) { return blocks * threads < (int64_t)1 << 32; }
bool page_size(int p) { return p == 16 || p == 32 || p == 64 || p == 128; }

// a buffer; where row is given, only the first `row` of each `ld` bytes of it
struct Span {
  const void* p;
  size_t bytes, row = 0, ld = 0;
};
bool hits(const Span& a, const Span& b) {
  if (!overlaps(a.p, a.bytes, b.p, b.bytes)) return false;
  if (!a.row || !b.row || a.ld != b.ld) return true;
  // rows of one stride, as the parts of a packed projection: apart within the stride
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  const size_t d = x <= y ? (y - x) % a.ld : (a.ld - (x - y) % a.ld) % a.ld;
  return d < a.row || a.ld - d < b.row;
}
// whether one of outs overlaps another of them or one of ins
bool clash(const Span* outs, int n_outs, const Span* ins, int n_ins) {
  for (int i = 0; i < n_outs; ++i) {
    for (int j = i + 1; j < n_outs; ++j)
      if (hits(outs[i], outs[j])) return true;
    for (int j = 0; j < n_ins; ++j)
      if (hits(outs[i], ins[j])) return true;
  }
  return false;
}
// `rows` rows of `row` elements, `ld` apart, to the end of the last
Span rows_of(const void* p, int64_t rows, int64_t ld, int64_t row) {
  return {p, rows > 0 ? ((size_t)(rows - 1) * ld + row) * 2 : 0, (size_t)row * 2, (size_t)ld * 2};
}

spear_status_t check_cache(const spear_kv_cache_t* c, bool buffers = true) {
  if (!c) return SPEAR_E_NULL;
  if (c->format != SPEAR_KV_INT8 && c->format != SPEAR_KV_E4M3) return SPEAR_E_DTYPE;
  if (c->act_dtype != SPEAR_F16 && c->act_dtype != SPEAR_BF16) return SPEAR_E_DTYPE;
  if (c->kv_heads < 1 || c->kv_heads > 1024 || (c->head_dim != 64 && c->head_dim != 128) ||
      !page_size(c->page_tokens) || c->reserved != 0 || c->pages < 0 ||
      c->pages >= ((int64_t)1 << 31) / c->page_tokens)
    return SPEAR_E_SHAPE;
  if (!buffers) return SPEAR_OK;
  if (c->pages && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return SPEAR_E_NULL;
  if (off16(c->k) || off16(c->v) || off16(c->k_scale) || off16(c->v_scale)) return SPEAR_E_ALIGN;
  return SPEAR_OK;
}
KvCache cache_of(const spear_kv_cache_t* c) {
  return {(uint8_t*)c->k, (uint8_t*)c->v, c->k_scale, c->v_scale, c->kv_heads, c->head_dim, c->page_tokens, (int)c->pages};
}
// the cache's four buffers
void cache_spans(const spear_kv_cache_t* c, Span (&s)[4]) {
  const size_t heads = (size_t)c->pages * c->kv_heads, codes = heads * c->page_tokens * c->head_dim;
  s[0] = {c->k, codes}, s[1] = {c->v, codes}, s[2] = {c->k_scale, heads * 4}, s[3] = {c->v_scale, heads * 4};
}

spear_status_t check_batch(const spear_kv_batch_t* b, bool buffers = true) {
  if (!b) return SPEAR_E_NULL;
  if (b->requests < 0 || b->requests > kKvRequests || b->tokens < 0 || b->tokens > kKvTokens || b->max_new < 1 ||
      (b->tokens && b->max_new > b->tokens) || b->width < 1 || b->width > (1 << 26) ||
      (b->table_ld != 0 && b->table_ld < b->width) || b->reserved != 0)
    return SPEAR_E_SHAPE;
  if (!buffers) return SPEAR_OK;
  if (!b->starts || (b->requests && (!b->lens || !b->table))) return SPEAR_E_NULL;
  if (off4(b->starts) || off4(b->lens) || off4(b->table)) return SPEAR_E_ALIGN;
  return SPEAR_OK;
}
int64_t table_ld(const spear_kv_batch_t* b) { return b->table_ld ? b->table_ld : b->width; }
size_t table_bytes(const spear_kv_batch_t* b) {
  return b->requests ? ((size_t)(b->requests - 1) * table_ld(b) + b->width) * 4 : 0;
}

}  // namespace

spear_status_t spear_kv_pages(const spear_kv_batch_t* b, const spear_kv_pages_t* a, void* hip_stream) {
  if (!b || !a) return SPEAR_E_NULL;
  const spear_status_t st = check_batch(b);
  if (st != SPEAR_OK) return st;
  if (!page_size(a->page_tokens) || a->n_free < 0) return SPEAR_E_SHAPE;
  if (!a->taken || (b->requests && (!a->held || !a->fresh)) || (a->n_free && !a->free_pages) ||
      (b->tokens && (!a->slots || !a->positions)))
    return SPEAR_E_NULL;
  if (off4(a->held) || off4(a->fresh) || off4(a->free_pages) || off4(a->slots) || off4(a->positions) || off4(a->taken))
    return SPEAR_E_ALIGN;
  const size_t R = b->requests, T = b->tokens;
  const Span outs[] = {{b->starts, (R + 1) * 4}, {b->lens, R * 4},      {b->table, table_bytes(b)},
                       {a->slots, T * 4},        {a->positions, T * 4}, {a->taken, 8}};
  const Span ins[] = {{a->held, R * 4}, {a->fresh, R * 4}, {a->free_pages, (size_t)a->n_free * 4}};
  if (clash(outs, 6, ins, 3)) return SPEAR_E_ALIAS;
  KvPagesParams p;
  p.R = b->requests, p.T = b->tokens, p.P = a->page_tokens, p.width = b->width, p.n_free = a->n_free;
  p.ld = table_ld(b);
  p.held = a->held, p.fresh = a->fresh, p.free_pages = a->free_pages;
  p.starts = b->starts, p.lens = b->lens, p.table = b->table;
  p.slots = a->slots, p.positions = a->positions, p.taken = a->taken;
  return hip_status(launch_kv_pages(p, (hipStream_t)hip_stream));
}

spear_status_t spear_rope_frequencies(int32_t rotary_dim, double base, double factor, double context,
                                      double low_turns, double high_turns, uint64_t* freqs) {
  if (rotary_dim < 0 || rotary_dim % 2 || rotary_dim > 1 << 20 || !(base > 1.0) || !std::isfinite(base) ||
      !(factor >= 1.0) || !std::isfinite(factor) || !(context >= 0.0) || !std::isfinite(context))
    return SPEAR_E_SHAPE;
  const bool parts = factor > 1.0 && context > 0.0;
  if (parts && !(high_turns > low_turns && std::isfinite(high_turns) && std::isfinite(low_turns))) return SPEAR_E_SHAPE;
  if (rotary_dim && !freqs) return SPEAR_E_NULL;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    // turns a position, at most 0.16
    long double f = std::pow((long double)base, -2.0L * i / rotary_dim) / 6.283185307179586476925286766559L;
    long double share = factor > 1.0 ? 0.0L : 1.0L;
    if (parts)
      share = std::min(1.0L, std::max(0.0L, (f * context - low_turns) / ((long double)high_turns - low_turns)));
    f *= share + (1.0L - share) / factor;
    freqs[i] = (uint64_t)std::llround(f * 18446744073709551616.0L);
  }
  return SPEAR_OK;
}

spear_status_t spear_kv_append(const spear_kv_cache_t* c, const spear_kv_append_t* a, void* hip_stream) {
  if (!a) return SPEAR_E_NULL;
  spear_status_t st = check_cache(c);
  if (st != SPEAR_OK) return st;
  const int64_t T = a->tokens, kv = (int64_t)c->kv_heads * c->head_dim;
  const int64_t qd = a->q ? (int64_t)a->heads * c->head_dim : 0;
  if (T < 0 || T > kKvTokens || (a->q && (a->heads < 1 || a->heads > 1024))) return SPEAR_E_SHAPE;
  const spear_rope_t& r = a->rope;
  if (r.rotary_dim < 0 || r.rotary_dim > c->head_dim || r.rotary_dim % 2 || r.interleaved < 0 || r.interleaved > 1 ||
      r.reserved != 0 || (r.rotary_dim && !std::isfinite(r.magnitude)))
    return SPEAR_E_SHAPE;
  bool ld_ok = true;
  auto ld = [&](int64_t v, int64_t row) {
    const int64_t l = v == 0 ? row : v;
    ld_ok = ld_ok && l >= row && l % 8 == 0 && l < ((int64_t)1 << 30);
    return l;
  };
  const int64_t kl = ld(a->k_ld, kv), vl = ld(a->v_ld, kv);
  const int64_t ql = a->q ? ld(a->q_ld, qd) : 0, ol = a->q ? ld(a->q_out_ld, qd) : 0;
  if (!ld_ok) return SPEAR_E_SHAPE;
  // Workgroups of a window: in a decoding step every token is a run of its own, in prompts
  // most of the many find none and cost their start. 4096 tokens, pages of 64: 46 us with one
  // a window, 50 with four, 55 with eight; 7 prompts of 300, pages of 32: 19, 10 and 10.
  const int subs = (int)(T <= 1024 ? std::min<int64_t>(T, 64) : 4);
  const int64_t kv_blocks = (T + 63) / 64 * subs * c->kv_heads * 2, q_blocks = a->q ? T : 0;
  if (!launches(kv_blocks + q_blocks, 256)) return SPEAR_E_SHAPE;
  if (T == 0) return SPEAR_OK;
  if (!a->k || !a->v || !a->slots || (a->q && !a->q_out) || (r.rotary_dim && (!r.freqs || !a->positions)))
    return SPEAR_E_NULL;
  if (off16(a->k) || off16(a->v) || off16(a->q) || (a->q && off16(a->q_out)) || off4(a->slots) || off4(a->positions) ||
      (r.rotary_dim && (reinterpret_cast<uintptr_t>(r.freqs) & 7u)))
    return SPEAR_E_ALIGN;
  Span outs[5];
  cache_spans(c, reinterpret_cast<Span(&)[4]>(outs));
  outs[4] = rows_of(a->q ? a->q_out : nullptr, T, ol, qd);
  const bool in_place = a->q && a->q == a->q_out && ql == ol;
  const Span ins[] = {rows_of(a->k, T, kl, kv),
                      rows_of(a->v, T, vl, kv),
                      {a->slots, (size_t)T * 4},
                      {a->positions, r.rotary_dim ? (size_t)T * 4 : 0},
                      {r.freqs, (size_t)r.rotary_dim / 2 * 8},
                      rows_of(in_place ? nullptr : a->q, T, ql, qd)};
  if (clash(outs, 5, ins, 6) || (in_place && clash(outs, 4, outs + 4, 1))) return SPEAR_E_ALIAS;
  if (c->pages == 0) return SPEAR_OK;  // every slot is outside
  KvAppendParams p;
  p.c = cache_of(c);
  p.r = {r.freqs, r.rotary_dim, r.interleaved, r.magnitude};
  p.T = (int)T, p.H = a->q ? a->heads : 0;
  p.q = (const uint16_t*)a->q, p.k = (const uint16_t*)a->k, p.v = (const uint16_t*)a->v;
  p.q_out = (uint16_t*)a->q_out;
  p.q_ld = ql, p.k_ld = kl, p.v_ld = vl, p.qo_ld = ol;
  p.slots = a->slots, p.positions = a->positions;
  p.log2_page = __builtin_ctz((unsigned)c->page_tokens);
  p.subs = subs, p.kv_blocks = (uint32_t)kv_blocks, p.q_blocks = (uint32_t)q_blocks;
  const auto launch = c->act_dtype == SPEAR_F16 ? launch_kv_append_f16 : launch_kv_append_bf16;
  return hip_status(launch(p, c->format, (hipStream_t)hip_stream));
}

spear_status_t spear_kv_read(const spear_kv_cache_t* c, int64_t n, const int32_t* slots, void* k_out, void* v_out,
                             void* hip_stream) {
  const spear_status_t st = check_cache(c);
  if (st != SPEAR_OK) return st;
  if (n < 0 || n >= ((int64_t)1 << 31) || !launches((n + 15) / 16 * c->kv_heads, 256)) return SPEAR_E_SHAPE;
  if (n == 0) return SPEAR_OK;
  if (!slots || !k_out || !v_out) return SPEAR_E_NULL;
  if (off4(slots) || off16(k_out) || off16(v_out)) return SPEAR_E_ALIGN;
  const size_t row = (size_t)n * c->kv_heads * c->head_dim * 2;
  const Span outs[] = {{k_out, row}, {v_out, row}};
  Span ins[5];
  cache_spans(c, reinterpret_cast<Span(&)[4]>(ins));
  ins[4] = {slots, (size_t)n * 4};
  if (clash(outs, 2, ins, 5)) return SPEAR_E_ALIAS;
  if (c->pages == 0) return SPEAR_OK;
  const KvReadParams p{cache_of(c), __builtin_ctz((unsigned)c->page_tokens), n, slots, (uint16_t*)k_out, (uint16_t*)v_out};
  const auto launch = c->act_dtype == SPEAR_F16 ? launch_kv_read_f16 : launch_kv_read_bf16;
  return hip_status(launch(p, c->format, (hipStream_t)hip_stream));
}

namespace {

spear_status_t check_attention(const spear_attention_t* a, bool buffers) {
  if (!a) return SPEAR_E_NULL;
  spear_status_t st = check_cache(a->cache, buffers);
  if (st == SPEAR_OK) st = check_batch(a->batch, buffers);
  if (st != SPEAR_OK) return st;
  if (a->heads < 1 || a->heads > 1024 || a->heads % a->cache->kv_heads || a->window < 0 ||
      (int64_t)a->batch->tokens * (a->heads / a->cache->kv_heads) >= (1 << 30) ||
      (int64_t)a->batch->tokens * a->heads >= (1 << 29))  // (with it any launch has fewer than 2^32 threads)
    return SPEAR_E_SHAPE;
  if (!buffers) return SPEAR_OK;
  if (!a->plan) return SPEAR_E_NULL;
  if (off16(a->plan) || off4(a->prefix)) return SPEAR_E_ALIGN;
  return SPEAR_OK;
}

// Rows, over all kv heads, from which on tiles are the large ones, which take half the
// time where there are enough of them. A prompt of 2048, 64 heads (131072 rows): 93 us in
// large tiles, 137 in small ones; of 1536 (98304): 76 and 84; a chunk of 1024 behind 8000
// tokens (65536): 414 and 418; a prompt of 1024, 32 heads (32768): 45 and 28.
constexpr int kFillRows = 98304;
// Stretches wanted of each kernel, over all kv heads, and a stretch's least steps.
// Few rows: of requests of unlike lengths one and a half a CU even out better than one (64
// requests of up to 8192 tokens: 35 us, 37 with one a CU, 37 with two), and heads of 64
// want more loads in flight (131000 tokens: 32 us, 35 with one); one request with heads of
// 128 is even by itself (131000 tokens: 57 us with one a CU, 65 with one and a half).
// Stretches of 8 steps, two turns of the waves: 13 requests 19 us, 25 in stretches of 16;
// 500 tokens 6.4, 7.8 in stretches of 4.
constexpr int kRowsGoal = 384, kRowsGoalOne = 256, kRowsLeast = 8;
// Small tiles: 13 requests 19 us, 21 at stretches of 8 steps or 256 stretches. Large ones
// have a CU each, and take all the same time between 4 and 8 steps.
constexpr int kMidGoal = 384, kMidLeast = 4, kTileGoal = 256, kTileLeast = 8;
// (stretches are shared out among kv heads only where there are fewer heads than the
// goal, so that counters are at most 2 (goal + heads))
static_assert(4 * kRowsGoal <= kAttnCounters && 4 * std::max(kTileGoal, kMidGoal) <= kAttnCounters, "a counter for each shared tile and head");

// Where the plan's and the workspace's parts lie, from sizes alone.
struct AttnLayout {
  AttnShape z;
  size_t items_rows, items_tile, plan_bytes;
  size_t parts_rows, parts_tile, work_bytes;
};
// the sizes that a plan and the calls it serves have in common, as one number
uint32_t plan_key(const spear_attention_t* a) {
  const spear_kv_cache_t* c = a->cache;
  const spear_kv_batch_t* b = a->batch;
  uint64_t h = 0xcbf29ce484222325ull;
  for (const int64_t v : {(int64_t)c->kv_heads, (int64_t)c->head_dim, (int64_t)c->page_tokens, (int64_t)b->requests, (int64_t)b->tokens,
                          (int64_t)b->max_new, (int64_t)b->width, (int64_t)a->heads, (int64_t)a->window,
                          (int64_t)(a->prefix != nullptr)})
    for (int i = 0; i < 32; i += 8) h = (h ^ ((v >> i) & 255)) * 0x100000001b3ull;
  return (uint32_t)(h ^ (h >> 32)) | 1u;
}
AttnLayout attention_layout(const spear_attention_t* a) {
  const spear_kv_cache_t* c = a->cache;
  const spear_kv_batch_t* b = a->batch;
  const int64_t hkv = c->kv_heads, group = a->heads / c->kv_heads, T = b->tokens, R = b->requests;
  const int64_t served = std::min(R, T);  // requests with a row
  const bool rows = group <= kRows, tile = (int64_t)b->max_new * group > kRows;
  AttnLayout l;
  AttnShape& z = l.z;
  z.goal_rows = (int)(((R == 1 && c->head_dim == 128 ? kRowsGoalOne : kRowsGoal) + hkv - 1) / hkv);
  // sum over tiles of max(1, ceil(steps / c)) with c >= all steps / goal
  z.max_rows = rows ? (int)R + z.goal_rows : 0;
  z.least_rows = kRowsLeast;
  const int big = tile_rows(c->head_dim);
  z.tile_rows = (T * group + big - 1) / big * hkv < kFillRows / big ? kMidRows : big;
  z.goal_tile = (int)(((z.tile_rows == kMidRows ? kMidGoal : kTileGoal) + hkv - 1) / hkv);
  z.least_tile = z.tile_rows == kMidRows ? kMidLeast : kTileLeast;
  z.max_tile = tile ? (int)(T * group / z.tile_rows + served) + z.goal_tile : 0;
  // and over those of more than one, ceil(steps / c) <= 2 steps / c
  z.part_rows = rows && z.goal_rows > 1 ? 2 * z.goal_rows : 0;
  z.part_tile = tile && z.goal_tile > 1 ? 2 * z.goal_tile : 0;
  l.items_rows = 0;
  l.items_tile = l.items_rows + (size_t)z.max_rows * sizeof(AttnItem);
  l.plan_bytes = std::max<size_t>(sizeof(AttnItem), l.items_tile + (size_t)z.max_tile * sizeof(AttnItem));
  // The counters have places of their own that every call of any sizes has in
  // common: another call's partial results never lie on them.
  l.parts_rows = 2 * kAttnCounters * sizeof(uint32_t);
  l.parts_tile = l.parts_rows + (size_t)z.part_rows * hkv * kRows * (c->head_dim + 2) * 4;
  l.work_bytes = (l.parts_tile + (size_t)z.part_tile * hkv * z.tile_rows * (c->head_dim + 2) * 4);
  return l;
}

}  // namespace

spear_status_t spear_attention_sizes(const spear_attention_t* a, size_t* plan_bytes, size_t* workspace_bytes) {
  if (!a || !plan_bytes || !workspace_bytes) return SPEAR_E_NULL;
  const spear_status_t st = check_attention(a, false);
  if (st != SPEAR_OK) return st;
  const AttnLayout l = attention_layout(a);
  *plan_bytes = l.plan_bytes;
  *workspace_bytes = l.work_bytes;
  return SPEAR_OK;
}

spear_status_t spear_attention_plan(const spear_attention_t* a, void* hip_stream) {
  const spear_status_t st = check_attention(a, true);
  if (st != SPEAR_OK) return st;
  const spear_kv_cache_t* c = a->cache;
  const spear_kv_batch_t* b = a->batch;
  const AttnLayout l = attention_layout(a);
  if (a->plan_bytes < l.plan_bytes) return SPEAR_E_WORKSPACE;
  const size_t R = b->requests;
  const Span outs[] = {{a->plan, l.plan_bytes}};
  const Span ins[] = {{b->starts, (R + 1) * 4}, {b->lens, R * 4}, {b->table, table_bytes(b)}, {a->prefix, R * 4}};
  if (clash(outs, 1, ins, 4)) return SPEAR_E_ALIAS;
  if (b->tokens == 0 || R == 0) return SPEAR_OK;
  AttnPlanParams p;
  p.R = b->requests, p.T = b->tokens, p.P = c->page_tokens, p.Hkv = c->kv_heads, p.group = a->heads / c->kv_heads;
  p.max_new = b->max_new, p.width = b->width, p.window = a->window ? std::min(a->window, kKvLength) : kKvLength;
  p.pages = (int)c->pages;
  p.key = plan_key(a);
  p.starts = b->starts, p.lens = b->lens, p.prefix = a->prefix;
  p.z = l.z;
  p.items_rows = (AttnItem*)((char*)a->plan + l.items_rows);
  p.items_tile = (AttnItem*)((char*)a->plan + l.items_tile);
  return hip_status(launch_attention_plan(p, (hipStream_t)hip_stream));
}

spear_status_t spear_attention(const spear_attention_t* a, void* hip_stream) {
  const spear_status_t st = check_attention(a, true);
  if (st != SPEAR_OK) return st;
  const spear_kv_cache_t* c = a->cache;
  const spear_kv_batch_t* b = a->batch;
  const int64_t T = b->tokens, row = (int64_t)a->heads * c->head_dim;
  const int64_t ql = a->q_ld ? a->q_ld : row, ol = a->out_ld ? a->out_ld : row;
  if (ql < row || ol < row || ql % 8 || ol % 8 || ql >= ((int64_t)1 << 30) || ol >= ((int64_t)1 << 30) ||
      !std::isfinite(a->scale) || !std::isfinite(a->softcap) || a->softcap < 0.f)
    return SPEAR_E_SHAPE;
  const AttnLayout l = attention_layout(a);
  if (a->plan_bytes < l.plan_bytes) return SPEAR_E_WORKSPACE;
  if (T == 0 || b->requests == 0) return SPEAR_OK;
  if (!a->q || !a->out) return SPEAR_E_NULL;
  if (off16(a->q) || off16(a->out) || off4(a->slopes) || off16(a->workspace)) return SPEAR_E_ALIGN;
  if (a->workspace_bytes < l.work_bytes || !a->workspace) return SPEAR_E_WORKSPACE;
  const size_t R = b->requests;
  const Span outs[] = {rows_of(a->out, T, ol, row), {a->workspace, l.work_bytes}};
  Span ins[11];
  cache_spans(c, reinterpret_cast<Span(&)[4]>(ins));
  ins[4] = {b->starts, (R + 1) * 4}, ins[5] = {b->lens, R * 4}, ins[6] = {b->table, table_bytes(b)};
  ins[7] = {a->prefix, R * 4}, ins[8] = {a->slopes, (size_t)a->heads * 4}, ins[9] = {a->plan, l.plan_bytes};
  ins[10] = rows_of(a->q, T, ql, row);
  if (clash(outs, 2, ins, 11)) return SPEAR_E_ALIAS;
  AttnParams p;
  p.c = cache_of(c);
  p.group = a->heads / c->kv_heads;
  p.window = a->window ? std::min(a->window, kKvLength) : kKvLength;
  p.key = plan_key(a);
  p.log2_page = __builtin_ctz((unsigned)c->page_tokens);
  p.ld = table_ld(b), p.q_ld = ql, p.out_ld = ol;
  p.table = b->table;
  p.q = (const uint16_t*)a->q, p.out = (uint16_t*)a->out;
  p.slopes = a->slopes, p.scale = a->scale, p.softcap = a->softcap;
  p.inv_cap = a->softcap > 0.f ? std::min(1.f / a->softcap, 3.40282347e38f) : 0.f;
  p.mid_blocks = (uint32_t)l.z.max_tile * c->kv_heads;
  p.items_rows = (const AttnItem*)((const char*)a->plan + l.items_rows);
  p.items_tile = (const AttnItem*)((const char*)a->plan + l.items_tile);
  p.counters_rows = (uint32_t*)a->workspace;
  p.counters_tile = p.counters_rows + kAttnCounters;
  p.parts_rows = (float*)((char*)a->workspace + l.parts_rows);
  p.parts_tile = (float*)((char*)a->workspace + l.parts_tile);
  const auto launch = c->act_dtype == SPEAR_F16 ? launch_attend_f16 : launch_attend_bf16;
  return hip_status(launch(p, l.z, c->format, (hipStream_t)hip_stream));
}
