// Parameters and launchers of the cache's kernels (spear_kv.hip) and of the
// attention over it (spear_attn.hip); the host side is spear_kv_api.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spear {

enum { KV_INT8 = 0, KV_E4M3 = 1 };
constexpr int kKvRequests = 4096;     // most requests of a step
constexpr int kKvTokens = 1 << 22;    // most rows of a step
constexpr int kKvLength = 1 << 30;    // a request's tokens stay below

// the cache, as the kernels see it (head_dim is a template argument or D)
struct KvCache {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int Hkv, D, P, pages;
};

struct KvPagesParams {
  int R, T, P, width, n_free;
  int64_t ld;
  const int32_t *held, *fresh, *free_pages;
  int32_t *starts, *lens, *table, *slots, *positions, *taken;
};

struct KvRope {
  const uint64_t* freqs;
  int rot, interleaved;
  float magnitude;
};

struct KvAppendParams {
  KvCache c;
  KvRope r;
  int T, H;  // H 0: no queries
  const uint16_t *q, *k, *v;
  uint16_t* q_out;
  int64_t q_ld, k_ld, v_ld, qo_ld;
  const int32_t *slots, *positions;
  int log2_page;
  int subs;  // workgroups that share the runs of a window of 64 tokens
  uint32_t kv_blocks, q_blocks;
};

struct KvReadParams {
  KvCache c;
  int log2_page;
  int64_t n;
  const int32_t* slots;
  uint16_t *k_out, *v_out;
};

// ---- attention ----
// A request's rows (its new tokens, each with the query heads of one kv head) go
// to attend_rows where they are at most kRows, else, in tiles, to attend_mid
// (kMidRows) or k_attend_tile (tile_rows). All walk the cache in steps of kStep tokens.
constexpr int kRows = 16, kMidRows = 32, kStep = 64;
constexpr int tile_rows(int head_dim) { return head_dim == 128 ? 256 : 128; }
constexpr int kAttnCounters = 2048;  // of each kernel

// one workgroup's share (of each kv head): some rows over some steps
struct AttnItem {
  uint32_t key;                   // of the sizes the plan was made for (0: none); a call of others does nothing
  int32_t r, row0, rows, pos0;    // request, its first row of the step, its rows, position of the first
  int32_t tile, s0, s1, splits;   // tile of its rows; steps; stretches the tile's steps are cut into
  int32_t split, part, first, end;  // which; the first one's place among the partial results (splits > 1);
                                  // tokens some row sees: first..end-1 and 0..prefix-1
  int32_t prefix, pad[2];
};

// sizes that the host fixes from the batch's and the heads' sizes alone
struct AttnShape {
  int tile_rows;               // kMidRows or tile_rows(head_dim)
  int goal_rows, goal_tile;    // stretches wanted: enough workgroups to fill the GPU
  int least_rows, least_tile;  // least steps of a stretch
  int max_rows, max_tile;      // items there can be
  int part_rows, part_tile;    // partial results there can be, a kv head
};

struct AttnPlanParams {
  int R, T, P, Hkv, group, max_new, width, window, pages;
  uint32_t key;
  const int32_t *starts, *lens, *prefix;
  AttnShape z;
  AttnItem *items_rows, *items_tile;
};

struct AttnParams {
  KvCache c;
  int group, window, log2_page;  // window: kKvLength for none
  uint32_t key;
  int64_t ld, q_ld, out_ld;
  const int32_t* table;
  const AttnItem *items_rows, *items_tile;
  const uint16_t* q;
  uint16_t* out;
  const float* slopes;
  float scale, softcap, inv_cap;  // inv_cap: 1 / softcap, finite
  uint32_t *counters_rows, *counters_tile;  // [part][Hkv]: kAttnCounters each
  float *parts_rows, *parts_tile;  // [part][Hkv][rows of O, their maxima, their sums]
  uint32_t mid_blocks;             // workgroups of k_attend_mid that take tiles
};

hipError_t launch_attention_plan(const AttnPlanParams& p, hipStream_t st);
hipError_t launch_kv_pages(const KvPagesParams& p, hipStream_t st);
#define SPEAR_KV_LAUNCHERS(D)                                                      \
  hipError_t launch_kv_append_##D(const KvAppendParams& p, int format, hipStream_t st); \
  hipError_t launch_kv_read_##D(const KvReadParams& p, int format, hipStream_t st); \
  hipError_t launch_attend_##D(const AttnParams& p, const AttnShape& z, int format, hipStream_t st);
SPEAR_KV_LAUNCHERS(f16)
SPEAR_KV_LAUNCHERS(bf16)
#undef SPEAR_KV_LAUNCHERS

}  // namespace spear
