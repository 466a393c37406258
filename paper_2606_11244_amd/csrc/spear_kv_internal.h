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
  int window;        // run starts a workgroup of the cache's part looks for
  int q_tokens;      // tokens a workgroup of the queries' part takes
  uint32_t kv_blocks, q_blocks;
};

struct KvReadParams {
  KvCache c;
  int64_t n;
  const int32_t* slots;
  uint16_t *k_out, *v_out;
};

struct KvAttendParams {
  KvCache c;
  int R, T, H, group, max_new, width, window_tokens;  // window_tokens: kKvLength: none
  int64_t ld, q_ld, out_ld;
  const int32_t *starts, *lens, *table, *prefix;
  const uint16_t* q;
  uint16_t* out;
  const float* slopes;
  float scale, softcap;
};

hipError_t launch_kv_pages(const KvPagesParams& p, hipStream_t st);
#define SPEAR_KV_LAUNCHERS(D)                                                      \
  hipError_t launch_kv_append_##D(const KvAppendParams& p, int format, hipStream_t st); \
  hipError_t launch_kv_read_##D(const KvReadParams& p, int format, hipStream_t st); \
  hipError_t launch_kv_attend_##D(const KvAttendParams& p, int format, hipStream_t st);
SPEAR_KV_LAUNCHERS(f16)
SPEAR_KV_LAUNCHERS(bf16)
#undef SPEAR_KV_LAUNCHERS

}  // namespace spear
