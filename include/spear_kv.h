/*
 * spear_kv.h -- C ABI of attention over a cache held in 8 bits, for the MI355X
 * (gfx950): what stands between a block's q, k, v projections and its output
 * projection (spear.h) when requests of unlike lengths are served together.
 *
 * A step of a serving program, every layer of it on the same batch:
 *
 *     spear_kv_pages         block tables, slots and positions of the new tokens
 *     spear_attention_plan   the attention's share of work, once for all layers
 *     spear_kv_append        rotary positions; keys and values into the cache
 *     spear_attention        the new tokens' queries over the cache
 *
 * all on the GPU from lengths that live there, so that one captured graph serves
 * steps whose lengths differ. The conventions of spear.h hold (device pointers
 * aligned to 16 bytes, host validation before any launch, caller-owned buffers,
 * calls ordered on `hip_stream`); int32 arrays of lengths, tables and slots need
 * 4 bytes only.
 *
 * The cache is a pool of pages of `page_tokens` tokens. A page holds K as
 * [kv_heads][page_tokens][head_dim] and V as [kv_heads][head_dim][page_tokens]
 * codes of 8 bits, with one fp32 scale a head for each; a code c stands for
 * c * scale. Scales are powers of two (as spear_kv_append writes them), from
 * 2^-100 on. A slot is page * page_tokens + place in the page.
 */
#ifndef SPEAR_KV_H
#define SPEAR_KV_H

#include "spear.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
  SPEAR_KV_INT8 = 0, /* two's complement, -127..127                             */
  SPEAR_KV_E4M3 = 1  /* OCP 8-bit floats of 4 exponent bits, -448..448          */
};

typedef struct {
  int32_t format;      /* SPEAR_KV_INT8 or SPEAR_KV_E4M3                        */
  int32_t act_dtype;   /* SPEAR_F16 or SPEAR_BF16: queries, keys, values, output */
  int32_t kv_heads;    /* 1..1024                                               */
  int32_t head_dim;    /* 64 or 128                                             */
  int32_t page_tokens; /* 16, 32, 64 or 128                                     */
  int32_t reserved;    /* 0                                                     */
  int64_t pages;       /* >= 0; pages * page_tokens < 2^31                      */
  void* k;             /* [pages][kv_heads][page_tokens][head_dim]              */
  void* v;             /* [pages][kv_heads][head_dim][page_tokens]              */
  float* k_scale;      /* [pages][kv_heads]                                     */
  float* v_scale;      /* [pages][kv_heads]                                     */
} spear_kv_cache_t;

/* The requests of a step. Request r has the rows starts[r]..starts[r+1]-1 of the
 * step's tokens, which are its newest, and lens[r] tokens in the cache, these
 * included; its tokens j stand in page table[r * table_ld + j / page_tokens]. */
typedef struct {
  int32_t requests;  /* 0..4096                                                 */
  int32_t tokens;    /* rows of the step, padding behind the last request too:
                        0..2^22                                                 */
  int32_t max_new;   /* 1..tokens: no request has more new tokens (of one that
                        has, attention computes the first max_new rows only)    */
  int32_t width;     /* entries of a table row: 1..2^26                         */
  int32_t table_ld;  /* entries between rows: >= width; 0 = width               */
  int32_t reserved;  /* 0                                                       */
  int32_t* starts;   /* [requests + 1], ascending, within 0..tokens             */
  int32_t* lens;     /* [requests]; a request whose lens is less than its rows
                        (0: not served) has zeros for the rows without a key    */
  int32_t* table;    /* [requests][width]; ids outside the cache's pages are
                        taken as tokens that no row sees                        */
} spear_kv_batch_t;

/* Block tables and slot maps from lengths, in one launch. Request r has held[r]
 * tokens in the cache, whose pages its table row names, and gets fresh[r] new
 * ones. Pages that these need beyond the row's are taken from free_pages in
 * request order and entered in the row. Written: the batch's starts (of all
 * requests, cut at `tokens`) and lens (held + fresh), for each row of the step
 * its slot and position (-1 and 0 for padding), and taken[0], how many free pages
 * were taken, taken[1], how many requests were not served. Not served is a
 * request with a negative length or of 2^30 tokens or more, whose rows pass
 * `tokens`, whose tokens pass its table row, or whose pages pass the free ones
 * (once they do, no later request gets any): its lens is 0, its slots are -1, its
 * positions 0, its table row is as it was. A token whose table entry is negative
 * or of a slot past 2^31 has slot -1. */
typedef struct {
  int32_t page_tokens;        /* 16, 32, 64 or 128                              */
  int32_t n_free;             /* >= 0                                           */
  const int32_t* held;        /* [requests]                                     */
  const int32_t* fresh;       /* [requests]                                     */
  const int32_t* free_pages;  /* [n_free]                                       */
  int32_t* slots;             /* [tokens]                                       */
  int32_t* positions;         /* [tokens]                                       */
  int32_t* taken;             /* [2]                                            */
} spear_kv_pages_t;

/* SPEAR_E_NULL for a missing pointer whose array is not empty; SPEAR_E_SHAPE for
 * sizes outside the above; SPEAR_E_ALIGN for an array off 4 bytes; SPEAR_E_ALIAS
 * where an output overlaps another array. */
spear_status_t spear_kv_pages(const spear_kv_batch_t* batch, const spear_kv_pages_t* args,
                              void* hip_stream);

/* Rotary positions. Feature pair i of the first rotary_dim features of a head (of
 * features i and i + rotary_dim/2, or 2i and 2i + 1 if interleaved) is turned at
 * position p by p * freqs[i] of 2^64, the whole being one turn: the product modulo
 * one turn is exact at every position. Its length is multiplied by magnitude. The
 * other features pass unchanged. */
typedef struct {
  int32_t rotary_dim;    /* even, 0..head_dim; 0: no rotation                   */
  int32_t interleaved;   /* 0 or 1                                              */
  float magnitude;       /* finite                                              */
  int32_t reserved;      /* 0                                                   */
  const uint64_t* freqs; /* [rotary_dim / 2], aligned to 8                      */
} spear_rope_t;

/* Host-only: fills freqs (host memory) for rotary_dim features of base `base`:
 * f_i = base^(-2i/rotary_dim) radians a position, and for contexts longer than the
 * `context` positions a model was trained on f_i (s + (1 - s) / factor), where s
 * falls from 1 to 0 as the turns f_i makes in `context` positions go from
 * high_turns to low_turns (linearly in the turns). factor 1: f_i itself; context
 * 0: every f_i / factor. SPEAR_E_NULL, or SPEAR_E_SHAPE for an odd or negative
 * rotary_dim, base <= 1, factor < 1, a negative context, or high_turns <=
 * low_turns where they are read. */
spear_status_t spear_rope_frequencies(int32_t rotary_dim, double base, double factor, double context,
                                      double low_turns, double high_turns, uint64_t* freqs);

/* New tokens into the cache, one launch: k is turned and written, v written, each
 * token at its slot, and q (unless NULL) turned into q_out. q is turned in fp32 and
 * rounded once; a code of k is the nearest to the rotation in 64 bits. The scale of a
 * page and head is the least power of two whose multiple by 127 (INT8) or 448 (E4M3)
 * reaches every magnitude (in fp32) it has been given since its first place was
 * written; it never shrinks before, and where it
 * grows the codes already there are divided to match (rounded to nearest even:
 * E4M3 codes keep their value down to the format's least steps, INT8 codes are off
 * by less than one step in all). Codes are rounded to nearest even and no code
 * stands for a value past the activation type's largest. Infinities become the
 * largest code and NaN zero; neither counts for the scale.
 *
 * Tokens of one page have to follow each other, with slots ascending by one (as
 * spear_kv_pages gives them): the first of them tells how much of the page is
 * filled, and a page whose tokens come otherwise holds unspecified codes. Tokens
 * whose slot is outside the cache are skipped, q included. Codes behind the last
 * written place are left as they were. */
typedef struct {
  int32_t tokens;           /* 0..2^22                                          */
  int32_t heads;            /* query heads; read with q: 1..1024                */
  const void* q;            /* [tokens][heads][head_dim]; NULL: none            */
  const void* k;            /* [tokens][kv_heads][head_dim]                     */
  const void* v;            /* [tokens][kv_heads][head_dim]                     */
  void* q_out;              /* [tokens][heads][head_dim]; may be q, same rows   */
  int64_t q_ld, k_ld, v_ld, q_out_ld; /* elements between tokens: at least
                               their heads' features and a multiple of 8; 0 =
                               dense                                            */
  const int32_t* slots;     /* [tokens]                                         */
  const int32_t* positions; /* [tokens]; read with a rotation                   */
  spear_rope_t rope;
} spear_kv_append_t;

/* SPEAR_E_NULL for a missing pointer; SPEAR_E_DTYPE for an unknown format or act
 * dtype; SPEAR_E_SHAPE for sizes or strides outside the above, or more heads and
 * tokens than one launch takes (2^24 workgroups: one a token with q, and kv_heads / 8
 * a token); SPEAR_E_ALIGN; SPEAR_E_ALIAS where q_out overlaps an input (unless it is q with the same row
 * stride) or a buffer of the cache overlaps any other. */
spear_status_t spear_kv_append(const spear_kv_cache_t* cache, const spear_kv_append_t* args,
                               void* hip_stream);

/* What cached tokens stand for: k_out[i], v_out[i] [kv_heads][head_dim] in the act
 * dtype of the token at slots[i], rows of slots outside the cache left as they
 * were. n in 0..2^31-1, n * kv_heads below 2^28. Errors as for spear_kv_append. */
spear_status_t spear_kv_read(const spear_kv_cache_t* cache, int64_t n, const int32_t* slots, void* k_out,
                             void* v_out, void* hip_stream);

/* Attention of a step's rows over the cache. Row i of a request stands at position
 * lens - rows + i; with p its position, head h of it reads kv head h / (heads /
 * kv_heads), and
 *
 *     s_j = scale q . k_j,  or  softcap tanh(scale q . k_j / softcap)
 *     s_j = s_j - slopes[h] |p - j|
 *     out = sum_j e^s_j v_j / sum_j e^s_j   over the tokens j that the row sees:
 *           j <= p and p - j < window (0: any), or j < prefix[r]; j < lens[r]
 *
 * and zeros for a row that sees none. q.k, the softmax and the sums over j are
 * held in fp32; the weights e^(s_j - max) are rounded to the act dtype (in fp16 small
 * ones to 2^-28 of the largest) for their product with v (whose values it holds
 * exactly, in fp16 to 2^-25) and, of requests of more than 16 rows a kv head, in their
 * sum; out is rounded once. In bf16 the sums over j may leave fp32's range where a
 * value times the request's tokens passes 2^115.
 * Rows behind the last request are left as they were. Codes and scales of tokens that
 * no row of a request sees may hold anything; those seen are finite. */
typedef struct {
  const spear_kv_cache_t* cache;
  const spear_kv_batch_t* batch;
  int32_t heads;         /* a multiple of kv_heads, 1..1024; tokens * heads /
                            kv_heads < 2^30, tokens * heads < 2^29              */
  int32_t window;        /* >= 0; 0: none                                       */
  const int32_t* prefix; /* [requests]; NULL: none                              */
  void* plan;            /* spear_attention_sizes' plan_bytes                   */
  size_t plan_bytes;
  const void* q;         /* [tokens][heads][head_dim]                           */
  void* out;             /* [tokens][heads][head_dim]                           */
  int64_t q_ld, out_ld;  /* elements between tokens: at least heads * head_dim
                            and a multiple of 8; 0 = dense                      */
  const float* slopes;   /* [heads], finite; NULL: none                         */
  float scale;           /* finite                                              */
  float softcap;         /* finite, >= 0; 0: none                               */
  void* workspace;       /* zero-filled once before its first use               */
  size_t workspace_bytes;
} spear_attention_t;

/* Bytes of the plan and of the workspace, from the cache's, the batch's and the
 * heads' sizes alone (host-only; no pointer but cache and batch is read). */
spear_status_t spear_attention_sizes(const spear_attention_t* args, size_t* plan_bytes,
                                     size_t* workspace_bytes);

/* Writes the plan: which rows and stretches of the cache go to which workgroup,
 * from starts, lens, window and prefix. It serves every spear_attention whose
 * cache, batch, heads, window and prefix are the same in size and content (the
 * layers of a step), until one of them changes. Where sizes differ the attention
 * writes nothing. With starts that descend or lie outside 0..tokens the step's rows
 * of `out` hold unspecified values or what they held; nothing else is touched, and a
 * later call is as any other. Errors as for spear_attention; q, out and the workspace
 * are not looked at. */
spear_status_t spear_attention_plan(const spear_attention_t* args, void* hip_stream);

/* Errors: SPEAR_E_NULL, SPEAR_E_DTYPE, SPEAR_E_SHAPE, SPEAR_E_ALIGN; SPEAR_E_WORKSPACE
 * for a plan or workspace smaller than needed; SPEAR_E_ALIAS where out overlaps
 * another buffer. The workspace may be shared with other calls of this function in
 * stream order; calls that overlap in time need one each. */
spear_status_t spear_attention(const spear_attention_t* args, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SPEAR_KV_H */
