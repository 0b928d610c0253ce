// The paged 8-bit cache on the device: places inside a page, and what its kernels share.
#pragma once

#include "oscar_common.h"

// A step is 32 tokens of a kv head, 4 KB of key codes and 4 KB of value codes: the depth of one matrix
// instruction for values, two operand tiles for keys.  Lane l = 16 * q4 + n of a wave loads 16 bytes at 16 * l
// of each kilobyte, and has then
//   keys   kilobyte 2 * tile + half: token 16 * tile + n, channels 64 * half + 16 * q4 + 0 .. 15
//   values kilobyte pair            : tokens 16 * t2 + 4 * q4 + i of channels 32 * pair + 16 * c2 + n, at byte
//                                     8 * c2 + 4 * t2 + i
// i.e. an operand of 16 x 32 keys, and one of 16 x 32 values whose depth runs over tokens in the order in
// which the logits of the step come out of the matrix cores: probabilities go from results to operands without
// leaving their lane.
constexpr int Q8_STEP_TOKENS = 32;
constexpr int Q8_STEP_BYTES = Q8_STEP_TOKENS * OSCAR_D;
constexpr int Q8_PAGE_BYTES = OSCAR_R * OSCAR_D;
constexpr int Q8_PAGE_STEPS = OSCAR_R / Q8_STEP_TOKENS;

struct Q8Cache {
  int batch, max_pages, num_pages, heads, block;
  uint8_t *k_codes, *v_codes;
  float *k_scales, *v_scales;
  uint16_t *win_k, *win_v;
  const int32_t* table;
};

inline Q8Cache q8_device_view(const oscar_q8_cache* c) {
  return {c->batch, c->max_pages_per_seq, c->num_pages, c->n_kv_heads, c->block, reinterpret_cast<uint8_t*>(c->k_codes),
          reinterpret_cast<uint8_t*>(c->v_codes), c->k_scales, c->v_scales, reinterpret_cast<uint16_t*>(c->win_k),
          reinterpret_cast<uint16_t*>(c->win_v), c->block_table};
}

// The rows of a step: which belong to sequence b, and where its tokens stand.
struct Q8Rows {
  const int32_t *row_starts, *new_lens, *lens;
  int T;
  int64_t n_rows;
};
struct Q8Seq {
  int n, len, old;   // new tokens, all tokens, tokens before the step (below 0 where a caller's lengths do not fit)
  int64_t row;       // of the first new token
};
__device__ __forceinline__ Q8Seq q8_seq(const Q8Rows& r, int b) {
  Q8Seq s;
  s.n = r.new_lens ? min(max(r.new_lens[b], 0), r.T) : r.T;
  s.len = min(max(r.lens[b], 0), INT32_MAX - 4096);   // (a step or two past it is still a number)
  s.old = s.len - s.n;
  s.row = r.row_starts ? r.row_starts[b] : (int64_t)b * r.T;
  return s;
}

// The page of a sequence's token, or -1.
__device__ __forceinline__ int q8_page(const Q8Cache& c, int b, int page) {
  if (page >= c.max_pages) return -1;
  const int p = c.table[(int64_t)b * c.max_pages + page];
  return (uint32_t)p < (uint32_t)c.num_pages ? p : -1;
}

// The checks of a cache and of the rows of a step that the entry points share.
int oscar_check_q8_sizes(const oscar_q8_cache* c);
int oscar_check_q8_cache(const oscar_q8_cache* c);
