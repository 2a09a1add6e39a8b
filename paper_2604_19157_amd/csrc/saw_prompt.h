// Argument block and host plans shared by the kernels of packed queries: prompt attention (saw_prompt.hip) and accumulated attention
// weights (saw_weights.hip).
#pragma once

#include "saw_wave_util.h"

namespace saw {

struct PromptParams {
  // queries and outputs: packed rows, sequence b has tokens [cu_q[b], cu_q[b + 1])
  const void* q;
  void* out;                  // [T_q][n_q_heads][D] of the queries' type
  int64_t q_stride, T_q;
  const int32_t* cu_q;
  int32_t B, n_q_heads, n_kv_heads, group, dtype;
  float scale;                // sm_scale * log2(e)
  int32_t causal;
  // keys and values of 16 bits, packed
  const void *k, *v;
  int64_t k_stride, v_stride, T_k;
  const int32_t* cu_k;
  // ... or INT4 pages
  const uint8_t *k_codes, *v_codes;
  const float *k_meta, *v_meta;
  const int32_t *page_table, *seq_lens;
  int32_t max_pages, num_pages, bound;
  int32_t had_block, rot_k, rot_v, dense_k, dense_v, has_signs;
  const float* dense;         // learned rotation, fp32 [128][128], its transpose right behind it; null: none
  SignBits signs;
  // accumulated weights
  const float* prev;
  float* scores;
  int64_t score_stride;
  float* ws;
  uint16_t* query;            // rotated queries in the workspace, fp16, and what each row was divided by
  float* query_scale;
};

// Tokens of sequence b, whatever the offsets hold: inside [0, T] and not reversed.
__device__ __forceinline__ void packed_range(const int32_t* cu, int b, int64_t T, int& begin, int& n) {
  const int64_t lo = min((int64_t)max(cu[b], 0), T), hi = min((int64_t)max(cu[b + 1], 0), T);
  begin = (int)lo;
  n = (int)max(hi - lo, (int64_t)0);
}

}  // namespace saw
