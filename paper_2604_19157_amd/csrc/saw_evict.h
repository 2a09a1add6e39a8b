// Argument block of the eviction kernels.
#pragma once

#include "saw_wave_util.h"

namespace saw {

struct EvictParams {
  uint8_t* codes[2];          // K, V
  float* meta[2];
  const float* scores;        // [B][n_kv_heads][score_stride]
  int64_t score_stride, score_out_stride;
  const int32_t *page_table, *seq_lens, *dst_table;
  int32_t max_pages, dst_pages, num_pages, n_kv_heads, bound, budget, recent;
  int32_t *new_lens, *kept;
  float* scores_out;          // or null
};

}  // namespace saw
