// Rotation of a query row and back-rotation of an output row by one wavefront, in LDS.
#pragma once

#include "saw_prompt.h"

namespace saw {

// q R and o R^T of one row in LDS (128 floats; of 64 channels the first half)
// LOADS: of a learned rotation's rows at once, 8 where registers are short
template <int LOADS = 16>
__device__ __forceinline__ void rotate_row(const PromptParams& p, float* x, int D, int lane) {
  if (p.rot_k) {
    if (p.has_signs)
      for (int c = lane; c < D; c += 64) x[c] = apply_sign(p.signs, c, x[c]);
    wave_sync();
    wave_lds_fwht128<1>(x, p.had_block, lane);
    for (int c = lane; c < D; c += 64) x[c] *= had_norm(p.had_block);
    wave_sync();
  }
  if (p.dense_k) wave_lds_matvec128<1, LOADS>(x, p.dense, lane);
}
__device__ __forceinline__ void unrotate_row(const PromptParams& p, float* x, int D, int lane) {
  if (p.dense_v) wave_lds_matvec128<1>(x, p.dense + kDenseD * kDenseD, lane);
  if (p.rot_v) {
    wave_lds_fwht128<1>(x, p.had_block, lane);
    for (int c = lane; c < D; c += 64) x[c] = apply_sign(p.signs, c, x[c] * had_norm(p.had_block));
    wave_sync();
  }
}

}  // namespace saw
