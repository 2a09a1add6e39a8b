// Rotation of a query row and back-rotation of an output row by one wavefront, in LDS.
#pragma once

#include "saw_prompt.h"

namespace saw {

// q R and o R^T of NV rows in LDS (128 floats each; of 64 channels the first half).  A learned rotation's 64 KiB are read once for all of them.
// LOADS: of its rows at once, 8 where registers are short
template <int LOADS = 16, int NV = 1>
__device__ __forceinline__ void rotate_row(const PromptParams& p, float* x, int D, int lane) {
  if (p.rot_k) {
    if (p.has_signs)
      for (int v = 0; v < NV; ++v)
        for (int c = lane; c < D; c += 64) x[128 * v + c] = apply_sign(p.signs, c, x[128 * v + c]);
    wave_sync();
    wave_lds_fwht128<NV>(x, p.had_block, lane);
    for (int v = 0; v < NV; ++v)
      for (int c = lane; c < D; c += 64) x[128 * v + c] *= had_norm(p.had_block);
    wave_sync();
  }
  if (p.dense_k) wave_lds_matvec128<NV, LOADS>(x, p.dense, lane);
}
template <int LOADS = 16, int NV = 1>
__device__ __forceinline__ void unrotate_row(const PromptParams& p, float* x, int D, int lane) {
  if (p.dense_v) wave_lds_matvec128<NV, LOADS>(x, p.dense + kDenseD * kDenseD, lane);
  if (p.rot_v) {
    wave_lds_fwht128<NV>(x, p.had_block, lane);
    for (int v = 0; v < NV; ++v)
      for (int c = lane; c < D; c += 64) x[128 * v + c] = apply_sign(p.signs, c, x[128 * v + c] * had_norm(p.had_block));
    wave_sync();
  }
}

}  // namespace saw
