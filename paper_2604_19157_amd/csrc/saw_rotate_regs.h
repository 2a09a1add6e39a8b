// Block Hadamard transforms of rows that stand across the registers of two half-wavefronts, 64 (32) values of 128 (64) channels a lane:
// the layouts of a query as B operand and of an output as accumulators.  A stage between registers is one addition a value; the stage
// between the halves a register exchange more.
#pragma once

#include "saw_prompt_tile.h"

namespace saw {

// One stage in a lane's own values: pairs (i, i + st)
template <int N>
__device__ __forceinline__ void fwht_own(float (&x)[N], int st) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (!(i & st)) { const float a = x[i], b = x[i + st]; x[i] = a + b; x[i + st] = a - b; }
}
// ... and between the two halves of the wavefront
template <int N>
__device__ __forceinline__ void fwht_halves(float (&x)[N], int lane) {
  const float side = lane < 32 ? 1.f : -1.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float lo, hi;
    swap32(x[i], x[i], lo, hi);
    x[i] = fmaf(side, hi, lo);
  }
}
// Channel of value i in half h: bits of i with the half's bit put in at HALF_BIT.
template <int HALF_BIT>
__host__ __device__ constexpr int spread_channel(int i) { return (i & ((1 << HALF_BIT) - 1)) | (i >> HALF_BIT) << (HALF_BIT + 1); }

// Un-normalised transform in blocks of `block` channels
template <int D, int HALF_BIT>
__device__ __forceinline__ void fwht_rows(float (&x)[D / 2], int block, int lane) {
#pragma unroll
  for (int bit = 0; (1 << bit) < D; ++bit)
    if ((1 << bit) < block) {                                            // (uniform)
      if (bit == HALF_BIT) fwht_halves(x, lane);
      else fwht_own(x, bit < HALF_BIT ? 1 << bit : 1 << (bit - 1));
    }
}
template <int D, int HALF_BIT>
__device__ __forceinline__ void sign_rows(float (&x)[D / 2], const SignBits& signs, int lane) {
#pragma unroll
  for (int i = 0; i < D / 2; ++i) {
    const int c = spread_channel<HALF_BIT>(i);                           // of half 0
    const uint32_t mine = lane < 32 ? signs.w[c >> 5] >> (c & 31) : signs.w[(c | 1 << HALF_BIT) >> 5] >> ((c | 1 << HALF_BIT) & 31);
    x[i] = __uint_as_float(__float_as_uint(x[i]) ^ (mine << 31));
  }
}

}  // namespace saw
