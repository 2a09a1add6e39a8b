// Building blocks of the kernels whose queries come as packed rows of several tokens: row tiles, the search for a tile's sequence, and
// the products of a 64-key tile in shared memory.
//
// Row tiles.  Query token i and head g of a group are row i G + g of their (sequence, kv head): the heads of a group share every key they
// read, and a causal tile spans few tokens.  Sequence b owns the tiles from floor(cu[b] G / R) + b on: floor(x + y) >= floor(x) +
// floor(y) leaves room for ceil(n G / R) of them, so that a block finds its sequence by a search in cu and no table is built first.
#pragma once

#include "saw_prompt.h"

namespace saw {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// The last b of [0, n) with key(b) <= value, or -1, by a wavefront: 64 candidates a step.  key does not decrease; if it does (offsets that
// are none), some b of the range.
template <typename F>
__device__ __forceinline__ int last_not_above(int n, int64_t value, int lane, F key) {
  int lo = 0, span = n;
  bool first = true;
  while (span > 1 || first) {
    const int stride = (span + 63) / 64;
    const int b = lo + lane * stride;
    const uint64_t yes = __ballot(b < lo + span && key(b) <= value);
    const int k = __popcll(yes);
    if (first && k == 0) return -1;
    first = false;
    const int end = lo + span;
    lo += max(k - 1, 0) * stride;
    span = min(stride, end - lo);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int64_t clamped_offset(const int32_t* cu, int b, int64_t T) { return min((int64_t)max(cu[b], 0), T); }

struct RowTile {
  int b, begin, n;        // sequence, its first token and tokens
  int row0, rows;         // first row of the tile among the sequence's n G, rows of the tile
};
// false: the tile is nobody's
__device__ __forceinline__ bool find_row_tile(const PromptParams& p, int64_t tile, int R, int lane, RowTile& t) {
  const int64_t T = p.T_q;
  t.b = last_not_above(p.B, tile, lane, [&](int b) { return clamped_offset(p.cu_q, b, T) * p.group / R + b; });
  if (t.b < 0) return false;
  packed_range(p.cu_q, t.b, T, t.begin, t.n);
  const int64_t first = (int64_t)t.begin * p.group / R + t.b, row0 = (tile - first) * R, all = (int64_t)t.n * p.group;
  if (row0 < 0 || row0 >= all) return false;
  t.row0 = (int)row0;
  t.rows = (int)min((int64_t)R, all - row0);
  return true;
}
inline int64_t row_tiles(int64_t T, int G, int R, int B) { return T * G / R + B; }

// Operand types of the two products: bits of K / V, the matrix instruction, and the rounding of a pair of weights (nearest even).
//   kRaise: weights are relative to 2^(m - kRaise), m the row's maximum so far, up to 2^8 behind (tile_weights).  fp16 ones so go up to 2^15 and are
// off by half a step, 2^-11, down to 2^-21 of the largest weight; below by 2^-32 of the largest at most (relative to the maximum itself, by
// 2^-25: a strong token and 131072 others of 2^-25 of its weight each would lose their 0.4 % of the row).  bf16 has fp32's exponents.
struct MathBf16 {
  static constexpr float kRaise = 0.f;
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }
};
struct MathF16 {
  static constexpr float kRaise = 7.f;
  static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2)); }
};

constexpr int kTileKeys = 64;

// Ids of the four pages of a tile of 64 keys, fetched a tile ahead of the keys, which cannot be requested without them.  Pages behind the
// sequence's last are not looked at (the last again); ids out of range are page 0.  (A vector load whose lanes are read out at the use:
// scalar loads on their way make every wait for shared memory a wait for them as well, few rows 58 -> 70 us.)
struct TilePages {
  int ahead;
  __device__ __forceinline__ void fetch(const int32_t* pages, int tile, int len) { ahead = pages[min(4 * tile + (int)(threadIdx.x & 3), (len - 1) >> 4)]; }
  // (page, kv head) tiles of the pools, counted in 32 bits: 2^32 of them would be 2 TiB of codes and more
  uint32_t at[4];
  __device__ __forceinline__ void ready(const PromptParams& p, int h) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = __builtin_amdgcn_readlane(ahead, i);
      at[i] = (uint32_t)(id < 0 || id >= p.num_pages ? 0 : id) * (uint32_t)p.n_kv_heads + (uint32_t)h;
    }
  }
  __device__ __forceinline__ uint32_t tile_of(int key) const {              // of key `key` of the 64
    const uint32_t lo = key & 16 ? at[1] : at[0], hi = key & 16 ? at[3] : at[2];
    return key & 32 ? hi : lo;
  }
};
// A vector's codes and its (scale, zero) pair, in pools of 16 vectors a tile.
template <int D>
__device__ __forceinline__ const uint8_t* vector_codes(const uint8_t* codes, uint32_t tile, int key) {
  return codes + (uint64_t)tile * (8 * D) + (uint32_t)(key & 15) * (D / 2);
}
__device__ __forceinline__ const f32x2* vector_pair(const float* meta, uint32_t tile, int key) {
  return (const f32x2*)((const char*)meta + (uint64_t)tile * 128 + (uint32_t)(key & 15) * 8);
}

// codes - 8 of a word, in the order 0 4 1 5 2 6 3 7: 0x6400 + c is 1024 + c.  (The two constants in registers: with both as literals the
// masking is two instructions.)
struct CodeBits {
  uint32_t mask, one;
  __device__ __forceinline__ CodeBits() { asm("v_mov_b32 %0, 0xf000f\n\tv_mov_b32 %1, 0x64006400" : "=&v"(mask), "=v"(one)); }
};
__device__ __forceinline__ u32x4 centred(uint32_t w, CodeBits bits) {
  u32x4 r;
  const f16x2 off = {(_Float16)1032.f, (_Float16)1032.f};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, ((w >> (4 * i)) & bits.mask) | bits.one) - off);
  return r;
}

// A tile of 64 keys in shared memory: rows of D 16-bit values in 16-byte chunks, the chunks of a row exchanged so that whatever a
// read takes at once (256 bytes a clock) lies on different banks.  K: operand reads take one chunk of 16 rows.  V: transposing reads take 32
// bytes of four rows for each 16 lanes.  Rows of 64 channels stand two to 256 bytes.  (Exchanges that keep only 128 bytes a clock apart:
// half of the cycles of all LDS reads were conflicts, 8192 causal tokens 550 us.)
template <int D>
__device__ __forceinline__ int k_place(int row, int chunk) { return chunk ^ (D == 128 ? row & 15 : (row >> 1) & 7); }
template <int D>
__device__ __forceinline__ int v_place(int row, int chunk) {
  return chunk ^ (D == 128 ? 4 * (row & 3) + 2 * ((row >> 2) & 1) : 4 * ((row >> 1) & 1) + 2 * ((row >> 2) & 1));
}

// What a wavefront keeps of its 32 rows while it goes over the keys.  Products are taken transposed: S^T = K Q^T has a query per
// lane column and 16 of 32 keys in the lane's registers, so that maximum and sum of a row are lane-local up to the other half of the
// wavefront, and the weights are the B operand of O^T = V^T P^T as they stand - the keys of a k-step come in the order that S^T left
// them in (4 (lane / 32) + 0..3 and + 8), and the transposing reads of V follow it.
template <int D>
struct RowState {
  f32x16 o[D / 32];       // O^T: channel 32 t + 8 (r / 4) + 4 (lane / 32) + r % 4 of query lane % 32, relative to 2^ref
  float m, ref, sum;      // maximum that the state refers to (log2 units, -inf: none yet; ref: m - kRaise, 0 then); this half's sum of weights
};

// S^T of one tile against the queries in qf.  The two halves of the keys alternate, so that a product does not wait for the sum of the one
// before it, and operands are read six products ahead (left to itself the compiler waits for each: 8192 causal tokens 530 us instead of 522).
template <int D, typename M1>
__device__ __forceinline__ void tile_logits(const char* k, const u32x4 (&qf)[D / 16], f32x16 (&s)[2], int lane) {
  constexpr int kAhead = 6, kAll = 2 * (D / 16);
  const int row = lane & 31;
  const char* const at = k + row * (2 * D);
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const u32x4 a = *(const u32x4*)(at + kb * 32 * (2 * D) + 16 * k_place<D>(row, 2 * ks + (lane >> 5)));
      s[kb] = M1::mfma(a, qf[ks], s[kb]);
    }
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
  for (int i = 0; i < kAll - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
  __builtin_amdgcn_sched_barrier(0);
}

// Keys that a lane's query does not see get -infinity; `left`: keys of the tile that it sees.
__device__ __forceinline__ void tile_mask(f32x16 (&s)[2], int left, int lane) {
  const int mine = left - 4 * (lane >> 5);
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[kb][r] = 32 * kb + 8 * (r >> 2) + (r & 3) < mine ? s[kb][r] : -INFINITY;
}

// Logits become weights relative to the state's reference, which moves only when a row's maximum has grown by more than 2^8 since: the
// sums keep 24 bits whatever they are relative to, and the rescaling of all of O is left out for most tiles.
template <int D, typename M2>
__device__ __forceinline__ void tile_weights(f32x16 (&s)[2], float scale, RowState<D>& st, u32x4 (&pf)[4]) {
  float top = s[0][0];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
  top = max_xor32(top) * scale;
  if (__any(top > st.m + 8.f)) {
    const float m = fmaxf(st.m, top);
    const float alpha = fast_exp2(st.m - (m == -INFINITY ? 0.f : m));
    st.m = m;
    st.ref = m == -INFINITY ? 0.f : m - M2::kRaise;
    st.sum *= alpha;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[t][r] *= alpha;
  }
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[kb][r] = fast_exp2(fmaf(s[kb][r], scale, -st.ref));
      sum[r & 3] += s[kb][r];
    }
#pragma unroll
    for (int r = 0; r < 16; r += 2) pf[2 * kb + (r >> 3)][(r & 7) >> 1] = M2::pack(s[kb][r], s[kb][r + 1]);
  }
  st.sum += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// O^T += V^T P^T
template <int D, typename M2>
__device__ __forceinline__ void tile_values(const char* v, const u32x4 (&pf)[4], RowState<D>& st, int lane) {
  const int i = lane & 15, key = 4 * (lane >> 5) + (i >> 2);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
      const int chunk = 4 * t + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
      const char* const at = v + (16 * ks + key) * (2 * D) + 16 * v_place<D>(key, chunk) + 8 * (i & 1);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(at + 8 * (2 * D)));
      const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
      st.o[t] = M2::mfma((u32x4{l2.x, l2.y, h2.x, h2.y}), pf[ks], st.o[t]);
    }
  }
}

}  // namespace saw
