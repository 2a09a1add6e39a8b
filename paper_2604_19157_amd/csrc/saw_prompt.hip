// Attention of packed queries: softmax(q K^T s) V with K and V of 16 bits or read from the INT4 pages.
#include <type_traits>

#include "saw_prompt_tile.h"
#include "saw_rotate_regs.h"
#include "saw_rotate_row.h"

namespace saw {

// kKvCodes: the INT4 pages, keys as exact codes and their scales on the logits.
enum { kKvBf16, kKvF16, kKvInt4, kKvCodes };
constexpr bool int4_pages(int kv) { return kv >= kKvInt4; }

// Channels of one vector that a lane holds: lane, lane + 64.  page: of position j, INT4 (eight positions from a multiple of eight on share theirs).
template <int D, int KV>
struct RowSource {
  const PromptParams& p;
  int b, h, k0, lane;
  __device__ int page_of(int j) const {
    if constexpr (!int4_pages(KV)) return 0;
    const int page = p.page_table[(int64_t)b * p.max_pages + (j >> 4)];
    return page < 0 || page >= p.num_pages ? 0 : page;
  }
  __device__ f32x2 value_pair_of(int page, int j) const { return *(const f32x2*)(p.v_meta + 2 * (((int64_t)page * p.n_kv_heads + h) * 16 + (j & 15))); }
  __device__ void load(bool value, int page, int j, float (&x)[D / 64]) const {
    if constexpr (int4_pages(KV)) {
      const int64_t vec = ((int64_t)page * p.n_kv_heads + h) * 16 + (j & 15);
      const float* const m = (value ? p.v_meta : p.k_meta) + 2 * vec;
      const uint8_t* const c = (value ? p.v_codes : p.k_codes) + vec * (D / 2);
#pragma unroll
      for (int e = 0; e < D / 64; ++e) {
        const int ch = lane + 64 * e;
        x[e] = m[0] * ((float)((c[ch >> 1] >> (4 * (ch & 1))) & 15) - m[1]);
      }
    } else {
      const uint16_t* const src = (const uint16_t*)(value ? p.v : p.k) + (int64_t)(k0 + j) * (value ? p.v_stride : p.k_stride) + (int64_t)h * D;
#pragma unroll
      for (int e = 0; e < D / 64; ++e) x[e] = KV == kKvBf16 ? bf16_to_f32(src[lane + 64 * e]) : f16_to_f32(src[lane + 64 * e]);
    }
  }
};

// ---------------------------------------------------------------------------------------------------------------------------------
// A rotated query becomes fp16 times 2^-e with the row's largest channel in [2^14, 2^15): relative rounding 2^-11 whatever the row's
// size down to 2^-28 of the largest channel, smaller ones are off by 2^-39 of it.
__device__ __forceinline__ int query_exponent(float top) { return min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 120) - 14; }

// What logits are multiplied by is no less (products of fp16 are below 2^37, so that they stay as good as zero): zero times a masked logit
// would be no number.
constexpr float kLeastScale = 0x1p-126f;

// Queries under a learned rotation, whose 64 KiB a block of rows would read again: a wavefront for NV rows, which read them once.
//   ws: [rows][D] fp16 | [rows] float 2^e
template <int D, int NV>
__global__ __launch_bounds__(256) void prompt_query_kernel(PromptParams p) {
  constexpr int E = D / 64;
  __shared__ __attribute__((aligned(16))) float rows[4][NV * 128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = p.T_q * p.n_q_heads, row0 = (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave) * NV;
  if (row0 >= n) return;
  float* const x = rows[wave];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int64_t row = min(row0 + v, n - 1), at = row / p.n_q_heads * p.q_stride + row % p.n_q_heads * D;
    if (E == 1) x[128 * v + lane + 64] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) x[128 * v + lane + 64 * e] = load_elem(p.q, p.dtype, at + lane + 64 * e);
  }
  wave_sync();
  rotate_row<NV == 1 ? 16 : 8, NV>(p, x, D, lane);
  for (int v = 0; v < NV && row0 + v < n; ++v) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(x[128 * v + lane + 64 * e]));
    top = max_xor32(max_xor16(row_allmax_positive(top)));
    const int ex = query_exponent(top);
    const float down = __uint_as_float((uint32_t)(127 - ex) << 23);
    uint16_t* const q = p.query + (row0 + v) * D;
#pragma unroll
    for (int e = 0; e < E; ++e) q[lane + 64 * e] = f32_to_f16(x[128 * v + lane + 64 * e] * down);
    if (lane == 0) p.query_scale[row0 + v] = __uint_as_float((uint32_t)(127 + ex) << 23);
  }
}

// Keys and values of a tile on their way from the INT4 pages to shared memory: 16-byte pieces of 32 codes and the pairs of their tokens,
// requested a tile ahead.
template <int D, int NW>
struct CodePieces {
  static constexpr int kPieces = 2 * kTileKeys * (D / 32), kEach = kPieces / (64 * NW);
  static_assert(kEach * 64 * NW == kPieces, "whole pieces per thread");
  u32x4 codes[kEach];
  f32x2 pair[kEach];
  f32x2 key_pair, value_pair;   // of key `lane` of the tile, for the tile's exponents
};

// c s - s z of the eight codes of a word, as 16-bit values in channel order
template <typename M>
__device__ __forceinline__ u32x4 widen_codes(uint32_t w, float s, float sz) {
  uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
  // (kept as they are: the compiler would take every code out of w by itself, an instruction each, where the conversion can name its byte)
  asm("" : "+v"(even), "+v"(odd));
  u32x4 x;
  x.x = M::pack(fmaf((float)(even & 0xff), s, -sz), fmaf((float)(odd & 0xff), s, -sz));
  x.y = M::pack(fmaf((float)((even >> 8) & 0xff), s, -sz), fmaf((float)((odd >> 8) & 0xff), s, -sz));
  x.z = M::pack(fmaf((float)((even >> 16) & 0xff), s, -sz), fmaf((float)((odd >> 16) & 0xff), s, -sz));
  x.w = M::pack(fmaf((float)(even >> 24), s, -sz), fmaf((float)(odd >> 24), s, -sz));
  return x;
}
// ... of 32 codes to four places of a row; EXACT: the codes as they are, minus 8
template <typename M, int D, bool VALUE, bool EXACT = false>
__device__ __forceinline__ void put_piece(char* tile, int row, int piece, u32x4 w, float s, float sz) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int chunk = 4 * piece + i;
    *(u32x4*)(tile + row * (2 * D) + 16 * (VALUE ? v_place<D>(row, chunk) : k_place<D>(row, chunk))) = EXACT ? centred(w[i], CodeBits()) : widen_codes<M>(w[i], s, sz);
  }
}
// Products of a row's query and codes minus 8 become logits, s_j (q . (c_j - 8) - (z_j - 8) sum q); pairs: code_pair of the tile's keys.
__device__ __forceinline__ void code_logits(f32x16& x, const f32x2* pairs, int kb, float sum_q, int lane) {
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    const f32x4 two = *(const f32x4*)&pairs[32 * kb + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 2)];
    x[r] = fmaf(two.y, sum_q, x[r]) * two.x;
    x[r + 1] = fmaf(two.w, sum_q, x[r + 1]) * two.z;
  }
}
// Sum of a row's channels as they are multiplied.
template <int D>
__device__ __forceinline__ float channel_sum(const u32x4 (&qf)[D / 16]) {
  float sum = 0.f;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += f16_to_f32(qf[ks][i] & 0xffffu) + f16_to_f32(qf[ks][i] >> 16);
  return add_xor32(sum);
}

// The largest that a token's values can be, from its pair alone; infinity if that is no number.
__device__ __forceinline__ float largest_value(f32x2 pair) {
  const float sz = pair.x * pair.y, most = fmaxf(fabsf(sz), fabsf(fmaf(15.f, pair.x, -sz)));
  return most < INFINITY ? most : INFINITY;
}
// What code_logits needs of a key's pair.  (A key that is no number has no logit: its sum of codes would hide that.)
__device__ __forceinline__ f32x2 code_pair(f32x2 pair) { return f32x2{largest_value(pair) < INFINITY ? pair.x : NAN, 8.f - pair.y}; }

// Sums of values with a larger unit are looked at once more when they have it: below it fp32 holds 2^15 (tile_weights) times 2^15 times 2^31 tokens.
constexpr float kLargeUnit = 0x1p60f;

// 16-bit numbers of a word that are none become zero.
template <typename M>
__device__ __forceinline__ uint32_t numbers_only(uint32_t w) {
  constexpr uint32_t kExponent = std::is_same<M, MathBf16>::value ? 0x7f80 : 0x7c00;
  return ((w & kExponent) == kExponent ? 0 : w & 0xffffu) | (((w >> 16) & kExponent) == kExponent ? 0 : w & 0xffff0000u);
}

template <int D>
__device__ __forceinline__ void clear(RowState<D>& st) {
  st.m = -INFINITY; st.ref = 0.f; st.sum = 0.f;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.o[t][r] = 0.f;
}
// some output sum of the lane's row is no number
template <int D>
__device__ __forceinline__ bool no_sum(const RowState<D>& st) {
  float odd = 0.f;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd = fmaf(st.o[t][r], 0.f, odd);
  return odd != odd;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

__device__ __forceinline__ float wave_max(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(max_xor32(max_xor16(row_allmax_positive(x))))));
}

// The power of two that dequantised keys, or values and the output sums with them, are divided by: the first tile's largest lands at 2^6,
// and it is raised where a tile's would pass 2^15.  So fp16 holds any scale: a number is off by half a step (2^-11), or by 2^-31 of the
// largest so far.  (A power for every tile by itself would be a maximum over all lanes for each: 2048 tokens over 16384 760 us, ragged
// fp16 chunks 174.)
//   Rows need not see the key that sets the unit.  `floor` is no more than the largest that any row met (of keys that all of the
// wavefront's rows see); where the unit is set by one 2^12 times as large the sums are given up, and finish_rows takes the rows again.
//   Tokens that are no numbers do not count.
struct Unit {
  int e = 0;
  float limit = 0.f, floor = 0.f;
  bool lost = false;
  __device__ __forceinline__ bool passed(float mine, bool first) const { return first || __any(mine >= limit); }
  // mine: the largest of the lane's keys; all_see: of those that every row sees, `whole`: all of the tile.  true: raised by 2^by
  template <typename F>
  __device__ __forceinline__ bool fit(float mine, bool first, bool whole, int& by, F all_see) {
    if (!passed(mine, first)) return false;
    auto number = [](float x) { return x < INFINITY ? x : 0.f; };
    const float top = wave_max(number(mine));
    if (!first && top < limit) return false;
    floor = whole ? top : fmaxf(floor, wave_max(number(all_see())));
    lost = lost || top > 4096.f * floor;
    const int to = max((int)(__float_as_uint(top) >> 23) - 127, -100) - 6;
    by = min(to - e, 126);
    e = to;
    limit = to + 15 > 127 ? INFINITY : power_of_two(to + 15);
    return !first;
  }
  __device__ __forceinline__ float down() const { return power_of_two(-e); }
  __device__ __forceinline__ float up() const { return power_of_two(e); }
};
template <int D>
__device__ __forceinline__ void rescale(RowState<D>& st, float by) {
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.o[t][r] *= by;
}

// The queries of a lane column as B operand: channels of k-step ks, half h and place i have bits (ks, h, i), h at bit HALF_BIT.  Those for
// the INT4 pages are rotated here, in registers, and become fp16 times 2^-e (prompt_query_kernel does the same for a learned rotation);
// returns what turns a logit into log2 units.  CODES: the eight channels of a word of codes in the order of `centred`.
template <int D, int KV, int HALF_BIT, bool CODES = false, typename F>
__device__ __forceinline__ float row_query(const PromptParams& p, int64_t token, int head, int lane, u32x4 (&qf)[D / 16], F second) {
  const int half = lane >> 5;
  const bool ready = int4_pages(KV) && p.dense_k;
  const int64_t at = token * p.n_q_heads + head;
  const uint16_t* const src = ready ? p.query + at * D : (const uint16_t*)p.q + token * p.q_stride + (int64_t)head * D;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const u32x4*)(src + (spread_channel<HALF_BIT>(8 * ks) | half << HALF_BIT));
  if constexpr (int4_pages(KV)) {
    if (ready) {
      if (CODES)
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const u32x4 w = qf[ks];
          qf[ks] = u32x4{(w.x & 0xffffu) | w.z << 16, w.x >> 16 | (w.z & 0xffff0000u), (w.y & 0xffffu) | w.w << 16, w.y >> 16 | (w.w & 0xffff0000u)};
        }
#pragma unroll
      for (int i = 0; i < D / 4; ++i) second(i / 4, i % 4, f16_to_f32(qf[i / 4][i % 4] & 0xffffu), f16_to_f32(qf[i / 4][i % 4] >> 16));
      return fmaxf(p.scale * p.query_scale[at], kLeastScale);
    }
    float x[D / 2];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (p.dtype == SAW_BF16) widen2<SAW_BF16>(qf[ks][i], x[8 * ks + 2 * i], x[8 * ks + 2 * i + 1]);
        else widen2<SAW_F16>(qf[ks][i], x[8 * ks + 2 * i], x[8 * ks + 2 * i + 1]);
      }
    float top = 0.f;
    if (p.rot_k) {
      if (p.has_signs) sign_rows<D, HALF_BIT>(x, p.signs, lane);
      fwht_rows<D, HALF_BIT>(x, p.had_block, lane);
    }
    const float norm = p.rot_k ? had_norm(p.had_block) : 1.f;
#pragma unroll
    for (int i = 0; i < D / 2; ++i) {
      x[i] *= norm;
      top = fmaxf(top, fabsf(x[i]));
    }
    const int ex = query_exponent(max_xor32(top));
    const float down = __uint_as_float((uint32_t)(127 - ex) << 23);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i)
{
        const float a = x[8 * ks + (CODES ? i : 2 * i)] * down, b = x[8 * ks + (CODES ? i + 4 : 2 * i + 1)] * down;
        qf[ks][i] = MathF16::pack(a, b);
        second(ks, i, a, b);
      }
    return fmaxf(p.scale * __uint_as_float((uint32_t)(127 + ex) << 23), kLeastScale);
  }
  return p.scale;
}

// This split's (reference, sum) of every row, behind the records of all splits: log2 of what sum and record are relative to.
template <int D>
__device__ __forceinline__ float2* partial_sums(const PromptParams& p) {
  const int64_t rows = p.T_q * p.n_q_heads;
  return (float2*)(p.ws + (int64_t)gridDim.y * rows * D) + (int64_t)blockIdx.y * rows;
}

// The first positions of [j0, j1), j0 a multiple of eight, whose value is NaN, +infinity, -infinity in the lane's channels, and, INT4, of a token whose
// value is a number there and not in all its channels.
template <int D, int KV>
__device__ __forceinline__ void first_odd_values(const RowSource<D, KV>& src, int j0, int j1, int (&first)[3][D / 64], int& mixed) {
  constexpr int E = D / 64, kAhead = 8;                                   // values on their way at once
  mixed = INT32_MAX;
#pragma unroll
  for (int e = 0; e < E; ++e) first[0][e] = first[1][e] = first[2][e] = INT32_MAX;
  for (int j = j0; j < j1; j += kAhead) {
    float v[kAhead][E];
    const int page = src.page_of(j);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) src.load(true, page, min(j + u, j1 - 1), v[u]);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int at = min(j + u, j1 - 1);
      bool none = true;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (v[u][e] != v[u][e]) first[0][e] = min(first[0][e], at);
        if (v[u][e] == INFINITY) first[1][e] = min(first[1][e], at);
        if (v[u][e] == -INFINITY) first[2][e] = min(first[2][e], at);
        none = none && !(fabsf(v[u][e]) < INFINITY);
      }
      if constexpr (int4_pages(KV))
        if (!none && largest_value(src.value_pair_of(page, at)) == INFINITY) mixed = min(mixed, at);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) mixed = min(mixed, __shfl_xor(mixed, d));
}

// A channel's sum, given the first positions of odd values and how many positions its row sees
__device__ __forceinline__ float odd_sum(int nan, int pos, int neg, int sees, float o) {
  return min(nan, max(pos, neg)) < sees ? NAN : pos < sees ? INFINITY : neg < sees ? -INFINITY : o;
}

// Values that are no numbers.  A masked key's weight is zero, and one that is seen may be rounded to zero, but zero times infinity is no number.
// So they are left out, and the first positions of those that were (one reading of the values) say which sums are infinite or none:
//   * tokens in the INT4 pages, whose pairs tell, right away.  What is no number even then - sums of finite values that overflow, tokens that have
//     numbers in some channels only - and sums that lost their precision (Unit) are rows that are taken again, eight keys at a time over
//     the keys that each sees.
//   * 16-bit values, which no instruction looks at on their way, once a sum ended as none: the wavefront goes over its keys again.

// ... with keys and values from memory to operand registers.  (bf16: weights up to 1, with which fewer sums of large values overflow.)
struct LowBf16 : MathBf16 { static constexpr float kRaise = -8.f; };
template <int D, typename M>
__device__ __forceinline__ void rows_of_numbers(const PromptParams& p, int h, int k0, int len, int t0, int t1, int sees, int wend,
                                                const u32x4 (&qf)[D / 16], float scale, RowState<D>& st, int lane) {
  const int half = lane >> 5, in = lane & 31;
  const uint16_t* const k = (const uint16_t*)p.k + (int64_t)k0 * p.k_stride + (int64_t)h * D + 8 * half;
  const uint16_t* const v = (const uint16_t*)p.v + (int64_t)k0 * p.v_stride + (int64_t)h * D + in;
  clear(st);
  for (int t = t0; t < t1 && t * kTileKeys < wend; ++t) {
    f32x16 s[2];
    u32x4 pf[4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int64_t key = min(t * kTileKeys + 32 * kb + in, len - 1);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) s[kb] = M::mfma(*(const u32x4*)(k + key * p.k_stride + 16 * ks), qf[ks], s[kb]);
    }
    tile_mask(s, sees - t * kTileKeys, lane);
    tile_weights<D, typename std::conditional<std::is_same<M, MathBf16>::value, LowBf16, M>::type>(s, scale, st, pf);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const uint16_t* at[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) at[i] = v + (int64_t)min(t * kTileKeys + 16 * ks + 4 * half + (i & 3) + 8 * (i >> 2), len - 1) * p.v_stride;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = numbers_only<M>((uint32_t)at[2 * i][32 * c] | (uint32_t)at[2 * i + 1][32 * c] << 16);
        st.o[c] = M::mfma(w, pf[ks], st.o[c]);
      }
    }
  }
}

// The end of a wavefront's 32 rows: outputs, or partial records [split][row][D] and [split][row] (reference, sum) where the keys are split
// or a learned rotation has to be undone.  scale: of the rows' logits; sees: keys that the lane's row sees, wend: the last row; odd: values were
// left out (INT4); lost: the sums are not precise enough.
template <int D, int KV, int HALF_BIT, bool CODES = false>
__device__ __forceinline__ void finish_rows(const PromptParams& p, const RowTile& rt, int w0, int last, int row, int h, int64_t token, int head,
                                            int k0, int len, int t0, int t1, int sees, int wend, bool odd, bool lost, const u32x4 (&qf)[D / 16], float scale,
                                            RowState<D>& st, int lane) {
  constexpr bool kInt4 = int4_pages(KV);
  const int shift = __builtin_ctz(p.group);
  float sum = add_xor32(st.sum);
  const int64_t at = token * p.n_q_heads + head;
  const bool split = gridDim.y > 1 || (kInt4 && p.dense_v);
  const int64_t rows = p.T_q * p.n_q_heads;
  float* const records = p.ws + (int64_t)blockIdx.y * rows * D;
  float2* const ml = partial_sums<D>(p);
  uint32_t again = 0;                                                     // rows that are taken again
  if constexpr (!kInt4) odd = __any(row <= last && no_sum<D>(st));
  if (w0 <= last && (odd || lost)) {
    constexpr int E = D / 64, kAhead = 8;                                 // keys at once
    using M = typename std::conditional<KV == kKvBf16, MathBf16, MathF16>::type;
    if constexpr (!kInt4) {
      rows_of_numbers<D, M>(p, h, k0, len, t0, t1, sees, wend, qf, scale, st, lane);
      sum = add_xor32(st.sum);
    }
    const RowSource<D, KV> src = {p, rt.b, h, k0, lane};
    int first[3][E], mixed;
    first_odd_values(src, t0 * kTileKeys, min(wend, t1 * kTileKeys), first, mixed);
    bool redo = lost || mixed < sees;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int from = (32 * t + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) & 63;
        const int nan = __shfl(first[0][t / 2], from), pos = __shfl(first[1][t / 2], from), neg = __shfl(first[2][t / 2], from);
        redo = redo || !(fabsf(st.o[t][r]) < INFINITY);
        st.o[t][r] = sum == sum ? odd_sum(nan, pos, neg, sees, st.o[t][r]) : NAN;       // (a logit is none: nor is anything of the row)
      }
    const uint64_t which = __ballot(kInt4 && redo && row <= last && sum == sum);
    again = __builtin_amdgcn_readfirstlane((uint32_t)which | (uint32_t)(which >> 32));
    if constexpr (kInt4) for (uint32_t left = again; left; left &= left - 1) {
      const int i = __builtin_ctz(left), tok_i = (w0 + i) >> shift;
      const int64_t mine = (int64_t)(rt.begin + tok_i) * p.n_q_heads + h * p.group + ((w0 + i) & (p.group - 1));
      const int sees_i = max(min(len, len - rt.n + tok_i + 1), 0);
      const int end = min(sees_i, t1 * kTileKeys);
      const float row_scale = __shfl(scale, i);
      float q[E], acc[E], m = -INFINITY, den = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) { q[e] = 0.f; acc[e] = 0.f; }
      // (channel c of row i is in register c's place of lane i or i + 32)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = lane + 64 * e, half = (c >> HALF_BIT) & 1, in = (c & ((1 << HALF_BIT) - 1)) | c >> (HALF_BIT + 1) << HALF_BIT;
        const int v = CODES ? (in & ~7) | 2 * (in & 3) | ((in >> 2) & 1) : in;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t w = __shfl((int)qf[ks][d], i + 32 * half), x = v & 1 ? w >> 16 : w & 0xffffu;
            if (v >> 1 == 4 * ks + d) q[e] = f16_to_f32(x) * row_scale;
          }
      }
      for (int j = t0 * kTileKeys; j < end; j += kAhead) {
        float kv[kAhead][E], x[kAhead], top = m;
        const int page = src.page_of(j);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) src.load(false, page, min(j + u, end - 1), kv[u]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          x[u] = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) x[u] = fmaf(q[e], kv[u][e], x[u]);
          x[u] = add_xor32(add_xor16(row_allsum(x[u])));
          if (j + u < end) top = fmaxf(top, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) src.load(true, page, min(j + u, end - 1), kv[u]);
        const float ref = top == -INFINITY ? 0.f : top, alpha = fast_exp2(m - ref);
        m = top;
        den *= alpha;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= alpha;
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (j + u < end) {
            const float w = fast_exp2(x[u] - ref);
            den += w;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(w, kv[u][e], acc[e]);
          }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = odd_sum(first[0][e], first[1][e], first[2][e], sees_i, acc[e]);
      if (split) {
#pragma unroll
        for (int e = 0; e < E; ++e) records[mine * D + lane + 64 * e] = acc[e];
        if (lane == 0) ml[mine] = make_float2(m, den);
      } else {
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = den == 0.f ? 0.f : acc[e] / den;
        if (p.rot_v) {                                                   // (lane + 64 e: bits 0 to 5 across the lanes, the last in the lane)
          for (int st = 1; st < p.had_block && st < 64; st <<= 1)
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float other = __shfl_xor(x[e], st);
              x[e] = lane & st ? other - x[e] : x[e] + other;
            }
          if (E == 2 && p.had_block == 128) { const float a = x[0], b = x[E - 1]; x[0] = a + b; x[E - 1] = a - b; }
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] = apply_sign(p.signs, lane + 64 * e, x[e] * had_norm(p.had_block));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) store_elem(p.out, p.dtype, mine * D + lane + 64 * e, x[e]);
      }
    }
  }
  const bool done = row > last || (again >> (lane & 31) & 1);
  if (split) {
    if (done) return;
    if (lane < 32) ml[at] = make_float2(st.m == -INFINITY ? st.m : st.ref, sum);
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *(f32x4*)(records + at * D + 32 * t + 2 * r + 4 * (lane >> 5)) = f32x4{st.o[t][r], st.o[t][r + 1], st.o[t][r + 2], st.o[t][r + 3]};
    return;
  }
  float inv = sum == 0.f ? 0.f : 1.f / sum;
  float x[D / 2];
#pragma unroll
  for (int i = 0; i < D / 2; ++i) x[i] = st.o[i / 16][i % 16];
  if (kInt4 && p.rot_v) {
    fwht_rows<D, 2>(x, p.had_block, lane);                               // (accumulators: the half is bit 2 of the channel)
    if (p.has_signs) sign_rows<D, 2>(x, p.signs, lane);
    inv *= had_norm(p.had_block);
  }
  if (done) return;
#pragma unroll
  for (int i = 0; i < D / 2; i += 4) {
    const bool bf16 = kInt4 ? p.dtype == SAW_BF16 : KV == kKvBf16;
    *(u32x2*)((uint16_t*)p.out + at * D + spread_channel<2>(i) + 4 * (lane >> 5)) =
        bf16 ? u32x2{MathBf16::pack(x[i] * inv, x[i + 1] * inv), MathBf16::pack(x[i + 2] * inv, x[i + 3] * inv)}
             : u32x2{MathF16::pack(x[i] * inv, x[i + 1] * inv), MathF16::pack(x[i + 2] * inv, x[i + 3] * inv)};
  }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Attention of packed rows.  A block takes 32 rows per wavefront and goes over the keys in tiles of 64, double-buffered in shared memory,
// one barrier a tile.  Keys and values of 16 bits come from memory straight into the buffer (each transfer has a whole tile's
// products to arrive in).  Those of the INT4 pages are requested a tile ahead into registers and written behind the tile's products:
// as fp16 times powers of two (Unit), each once per block and not once per row.
//   Roundings: weights to the type of the values, whose half step the output has anyway; over the pages queries, weights and values to
// fp16, and keys too where outputs are bf16 (off by 2.0e-3 with four channels of the keys 20 times as large as the others, 1.6e-3 of it bf16's
// own).  With fp16 outputs keys stay exact codes and their scales and zero-points meet the logits (kKvCodes): 5.3e-4 instead of 1.2e-3, of which
// fp16's own is 2.1e-4, for 32 multiplications and 32 additions a tile more (2048 tokens over 16384 755 us instead of 714, ragged chunks of 64
// channels 176 and 162).  Two limbs of the query as in saw_weights.hip are half as much matrix work again: those chunks 208 us for 3.3e-4.
//   Bound by the matrix cores at the clock that they leave, with the exponentials behind them: 8192 causal tokens, 32 query and 8 kv heads
// of 128 channels, 508 to 529 us from card to card, 1.04 to 1.08 PFLOP/s (a library product of 8192^3 1.27); 64 channels, where a logit has half the
// products, 0.86; 2048 tokens over 16384 in the pages 709 to 725 us, 0.81 to 0.82, with 200 M instructions of the vector ALU, 0.3 of them for the codes.
template <int D, int KV, int NW>
__global__ __launch_bounds__(64 * NW, D == 64 && KV == kKvCodes ? 3 : 2) void prompt_kernel(PromptParams p) {
  constexpr int R = 32 * NW, kRow = 2 * D, kTile = kTileKeys * kRow, kInstr = kTile / 1024, kRpi = 1024 / kRow;
  constexpr bool kInt4 = int4_pages(KV), kCodes = KV == kKvCodes;
  using M1 = typename std::conditional<KV == kKvBf16, MathBf16, MathF16>::type;      // queries and keys, weights and values
  using M2 = M1;
  __shared__ __attribute__((aligned(1024))) char lds[2][2][kTile];       // [buffer][K, V]
  __shared__ __attribute__((aligned(16))) f32x2 pairs[kCodes ? 2 : 1][kCodes ? kTileKeys : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % p.n_kv_heads;
  // (the last tiles of a causal sequence have the most keys and start first)
  const int64_t tile = (int64_t)gridDim.x / p.n_kv_heads - 1 - blockIdx.x / p.n_kv_heads;
  RowTile rt;
  if (!find_row_tile(p, tile, R, lane, rt)) return;
  int k0 = 0, len;
  if constexpr (kInt4) len = min(max(p.seq_lens[rt.b], 0), p.bound);
  else packed_range(p.cu_k, rt.b, p.T_k, k0, len);
  const int shift = __builtin_ctz(p.group);
  auto sees_of = [&](int row) { return p.causal ? max(min(len, len - rt.n + (row >> shift) + 1), 0) : len; };   // (of a row of the sequence)
  const int last = rt.row0 + rt.rows - 1;
  const int w0 = rt.row0 + 32 * wave, w1 = min(w0 + 31, last);            // the wavefront's rows; none if w0 > last
  const int row = w0 + (lane & 31);
  const int sees = row <= last ? sees_of(row) : 0;
  const int kend = sees_of(last), wend = w0 <= last ? sees_of(w1) : 0, wfull = w0 + 31 <= last ? sees_of(w0) : 0;
  const int nt = (kend + kTileKeys - 1) / kTileKeys, per = (nt + (int)gridDim.y - 1) / (int)gridDim.y;
  const int t0 = (int)blockIdx.y * per, t1 = min(nt, t0 + per);

  const int64_t token = rt.begin + (min(row, last) >> shift);
  const int head = h * p.group + (row & (p.group - 1));
  u32x4 qf[D / 16];
  const float scale = row_query<D, KV, 3, kCodes>(p, token, head, lane, qf, [](int, int, float, float) {});
  RowState<D> st;
  clear(st);

  bool odd = false;                                                       // (INT4) values that are no numbers were met
  Unit keys, values;
  const float sum_q = kCodes ? channel_sum<D>(qf) : 0.f;
  auto products = [&](int buf, int t, float tile_scale) {
    if (t * kTileKeys >= wend) return;
    f32x16 s[2];
    u32x4 pf[4];
    tile_logits<D, M1>(lds[buf][0], qf, s, lane);
    if constexpr (kCodes)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) code_logits(s[kb], pairs[buf], kb, sum_q, lane);
    if ((t + 1) * kTileKeys > wfull) tile_mask(s, sees - t * kTileKeys, lane);
    tile_weights<D, M2>(s, tile_scale, st, pf);
    tile_values<D, M2>(lds[buf][1], pf, st, lane);
  };

  const uint16_t* const kp = (const uint16_t*)p.k + (int64_t)k0 * p.k_stride + (int64_t)h * D;
  const uint16_t* const vp = (const uint16_t*)p.v + (int64_t)k0 * p.v_stride + (int64_t)h * D;
  if constexpr (!kInt4) {
    auto load = [&](int buf, int t) {
#pragma unroll
      for (int j = 0; j < kInstr / NW; ++j) {
        const int in = wave * (kInstr / NW) + j;                             // 1024 bytes: kRpi rows
        const int r = in * kRpi + lane / (D / 8), place = lane % (D / 8);
        const int64_t key = min(t * kTileKeys + r, len - 1);                 // (behind the end: the last key again, masked)
        __builtin_amdgcn_global_load_lds((const GLOBAL_AS void*)(kp + key * p.k_stride + 8 * k_place<D>(r, place)), (LDS_AS void*)(lds[buf][0] + in * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const GLOBAL_AS void*)(vp + key * p.v_stride + 8 * v_place<D>(r, place)), (LDS_AS void*)(lds[buf][1] + in * 1024), 16, 0, 0);
      }
    };
    if (t0 < t1) load(0, t0);
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1;
      __builtin_amdgcn_s_waitcnt(0x0F70);                                   // vmcnt(0): this wavefront's part of tile t is there
      lds_barrier();                                                        // ... everybody's is, and nobody reads the other buffer any more
      if (t + 1 < t1) load(buf ^ 1, t + 1);
      products(buf, t, scale);
    }
  } else {
    using Pieces = CodePieces<D, NW>;
    const int32_t* const pages = p.page_table + (int64_t)rt.b * p.max_pages;
    const int threads = 64 * NW;
    TilePages ids;
    auto request = [&](int t, Pieces& c) {
      ids.ready(p, h);
#pragma unroll
      for (int j = 0; j < Pieces::kEach; ++j) {
        const int piece = j * threads + threadIdx.x, value = piece >= Pieces::kPieces / 2, i = value ? piece - Pieces::kPieces / 2 : piece;
        const int key = i / (D / 32);
        const uint32_t tile = ids.tile_of(key);
        c.codes[j] = ((const u32x4*)vector_codes<D>(value ? p.v_codes : p.k_codes, tile, key))[i % (D / 32)];
        c.pair[j] = *vector_pair(value ? p.v_meta : p.k_meta, tile, key);
        if (t * kTileKeys + key >= len) c.pair[j] = f32x2{0.f, 0.f};         // (slots behind the end may hold anything)
      }
      c.key_pair = *vector_pair(p.k_meta, ids.tile_of(lane), lane);
      c.value_pair = *vector_pair(p.v_meta, ids.tile_of(lane), lane);
      if (t * kTileKeys + lane >= len) c.key_pair = c.value_pair = f32x2{0.f, 0.f};
    };
    const int seen = max(sees_of(w0), t0 * kTileKeys + 1);                   // keys in front of it are seen by every row that sees any
    auto put = [&](int buf, Pieces& c, int t) {                              // returns what the tile's logits are to be multiplied by
      const bool whole = (t + 1) * kTileKeys <= seen, mine = t * kTileKeys + lane < seen;
      const float key = largest_value(c.key_pair), value = largest_value(c.value_pair);
      int by;
      if constexpr (!kCodes) keys.fit(key, t == t0, whole, by, [&] { return mine ? key : 0.f; });
      else if (wave == 0) pairs[buf][lane] = code_pair(c.key_pair);
      if (values.passed(value, t == t0)) {
        if (__any(value == INFINITY)) {
          odd = true;
#pragma unroll
          for (int j = 0; j < Pieces::kEach; ++j)
            if (j * threads + (int)threadIdx.x >= Pieces::kPieces / 2 && largest_value(c.pair[j]) == INFINITY) c.pair[j] = f32x2{0.f, 0.f};
        }
        if (values.fit(value, t == t0, whole, by, [&] { return mine ? value : 0.f; })) rescale<D>(st, power_of_two(-by));
      }
      const float down = keys.down(), down_v = values.down();
#pragma unroll
      for (int j = 0; j < Pieces::kEach; ++j) {
        const int piece = j * threads + threadIdx.x, value = piece >= Pieces::kPieces / 2, i = value ? piece - Pieces::kPieces / 2 : piece;
        const float s = c.pair[j].x, sz = s * c.pair[j].y;
        if (value) put_piece<M2, D, true>(lds[buf][1], i / (D / 32), i % (D / 32), c.codes[j], s * down_v, sz * down_v);
        else put_piece<M1, D, false, kCodes>(lds[buf][0], i / (D / 32), i % (D / 32), c.codes[j], s * down, sz * down);
      }
      return kCodes ? 1.f : keys.up();
    };
    Pieces c;
    float tile_scale = 1.f;
    if (t0 < t1) {
      ids.fetch(pages, t0, len);
      request(t0, c);
      ids.fetch(pages, t0 + 1, len);
      tile_scale = put(0, c, t0);
    }
    for (int t = t0; t < t1; ++t) {
      const int buf = (t - t0) & 1;
      lds_barrier();
      if (t + 1 < t1) {
        request(t + 1, c);
        ids.fetch(pages, t + 2, len);
      }
      products(buf, t, fmaxf(scale * tile_scale, kLeastScale));
      if (t + 1 < t1) tile_scale = put(buf ^ 1, c, t + 1);
    }
    rescale<D>(st, values.up());
    if (values.up() > kLargeUnit) odd = odd || __any(row <= last && no_sum<D>(st));
  }
  finish_rows<D, KV, 3, kCodes>(p, rt, w0, last, row, h, token, head, k0, len, t0, t1, sees, wend, odd, keys.lost || values.lost, qf, scale, st, lane);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Few rows over the INT4 pages (draft tokens to verify, a decode step's queries): a block takes 32 rows, and its wavefronts share out the
// keys, every fourth tile each, so that none waits for another until they join their states at the end.  Keys go from memory to operand
// registers as exact codes - a lane holds one half of one key's channels, which the queries' k-steps follow - and their scales and zero-points to
// the logits, as in saw_weights.hip: half of the instructions of dequantised keys (16 tokens a sequence 79 -> 74 us); with 128 rows a
// block, where codes are widened once for all, it would be more of them.  Values go through 64 rows of shared memory of the wavefront's own for
// the transposing reads.
//   Bound by the vector ALU, 1200 instructions for 64 keys, half of them for the codes, by the conflicts of the values' writes (0.57 of the cycles
// that shared memory is addressed in) and by the longest sequences, whose blocks start with all the others: 32 sequences of 5 tokens over 512
// to 4096, 88 MB, 50 us and 6.6 for the merge.
//   LIMBS, for fp16 outputs: the query is two limbs, the second read from shared memory for every 32 keys (but for a learned rotation's, which come as
// one): off by 3.2e-4 instead of 5.2e-4, 32 x 5 tokens 57 us instead of 53.3.  bf16's own half step hides that: 1.7e-3 either way.
template <int D, bool LIMBS>
__global__ __launch_bounds__(256, 2) void few_rows_kernel(PromptParams p) {
  constexpr int NW = 4, kRow = 2 * D, kTile = kTileKeys * kRow, kHalfBit = D == 128 ? 6 : 5, kWords = D / 16, kPieces = D / 32;
  static_assert(kTile == 64 * (D / 2) * 4, "a state fits the wavefront's tile");
  __shared__ __attribute__((aligned(1024))) char lds[NW][kTile];
  __shared__ u32x4 limbs[LIMBS ? D / 16 : 1][64];
  __shared__ float2 join[NW][64];
  __shared__ __attribute__((aligned(16))) f32x2 pairs[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % p.n_kv_heads;
  RowTile rt;
  if (!find_row_tile(p, blockIdx.x / p.n_kv_heads, 32, lane, rt)) return;
  const int len = min(max(p.seq_lens[rt.b], 0), p.bound);
  const int shift = __builtin_ctz(p.group);
  const int last = rt.row0 + rt.rows - 1, row = rt.row0 + (lane & 31);
  auto sees_of = [&](int r) { return max(min(len, len - rt.n + (r >> shift) + 1), 0); };
  const int sees = row <= last ? sees_of(row) : 0, kend = sees_of(last), kfull = rt.rows == 32 ? sees_of(rt.row0) : 0;
  // (a tile for every wavefront at least: of a short sequence the last splits have none)
  const int nt = (kend + kTileKeys - 1) / kTileKeys, per = max((nt + (int)gridDim.y - 1) / (int)gridDim.y, NW);
  const int t0 = (int)blockIdx.y * per, t1 = min(nt, t0 + per);
  const int64_t token = rt.begin + (min(row, last) >> shift);
  const int head = h * p.group + (row & (p.group - 1));
  if (t0 >= t1 && gridDim.y > 1) {
    if (wave == 0 && lane < 32 && row <= last) partial_sums<D>(p)[token * p.n_q_heads + head] = make_float2(-INFINITY, 0.f);
    return;
  }
  const int32_t* const pages = p.page_table + (int64_t)rt.b * p.max_pages;
  char* const mine = lds[wave];

  u32x4 kc[2][kWords / 4], vc[kPieces];
  f32x2 kpair, vpair[kPieces];                                            // (of key `lane`; of the pieces' tokens)
  TilePages ids;
  auto request = [&]() __attribute__((always_inline)) {
    ids.ready(p, h);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int key = 32 * kb + (lane & 31);
      const uint32_t tile = ids.tile_of(key);
      const u32x4* const src = (const u32x4*)(vector_codes<D>(p.k_codes, tile, key) + (lane >> 5) * (D / 4));
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) kc[kb][i] = src[i];
    }
    kpair = *vector_pair(p.k_meta, ids.tile_of(lane), lane);
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int piece = 64 * j + lane, key = piece / kPieces;
      const uint32_t tile = ids.tile_of(key);
      vc[j] = ((const u32x4*)vector_codes<D>(p.v_codes, tile, key))[piece % kPieces];
      vpair[j] = *vector_pair(p.v_meta, tile, key);
    }
  };
  if (t0 + wave < t1) {
    ids.fetch(pages, t0 + wave, len);
    request();
    ids.fetch(pages, t0 + wave + NW, len);
  }
  u32x4 qf[D / 16];
  float sum_lo = 0.f;
  const float scale = row_query<D, kKvInt4, kHalfBit, true>(p, token, head, lane, qf, [&](int ks, int i, float a, float b) {
    if constexpr (LIMBS) {
      const uint32_t lo = MathF16::pack(a - f16_to_f32(qf[ks][i] & 0xffffu), b - f16_to_f32(qf[ks][i] >> 16));
      sum_lo += f16_to_f32(lo & 0xffffu) + f16_to_f32(lo >> 16);
      if (ks % NW == wave) limbs[ks][lane][i] = lo;
    }
  });
  const float sum_q = channel_sum<D>(qf) + add_xor32(sum_lo);
  if (LIMBS) lds_barrier();
  const CodeBits bits;
  RowState<D> st;
  clear(st);

  bool odd = false;                                                       // values that are no numbers were met
  Unit values;
  const int seen = max(sees_of(rt.row0), (t0 + wave) * kTileKeys + 1);
  for (int t = t0 + wave; t < t1; t += NW) {
    // (slots behind the end may hold anything)
    auto largest_of_values = [&](int end) {
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < kPieces; ++j)
        if (t * kTileKeys + (64 * j + lane) / kPieces < end) top = fmaxf(top, largest_value(vpair[j]));
      return top;
    };
    int by;
    const bool whole = (t + 1) * kTileKeys <= seen;
    const float top = largest_of_values(len);
    if (values.passed(top, t == t0 + wave)) {
      if (__any(top == INFINITY)) {
        odd = true;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
          if (largest_value(vpair[j]) == INFINITY) vpair[j] = f32x2{0.f, 0.f};
      }
      if (values.fit(largest_of_values(len), t == t0 + wave, whole, by, [&] { return largest_of_values(seen); })) rescale<D>(st, power_of_two(-by));
    }
    const float down_v = values.down();
    // logits: s_j (q . (c_j - 8) - (z_j - 8) sum q), with the codes exact and each pair from shared memory where its key stands
    pairs[wave][lane] = t * kTileKeys + lane < len ? code_pair(kpair) : f32x2{0.f, 0.f};
    f32x16 x[2];
    u32x4 pf[4];
    wave_sync();
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[kb][r] = 0.f;
      if (LIMBS) asm volatile("" ::: "memory");                              // (or the limbs would be kept in registers after all)
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const u32x4 k = centred(kc[kb][ks / 4][ks % 4], bits);
        if constexpr (LIMBS) x[kb] = MathF16::mfma(k, limbs[ks][lane], x[kb]);
        x[kb] = MathF16::mfma(k, qf[ks], x[kb]);
      }
      code_logits(x[kb], pairs[wave], kb, sum_q, lane);
      // (128 channels: or the compiler puts this off until the values are written, with all pairs in registers, and spills: 54 us become 87.  With
      // 64 they fit: 36 us put off, 38 in place.)
      if (D == 128) asm volatile("" : "+v"(x[kb]));
    }
    wave_sync();
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int key = (64 * j + lane) / kPieces;
      const bool there = t * kTileKeys + key < len;
      put_piece<MathF16, D, true>(mine, key, lane % kPieces, vc[j], there ? vpair[j].x * down_v : 0.f, there ? vpair[j].x * vpair[j].y * down_v : 0.f);
    }
    wave_sync();
    if (t + NW < t1) {
      request();
      ids.fetch(pages, t + 2 * NW, len);
    }
    if ((t + 1) * kTileKeys > kfull) tile_mask(x, sees - t * kTileKeys, lane);
    tile_weights<D, MathF16>(x, scale, st, pf);
    tile_values<D, MathF16>(mine, pf, st, lane);
  }
  // the other wavefronts' states join the first's
  wave_sync();
  rescale<D>(st, values.up());
  if (lane == 0) pairs[wave][0] = f32x2{odd || values.up() > kLargeUnit ? 1.f : 0.f, values.lost ? 1.f : 0.f};
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < D / 2; i += 4) *(f32x4*)(mine + i * 256 + 16 * lane) = f32x4{st.o[i / 16][i % 16], st.o[i / 16][i % 16 + 1], st.o[i / 16][i % 16 + 2], st.o[i / 16][i % 16 + 3]};
    join[wave][lane] = make_float2(st.m, st.sum);
  }
  __syncthreads();
  if (wave > 0) return;
  float m = st.m;
#pragma unroll
  for (int w = 1; w < NW; ++w) m = fmaxf(m, join[w][lane].x);
  const float ref = m == -INFINITY ? 0.f : m;
  const float alpha = fast_exp2(st.m - ref);
  st.sum *= alpha;
  rescale<D>(st, alpha);
  for (int w = 1; w < NW; ++w) {
    const float a = fast_exp2(join[w][lane].x - ref);
    st.sum = fmaf(a, join[w][lane].y, st.sum);
#pragma unroll
    for (int i = 0; i < D / 2; i += 4) {
      const f32x4 o = *(const f32x4*)(lds[w] + i * 256 + 16 * lane);
#pragma unroll
      for (int k = 0; k < 4; ++k) st.o[i / 16][i % 16 + k] = fmaf(a, o[k], st.o[i / 16][i % 16 + k]);
    }
  }
  st.m = m;
  st.ref = m == -INFINITY ? 0.f : m - MathF16::kRaise;
  float look = 0.f, lost = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) { look += pairs[w][0].x; lost += pairs[w][0].y; }
  finish_rows<D, kKvInt4, kHalfBit, true>(p, rt, rt.row0, last, row, h, token, head, 0, len, t0, t1, sees, kend, look != 0.f, lost != 0.f, qf, scale, st,
                                          lane);
}

// The output of a row from its partial records; false: the row is no sequence's.
template <int D>
__device__ __forceinline__ bool merged_row(const PromptParams& p, int splits, int64_t row, int lane, float (&o)[D / 64]) {
  constexpr int E = D / 64;
  const int64_t rows = p.T_q * p.n_q_heads;
  const int64_t token = row / p.n_q_heads;
  const int b = last_not_above(p.B, token, lane, [&](int i) { return clamped_offset(p.cu_q, i, p.T_q); });
  if (b < 0 || token >= clamped_offset(p.cu_q, b + 1, p.T_q)) return false;
  const float2* const ml = (const float2*)(p.ws + (int64_t)splits * rows * D);
  float2 mine = make_float2(-INFINITY, 0.f);                              // (a split a lane: kMaxKeySplits of them)
  if (lane < splits) mine = ml[lane * rows + row];
  const float m = max_xor32(max_xor16(row_allmax(mine.x)));
  const float weight = fast_exp2(mine.x - (m == -INFINITY ? 0.f : m));
  const float den = add_xor32(add_xor16(row_allsum(weight * mine.y)));
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  constexpr int kAhead = 8;                                               // records on their way at once
  for (int s0 = 0; s0 < splits; s0 += kAhead) {
    float v[kAhead][E];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = p.ws[(min(s0 + k, splits - 1) * rows + row) * D + E * lane + e];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), min(s0 + k, splits - 1)));
      if (s0 + k < splits && w != 0.f)                                     // (a split without keys leaves no record)
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(w, v[k][e], o[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = den == 0.f ? 0.f : o[e] / den;
  return true;
}

// Joins the partial records of a row: one wavefront a row, eight records on their way at once.  5120 rows in two splits 6.7 us, most of it
// latency.  (NV rows under a learned rotation, whose 64 KiB they read once.)
template <int D, bool INT4, int NV>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptParams p, int splits) {
  constexpr int E = D / 64;
  __shared__ __attribute__((aligned(16))) float rotated[4][INT4 ? NV * 128 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rows = p.T_q * p.n_q_heads, row0 = (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave) * NV;
  if (row0 >= rows) return;
  const bool turn = INT4 && (p.rot_v || p.dense_v);
  uint32_t whose = 0;                                                     // rows of a sequence
  float o[NV][E];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if (row0 + v < rows && merged_row<D>(p, splits, row0 + v, lane, o[v])) whose |= 1u << v;
    if (turn) {
      float* const x = rotated[wave] + 128 * v;
      if (E == 1) x[lane + 64] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) x[E * lane + e] = whose >> v & 1 ? o[v][e] : 0.f;
    }
  }
  if (!whose) return;
  if (turn) {
    wave_sync();
    unrotate_row<NV == 1 ? 16 : 8, NV>(p, rotated[wave], D, lane);
  }
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (whose >> v & 1)
#pragma unroll
      for (int e = 0; e < E; ++e)
        store_elem(p.out, p.dtype, (row0 + v) * D + E * lane + e, turn ? rotated[wave][128 * v + E * lane + e] : o[v][e]);
}

// How a call is handed out: rows of a block, splits of the keys.
//   * INT4 pages and at most 64 rows a sequence on average: blocks of 32 rows whose wavefronts share out the keys (32 sequences of 512 to 4096
//     tokens, 32 query / 8 kv heads: 5 new tokens 54 us, 181 in blocks of 128 rows); at most 192 with 128 to 384 (sequence, kv head) pairs, where
//     blocks of 128 rows are too few to be dealt out evenly (blocks of 32 and of 128 rows: 24 tokens, 16 sequences 70 us and 69, 24 94 and 106,
//     32 113 and 126, 48 171 and 182; 32 x 48 160 and 171; 31 x 1 and one chunk of 700 104 and 165; but 8 x 24 51 and 43, 64 x 24 206 and 185,
//     32 x 64 199 and 190; fp16, 24 tokens, 16 sequences 80 and 73, 24 104 and 111, 32 126 and 133, 48 188 and 193, 32 of 64 channels 76 and 96);
//   * 4096 rows a sequence and more, and a block for every compute unit: 256 rows, eight wavefronts, so that keys are brought in (and
//     codes widened) half as often (8192 causal tokens 520 us, 544 in blocks of 128; 2048 tokens over 16384 in the pages 708 and 777; but 19
//     packed prompts of 60 to 1437 tokens 181 and 178, four short ones 13.2 and 11.2);
//   * 128 rows otherwise.
// Keys are split while a call has fewer blocks than the chip holds, two for a compute unit (a little more in blocks of 32 rows, whose
// wavefronts go their own ways: two splits of 256 blocks 54 us, one 80, three 58; of 264 to 280 of uneven length 62, one 66 to 71), into parts of 256 keys at least.  Blocks are counted as those of
// sequences of like length: the grid has one more for each sequence, of which many are empty (with those counted too, 8 x 24 tokens 56 us instead
// of 43, 4 x 256 137 instead of 115).  A split where the chip is full already costs its records: two sequences of 2000 tokens, 512 blocks, 88 us,
// in two splits 161.
struct PromptPlan { int rows, splits; };
constexpr int kMaxKeySplits = 64;
static PromptPlan prompt_plan(bool int4, int D, int G, int Hkv, int64_t T, int B, int64_t max_k_len) {
  PromptPlan r = {128, 1};
  int64_t want = 512;
  const int64_t pairs = (int64_t)B * Hkv;
  if (int4 && T * G <= (pairs >= 128 && pairs <= 384 ? 192 : 64) * (int64_t)B) { r.rows = 32; want = 560; }
  else if ((D == 128 || !int4) && T * G >= 4096 * (int64_t)B && row_tiles(T, G, 256, B) * Hkv >= 256) r.rows = 256;
  const int64_t all = (int64_t)B * r.rows, blocks = B * ((T * G + all - 1) / all) * Hkv;             // of sequences of like length
  int64_t s = want / (blocks < 1 ? 1 : blocks), most = (max_k_len + 255) / 256;
  if (r.rows == 256) s = 1;
  if (s > most) s = most;
  r.splits = s < 1 ? 1 : s > kMaxKeySplits ? kMaxKeySplits : (int)s;
  return r;
}
static size_t record_bytes(int D, int64_t rows, int splits) { return (size_t)rows * splits * (D + 2) * 4; }
// Rows leave records where their keys are split, or for a learned rotation to be undone by the merge.
static bool keeps_records(const PromptPlan& plan, bool dense_v) { return plan.splits > 1 || dense_v; }

// Rows of a wavefront where a learned rotation has to be read: four from 8192 on (32 sequences of 8 new tokens, 32 heads, level; of 16 145 us in
// ones, 126 in eights, 114 in fours; of 64 465, 330 and 323; 2048 tokens over 16384 1003, 874 and 865).
constexpr int kTurnedAtOnce = 4;
static bool turn_many(const PromptParams& p) { return p.T_q * p.n_q_heads >= 8192; }
// Blocks of four wavefronts for `rows` rows, NV a wavefront.  (A grid's width is counted in threads, in 32 bits.)
static dim3 row_grid(int64_t rows, int NV) {
  const int64_t blocks = (rows + 4 * NV - 1) / (4 * NV);
  const unsigned wide = (unsigned)(blocks < 1 << 22 ? blocks : 1 << 22);
  return dim3(wide, (unsigned)((blocks + wide - 1) / wide));
}

template <int D, int KV>
static void launch_rows(const PromptParams& p, const PromptPlan& plan, hipStream_t st) {
  const int64_t rows = p.T_q * p.n_q_heads;
  const dim3 grid((unsigned)(row_tiles(p.T_q, p.group, plan.rows, p.B) * p.n_kv_heads), plan.splits), block(256);
  if constexpr (KV == kKvInt4 && D == kDenseD)
    if (p.dense_k) {
      if (turn_many(p)) prompt_query_kernel<D, kTurnedAtOnce><<<row_grid(rows, kTurnedAtOnce), block, 0, st>>>(p);
      else prompt_query_kernel<D, 1><<<row_grid(rows, 1), block, 0, st>>>(p);
    }
  if (plan.rows == 128) {
    if (KV == kKvInt4 && p.dtype == SAW_F16) prompt_kernel<D, KV == kKvInt4 ? kKvCodes : KV, 4><<<grid, block, 0, st>>>(p);
    else prompt_kernel<D, KV, 4><<<grid, block, 0, st>>>(p);
  }
  if constexpr (KV == kKvInt4)
    if (plan.rows == 32) {
      if (p.dtype == SAW_F16) few_rows_kernel<D, true><<<grid, block, 0, st>>>(p);
      else few_rows_kernel<D, false><<<grid, block, 0, st>>>(p);
    }
  if constexpr (D == 128 || KV != kKvInt4)
    if (plan.rows == 256) {
      if (KV == kKvInt4 && p.dtype == SAW_F16) prompt_kernel<D, KV == kKvInt4 ? kKvCodes : KV, 8><<<grid, dim3(512), 0, st>>>(p);
      else prompt_kernel<D, KV, 8><<<grid, dim3(512), 0, st>>>(p);
    }
  if constexpr (KV == kKvInt4 && D == kDenseD)
    if (p.dense_v && turn_many(p)) {
      prompt_merge_kernel<D, true, kTurnedAtOnce><<<row_grid(rows, kTurnedAtOnce), block, 0, st>>>(p, plan.splits);
      return;
    }
  if (keeps_records(plan, KV == kKvInt4 && p.dense_v)) prompt_merge_kernel<D, KV == kKvInt4, 1><<<row_grid(rows, 1), block, 0, st>>>(p, plan.splits);
}

int launch_prompt(PromptParams p, int D, bool int4, hipStream_t st) {
  const int64_t rows = p.T_q * p.n_q_heads;
  const PromptPlan plan = prompt_plan(int4, D, p.group, p.n_kv_heads, p.T_q, p.B, p.bound);
  if (row_tiles(p.T_q, p.group, plan.rows, p.B) * p.n_kv_heads * (plan.rows == 256 ? 512 : 256) > 0xffffffffLL) return SAW_EINVAL;
  if (int4) {
    // (behind the records, if there are any: rows of D + 2 floats)
    p.query_scale = p.ws + (keeps_records(plan, p.dense_v) ? ((D + 2) * rows * plan.splits + 3) / 4 * 4 : 0);
    p.query = (uint16_t*)(p.query_scale + (rows + 3) / 4 * 4);
    if (D == 128) launch_rows<128, kKvInt4>(p, plan, st);
    else launch_rows<64, kKvInt4>(p, plan, st);
  } else if (D == 128) {
    if (p.dtype == SAW_BF16) launch_rows<128, kKvBf16>(p, plan, st);
    else launch_rows<128, kKvF16>(p, plan, st);
  } else {
    if (p.dtype == SAW_BF16) launch_rows<64, kKvBf16>(p, plan, st);
    else launch_rows<64, kKvF16>(p, plan, st);
  }
  return hipGetLastError() == hipSuccess ? SAW_OK : SAW_ELAUNCH;
}

size_t prompt_bytes(int D, int Hq, int Hkv, int64_t T, int B, int64_t max_k_len) {
  const PromptPlan plan = prompt_plan(false, D, Hq / Hkv, Hkv, T, B, max_k_len);
  return 16 + (plan.splits > 1 ? record_bytes(D, T * Hq, plan.splits) : 0);
}
size_t paged_prompt_bytes(int D, int Hq, int Hkv, int64_t T, int B, int64_t max_k_len, bool dense_k, bool dense_v) {
  const PromptPlan plan = prompt_plan(true, D, Hq / Hkv, Hkv, T, B, max_k_len);
  const int64_t rows = T * Hq;
  return 32 + (keeps_records(plan, dense_v) ? record_bytes(D, rows, plan.splits) : 0) + (dense_k ? (size_t)(rows + 3) / 4 * 16 + (size_t)rows * D * 2 : 0);
}

}  // namespace saw
