// Accumulated attention weights: for every cached token the sum of its softmax weights over packed queries and the heads of a group.
//
//   x_ij = q~_i . s_j (c_j - z_j) = s_j (q~_i . (c_j - 8) - (z_j - 8) sum q~_i),   w_j = sum_i exp2(x_ij - m_i) / l_i
//
// Codes minus 8 are exact in fp16 and a rotated query is two fp16 limbs of its scaled self, so the matrix product is exact up to the sums:
// the result is an fp32 record that grows over many steps.  Keys stand in the lanes and rows in the registers, so a key's scale and
// zero-point are the lane's own, its sum over the rows needs no exchange but one at the end, and keys go from memory to operand registers
// without shared memory: a lane holds a quarter of one key's codes, and the products run over the channels in the order in which
// four instructions take the codes out of a word (0 4 1 5 2 6 3 7), which is how the query limbs are laid out.
// Two passes over the keys: maximum and sum of every row (split over the keys, joined by a small pass), then the weights.
//   32 tokens of 64 heads in each of two sequences over 12000 to 16000 keys: 52 and 44 us, 6 and 5 for queries and join.  Bound by the
// instructions of the vector ALU at two wavefronts a SIMD (14 M and 9.5 M, with 1.8 M matrix instructions in each pass); the
// keys are 19 MB.
#include "saw_prompt_tile.h"
#include "saw_rotate_row.h"

namespace saw {

constexpr int kWeightRows = 16;                 // rows of a matrix tile
constexpr int kWeightKeys = 64;                 // keys of a wavefront's step: four tiles of 16
constexpr int kGroupTiles = 16;                 // row tiles that a block of the first pass takes

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// What the passes know of a row: the scale of its limbs, the sum of its channels; then its maximum and 1 / sum.
struct RowInfo { float scale, sum_q, m, inv; };

// The workspace: operand registers of every (row tile, head), row infos, and the first pass's partial (maximum, sum) pairs.
template <int D>
struct WeightSpace {
  u32x4* limbs;             // [tile][head][limb][D / 32][64 lanes]
  RowInfo* info;            // [tile][head][16]
  float2* part;             // [chunk][tile][head][16]
  int64_t tiles;
  __host__ __device__ WeightSpace(float* ws, int64_t tiles, int heads) : tiles(tiles) {
    limbs = (u32x4*)ws;
    info = (RowInfo*)(limbs + tiles * heads * 2 * (D / 32) * 64);
    part = (float2*)(info + tiles * heads * kWeightRows);
  }
};

// One row of a tile: rotated, scaled to its largest channel in [2^14, 2^15), split into two fp16 limbs at its place among the operand
// registers; returns (2^e, sum of its channels as the limbs hold them).  By one wavefront; x: 128 floats of its own.
template <int D>
__device__ __forceinline__ f32x2 put_query_row(const PromptParams& p, int64_t token, int head, float* x, uint16_t* limbs, int r, int lane) {
  constexpr int E = D / 64;
  const int64_t src = token * p.q_stride + (int64_t)head * D;
  if (E == 1) x[lane + 64] = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) x[lane + 64 * e] = load_elem(p.q, p.dtype, src + lane + 64 * e);
  wave_sync();
  rotate_row<8>(p, x, D, lane);
  float top = 0.f, total = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(x[lane + 64 * e] * p.scale));
  top = max_xor32(max_xor16(row_allmax_positive(top)));
  const int ex = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 120) - 14;
  const float down = __uint_as_float((uint32_t)(127 - ex) << 23);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = lane + 64 * e, quarter = c / (D / 4), ks = c % (D / 4) / 8, i = 2 * (c % 4) + (c / 4) % 2;
    const float v = x[c] * p.scale * down;
    const uint16_t hi = f32_to_f16(v), lo = f32_to_f16(v - f16_to_f32(hi));
    total += f16_to_f32(hi) + f16_to_f32(lo);
    limbs[(ks * 64 + 16 * quarter + r) * 8 + i] = hi;
    limbs[((D / 32 + ks) * 64 + 16 * quarter + r) * 8 + i] = lo;
  }
  total = add_xor32(add_xor16(row_allsum(total)));
  wave_sync();
  return f32x2{__uint_as_float((uint32_t)(127 + ex) << 23), total};
}

// A row behind the last: zero.
template <int D>
__device__ __forceinline__ void put_no_row(u32x4* limbs, int r, int lane) {
  for (int i = lane; i < 2 * (D / 32) * 4; i += 64) limbs[i / 4 * 64 + 16 * (i % 4) + r] = u32x4{0, 0, 0, 0};
}

// Rotated queries of a row tile as operand registers: a wavefront a row.
template <int D>
__global__ __launch_bounds__(1024) void weight_query_kernel(PromptParams p, int64_t tiles) {
  __shared__ __attribute__((aligned(16))) float rows[kWeightRows][128];
  const int lane = threadIdx.x & 63, r = threadIdx.x >> 6, h = blockIdx.y;
  const WeightSpace<D> ws(p.ws, tiles, p.n_kv_heads);
  RowTile rt;
  if (!find_row_tile(p, blockIdx.x, kWeightRows, lane, rt)) return;
  const int64_t at = (int64_t)blockIdx.x * p.n_kv_heads + h;
  u32x4* const limbs = ws.limbs + at * 2 * (D / 32) * 64;
  f32x2 v = {1.f, 0.f};
  if (r < rt.rows) {
    const int row = rt.row0 + r;
    v = put_query_row<D>(p, rt.begin + row / p.group, h * p.group + row % p.group, rows[r], (uint16_t*)limbs, r, lane);
  } else {
    put_no_row<D>(limbs, r, lane);
  }
  if (lane == 0) ws.info[at * kWeightRows + r] = RowInfo{v.x, v.y, 0.f, 0.f};
}

// A wavefront's keys of one step as they come from memory: key 16 t + lane % 16, quarter lane / 16 of its codes.
template <int D>
struct KeyCodes {
  uint32_t w[4][D / 32];
  f32x2 pair[4];
};
template <int D>
__device__ __forceinline__ void request_keys(const PromptParams& p, TilePages& ids, int h, int lane, KeyCodes<D>& k) {
  ids.ready(p, h);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int key = 16 * t + (lane & 15);
    const uint8_t* const src = vector_codes<D>(p.k_codes, ids.at[t], key) + (lane >> 4) * (D / 8);
    if constexpr (D == 128) {
      const u32x4 x = *(const u32x4*)src;
#pragma unroll
      for (int i = 0; i < 4; ++i) k.w[t][i] = x[i];
    } else {
      const u32x2 x = *(const u32x2*)src;
#pragma unroll
      for (int i = 0; i < 2; ++i) k.w[t][i] = x[i];
    }
    k.pair[t] = *vector_pair(p.k_meta, ids.at[t], key);
  }
}
// A wavefront's steps, every `stride` keys: two of them on their way while a third is worked on, page ids one further ahead.
template <int D>
struct KeyStream {
  KeyCodes<D> codes[2];
  TilePages ids;
  const int32_t* pages;
  int end, stride, len;
  __device__ __forceinline__ void start(const PromptParams& p, int h, int key0, int lane) {
    if (key0 >= end) return;
    ids.fetch(pages, key0 / kWeightKeys, len);
    request_keys<D>(p, ids, h, lane, codes[0]);
    ids.fetch(pages, (key0 + stride) / kWeightKeys, len);
    if (key0 + stride < end) request_keys<D>(p, ids, h, lane, codes[1]);
    ids.fetch(pages, (key0 + 2 * stride) / kWeightKeys, len);
  }
  // behind the use of a slot at key0: what comes two steps later
  __device__ __forceinline__ void next(const PromptParams& p, int h, int key0, int lane, KeyCodes<D>& slot) {
    if (key0 + 2 * stride >= end) return;
    request_keys<D>(p, ids, h, lane, slot);
    ids.fetch(pages, (key0 + 3 * stride) / kWeightKeys, len);
  }
  template <typename F>
  __device__ __forceinline__ void each(int key0, F step) {
    while (key0 < end) {
      step(key0, codes[0]);
      key0 += stride;
      if (key0 >= end) break;
      step(key0, codes[1]);
      key0 += stride;
    }
  }
};

// A row tile in a wavefront's registers.
template <int D>
struct TileQueries {
  u32x4 q[2][D / 32];
  f32x4 info[4];                  // of rows 4 (lane / 16) + 0..3
  float sum_q[4];
  __device__ __forceinline__ u32x4 limb(int l, int ks) const { return q[l][ks]; }
  __device__ __forceinline__ void load(const u32x4* limbs, const RowInfo* info, int lane) {
#pragma unroll
    for (int l = 0; l < 2; ++l)
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) q[l][ks] = limbs[(l * (D / 32) + ks) * 64 + lane];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      this->info[r] = *(const f32x4*)&info[4 * (lane >> 4) + r];
      sum_q[r] = this->info[r].y;
    }
  }
};

// ... and one in shared memory, from where its limbs are read again for every 16 keys: registers for four wavefronts a SIMD.
template <int D>
struct SharedQueries {
  const u32x4* limbs;             // (the lane's)
  float scale[4], sum_q[4];
  __device__ __forceinline__ u32x4 limb(int l, int ks) const { return limbs[(l * (D / 32) + ks) * 64]; }
};

// 16 of a step's keys as operand registers; the pair of a slot behind the end, which may hold anything, becomes zero.
template <int D>
__device__ __forceinline__ f32x2 key_codes(const KeyCodes<D>& codes, CodeBits bits, int t, int key0, int len, int lane, u32x4 (&k)[D / 32]) {
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) k[ks] = centred(codes.w[t][ks], bits);
  return key0 + 16 * t + (lane & 15) < len ? codes.pair[t] : f32x2{0.f, 0.f};
}

// Logits of 16 rows and N times 16 keys, in log2 units divided by the rows' scales: of row 4 (lane / 16) + r and the lane's keys.  The sums
// of the 16 keys, or of one's limbs, alternate: a product would wait for the sum of the one before it.
template <int D, int N, typename Q>
__device__ __forceinline__ void tile_logits16(const Q& tq, const u32x4 (&k)[N][D / 32], const f32x2 (&pair)[N], f32x4 (&x)[N]) {
  constexpr int kLimbSums = N == 1 ? 2 : 1;
  f32x4 s[N][kLimbSums];
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int l = 0; l < kLimbSums; ++l) s[t][l] = f32x4{0.f, 0.f, 0.f, 0.f};
  if constexpr (N == 1) {
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
      for (int l = 1; l >= 0; --l) s[0][l] = mfma16(tq.limb(l, ks), k[0][ks], s[0][l]);
    s[0][0] += s[0][1];
  } else {
#pragma unroll
    for (int l = 1; l >= 0; --l)
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
        for (int t = 0; t < N; ++t) s[t][0] = mfma16(tq.limb(l, ks), k[t][ks], s[t][0]);
  }
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const float z8 = pair[t].y - 8.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[t][r] = fmaf(-z8, tq.sum_q[r], s[t][0][r]) * pair[t].x;
  }
}
// Hidden ones and those behind the sequence's end become -infinity.  (Row i sees the keys in front of first_hidden + its token.)
__device__ __forceinline__ void hide(f32x4& x, int key, int len, int first_hidden, int shift, int row0, int lane) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (key >= min(len, first_hidden + ((row0 + 4 * (lane >> 4) + r) >> shift))) x[r] = -INFINITY;
}

// Maximum and sum over rows of 16 lanes of four numbers at once: a step's operands are four instructions old, as far as DPP asks for.
#define ROW_STEP4(op, how)                                                                                                         \
  op " %0, %0, %0 " how " row_mask:0xf bank_mask:0xf\n\t" op " %1, %1, %1 " how " row_mask:0xf bank_mask:0xf\n\t"              \
  op " %2, %2, %2 " how " row_mask:0xf bank_mask:0xf\n\t" op " %3, %3, %3 " how " row_mask:0xf bank_mask:0xf\n\t"
#define ROW_ALL4(op) "s_nop 1\n\t" ROW_STEP4(op, "row_ror:1") ROW_STEP4(op, "row_ror:2") ROW_STEP4(op, "row_ror:4") ROW_STEP4(op, "row_ror:8")
__device__ __forceinline__ void row_allmax4(float (&v)[4]) { asm(ROW_ALL4("v_max_f32_dpp") : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3])); }
__device__ __forceinline__ void row_allsum4(float (&v)[4]) { asm(ROW_ALL4("v_add_f32_dpp") : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3])); }

// One pass over a chunk of the keys of a (sequence, kv head).  STATS: maximum and sum of each row of a group of row tiles over the
// chunk; otherwise the weights of the chunk's keys over all rows.  The wavefronts of a block share out the chunk's keys, or, SHARE_ROWS, the row
// tiles, and then add up their weights.
template <int D, bool STATS, bool SHARE_ROWS>
__global__ __launch_bounds__(256, 2) void weight_pass_kernel(PromptParams p, int64_t tiles, int chunk_keys, bool search) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % p.n_kv_heads, chunk = blockIdx.x / p.n_kv_heads;
  const WeightSpace<D> ws(p.ws, tiles, p.n_kv_heads);
  RowTile group;                // (STATS) of the batch's groups of row tiles, or number blockIdx.z of sequence blockIdx.y
  if (STATS && search && !find_row_tile(p, (int64_t)blockIdx.z * gridDim.y + blockIdx.y, kGroupTiles * kWeightRows, lane, group)) return;
  const int b = STATS && search ? group.b : (int)blockIdx.y;
  const int len = min(max(p.seq_lens[b], 0), p.bound);
  int begin, n;
  packed_range(p.cu_q, b, p.T_q, begin, n);
  const int64_t first_tile = (int64_t)begin * p.group / kWeightRows + b;
  const int shift = __builtin_ctz(p.group), first_hidden = len - n + 1;
  const int64_t rows = (int64_t)n * p.group;
  const int all = (int)((rows + kWeightRows - 1) / kWeightRows);
  const int g0 = !STATS ? 0 : search ? group.row0 / kWeightRows : (int)blockIdx.z * kGroupTiles, g1 = STATS ? min(all, g0 + kGroupTiles) : all;
  const int k0 = chunk * chunk_keys, k1 = min(len, k0 + chunk_keys);
  if (STATS && g0 >= g1) return;
  __shared__ float2 stats[4][STATS ? kGroupTiles * kWeightRows : 1];
  __shared__ float sums[4][STATS || !SHARE_ROWS ? 1 : kWeightKeys];
  if (STATS) {
    for (int r = lane; r < (g1 - g0) * kWeightRows; r += 64) stats[wave][r] = make_float2(-INFINITY, 0.f);
    wave_sync();
  }
  const int64_t record = ((int64_t)b * p.n_kv_heads + h) * p.score_stride;
  const CodeBits bits;
  TileQueries<D> tq;
  int held = -1;                // the row tile in tq: a single one is loaded once
  auto load_tile = [&](int g) {
    const int64_t at = (first_tile + g) * p.n_kv_heads + h;
    tq.load(ws.limbs + at * 2 * (D / 32) * 64, ws.info + at * kWeightRows, lane);
    held = g;
  };
  KeyStream<D> keys;
  keys.pages = p.page_table + (int64_t)b * p.max_pages;
  keys.end = k1; keys.stride = SHARE_ROWS ? kWeightKeys : 4 * kWeightKeys; keys.len = len;
  constexpr int kTileStep = SHARE_ROWS ? 4 : 1;
  const int start = SHARE_ROWS ? k0 : k0 + kWeightKeys * wave;
  keys.start(p, h, start, lane);
  keys.each(start, [&](int key0, KeyCodes<D>& codes) {
    u32x4 k[4][D / 32];
    f32x2 pair[4];
    float total[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 4; ++t) pair[t] = key_codes<D>(codes, bits, t, key0, len, lane, k[t]);
    // (rows behind the last are zeros, and zero times an infinite scale is no number)
    bool odd_scale = false;
    if (!STATS && rows % kWeightRows)
      odd_scale = __any(!(fmaxf(fmaxf(fabsf(pair[0].x), fabsf(pair[1].x)), fmaxf(fabsf(pair[2].x), fabsf(pair[3].x))) < INFINITY));
    keys.next(p, h, key0, lane, codes);
    // the first row that sees a key of the step: key0 < first_hidden + token
    const int first_token = max(key0 - first_hidden + 1, 0);
    for (int g = max(g0, (int)(((int64_t)first_token << shift) / kWeightRows)) + (SHARE_ROWS ? wave : 0); g < g1; g += kTileStep) {
      const int row0 = g * kWeightRows;
      const bool masked = key0 + kWeightKeys > min(first_hidden + (row0 >> shift), len);
      f32x4 x[4];
      if (g != held) load_tile(g);
      tile_logits16<D>(tq, k, pair, x);
      if (masked)
#pragma unroll
        for (int t = 0; t < 4; ++t) hide(x[t], key0 + 16 * t + (lane & 15), len, first_hidden, shift, row0, lane);
      if (odd_scale && g == all - 1)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (row0 + 4 * (lane >> 4) + r >= rows) x[t][r] = -INFINITY;
      f32x4 info[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) info[r] = tq.info[r];
      // (The next tile's queries arrive behind the exponentials: 32 tokens of 64 heads over 16000 keys 103 us, 111 without.  With 64
      // channels the registers for it cost a wavefront a SIMD: 86 us, 75 without.)
      if (D == 128 && g + kTileStep < g1) load_tile(g + kTileStep);
      if constexpr (STATS) {
        float2* const mine = &stats[wave][(g - g0) * kWeightRows + 4 * (lane >> 4)];
        float top[4], sum[4], m[4], old[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) top[r] = fmaxf(fmaxf(x[0][r], x[1][r]), fmaxf(x[2][r], x[3][r]));
        row_allmax4(top);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float2 was = mine[r];
          m[r] = fmaxf(was.x, top[r] * info[r].x);
          const float ref = m[r] == -INFINITY ? 0.f : m[r];
          sum[r] = (fast_exp2(fmaf(x[0][r], info[r].x, -ref)) + fast_exp2(fmaf(x[1][r], info[r].x, -ref))) +
                   (fast_exp2(fmaf(x[2][r], info[r].x, -ref)) + fast_exp2(fmaf(x[3][r], info[r].x, -ref)));
          old[r] = was.y * fast_exp2(was.x - ref);
        }
        row_allsum4(sum);
        wave_sync();
        if ((lane & 15) == 0)
#pragma unroll
          for (int r = 0; r < 4; ++r) mine[r] = make_float2(m[r], old[r] + sum[r]);
        wave_sync();
      } else {
        f32x2 mi[4];
        bool none = false;                                                 // (a row whose sum is no number: nor is any of its weights,
#pragma unroll
        for (int r = 0; r < 4; ++r) {                                      // but for those of the keys that it does not see)
          mi[r] = f32x2{info[r].z, info[r].w};
          none = none || mi[r].y != mi[r].y;
        }
        if (masked && __any(none))
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (mi[r].y != mi[r].y) {
              const int end = min(len, first_hidden + ((row0 + 4 * (lane >> 4) + r) >> shift));
#pragma unroll
              for (int t = 0; t < 4; ++t)
                if (key0 + 16 * t + (lane & 15) < end) total[t] = mi[r].y;
              mi[r].y = 0.f;
            }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int t = 0; t < 4; ++t) total[t] = fmaf(fast_exp2(fmaf(x[t][r], info[r].x, -mi[r].x)), mi[r].y, total[t]);
      }
    }
    if constexpr (!STATS) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float w = add_xor32(add_xor16(total[t]));
        const int key = key0 + 16 * t + lane;
        if (SHARE_ROWS) {
          if (lane < 16) sums[wave][16 * t + lane] = w;
        } else if (lane < 16 && key < len) {
          p.scores[record + key] = (p.prev ? p.prev[record + key] : 0.f) + w;
        }
      }
      if (SHARE_ROWS) {                                                    // (all wavefronts are at the same keys)
        __syncthreads();
        const int key = key0 + lane;
        if (wave == 0 && key < len)
          p.scores[record + key] = (p.prev ? p.prev[record + key] : 0.f) + ((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
        __syncthreads();
      }
    }
  });
  if constexpr (STATS) {
    __syncthreads();
    for (int r = threadIdx.x; r < (g1 - g0) * kWeightRows; r += 256) {
      const float2 a = stats[0][r], c = stats[1][r], d = stats[2][r], e = stats[3][r];
      const float m = fmaxf(fmaxf(a.x, c.x), fmaxf(d.x, e.x)), ref = m == -INFINITY ? 0.f : m;
      const float sum = (a.y * fast_exp2(a.x - ref) + c.y * fast_exp2(c.x - ref)) + (d.y * fast_exp2(d.x - ref) + e.y * fast_exp2(e.x - ref));
      const int64_t at = (first_tile + g0 + r / kWeightRows) * p.n_kv_heads + h;
      ws.part[((int64_t)chunk * tiles * p.n_kv_heads + at) * kWeightRows + r % kWeightRows] = make_float2(m, sum);
    }
  }
}

// Joins the partial (maximum, sum) pairs of a row tile and head: a lane for every sixteenth of the chunks of a row.
template <int D>
__global__ __launch_bounds__(256) void weight_join_kernel(PromptParams p, int64_t tiles, int chunks) {
  constexpr int kAhead = 4;                                               // pairs on their way at once
  __shared__ float2 part[4][kWeightRows];
  const WeightSpace<D> ws(p.ws, tiles, p.n_kv_heads);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15;
  RowTile rt;
  if (!find_row_tile(p, blockIdx.x, kWeightRows, lane, rt)) return;
  const int64_t at = ((int64_t)blockIdx.x * p.n_kv_heads + blockIdx.y) * kWeightRows + r, step = tiles * p.n_kv_heads * kWeightRows;
  float m = -INFINITY, sum = 0.f;
  for (int c0 = threadIdx.x >> 4; c0 < chunks; c0 += 16 * kAhead) {
    float2 v[kAhead];
    float top = m;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = c0 + 16 * k < chunks ? ws.part[(c0 + 16 * k) * step + at] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) top = fmaxf(top, v[k].x);
    const float ref = top == -INFINITY ? 0.f : top;
    sum *= fast_exp2(m - ref);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) sum = fmaf(v[k].y, fast_exp2(v[k].x - ref), sum);
    m = top;
  }
  const float here = max_xor32(max_xor16(m)), ref = here == -INFINITY ? 0.f : here;
  sum = add_xor32(add_xor16(sum * fast_exp2(m - ref)));
  if (lane < 16) part[wave][r] = make_float2(here, sum);
  __syncthreads();
  if (threadIdx.x >= 16) return;
  const float top = fmaxf(fmaxf(part[0][r].x, part[1][r].x), fmaxf(part[2][r].x, part[3][r].x)), all_ref = top == -INFINITY ? 0.f : top;
  float all = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) all = fmaf(part[w][r].y, fast_exp2(part[w][r].x - all_ref), all);
  ws.info[at].m = all_ref;
  ws.info[at].inv = all == 0.f || r >= rt.rows ? 0.f : 1.f / all;
}

// Statistics and weights in one launch, for batches of few rows a sequence that fill the chip by themselves (a decode step): a block takes
// a (sequence, kv head), reads its keys once and keeps the logits in shared memory while they fit; longer ones are worked out again.
// Sequences of more rows take a row tile after the other, the later ones on top of what the earlier wrote.  What bounds it is how many
// wavefronts a SIMD has to cover one another's waits: four of them, 128 registers each, which is why a step works on 16 keys at a time
// (64 sequences of 512 to 4096 tokens, 95 MB, 52 us; two passes 132).
constexpr int kKeptLogits = 16384, kStepWaves = 8;

template <int D>
__global__ __launch_bounds__(64 * kStepWaves, 4) void weight_step_kernel(PromptParams p) {
  __shared__ __attribute__((aligned(16))) float kept[kKeptLogits];
  __shared__ u32x4 limbs[2 * (D / 32) * 64];
  __shared__ RowInfo info[kWeightRows];
  __shared__ float2 stats[kStepWaves][kWeightRows];
  constexpr int kThreads = 64 * kStepWaves, kStride = kWeightKeys * kStepWaves;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x, b = blockIdx.y;
  const int len = min(max(p.seq_lens[b], 0), p.bound);
  int begin, n;
  packed_range(p.cu_q, b, p.T_q, begin, n);
  const int shift = __builtin_ctz(p.group), first_hidden = len - n + 1;
  const int rows = n << shift;
  const int64_t record = ((int64_t)b * p.n_kv_heads + h) * p.score_stride;
  const float* prev = p.prev;
  const int32_t* const pages = p.page_table + (int64_t)b * p.max_pages;
  if (rows == 0)
    for (int j = threadIdx.x; j < len; j += kThreads) p.scores[record + j] = prev ? prev[record + j] : 0.f;
  if (len == 0) return;
  for (int row0 = 0; row0 < rows; row0 += kWeightRows) {
    const int here = min(kWeightRows, rows - row0), start = kWeightKeys * wave;
    KeyCodes<D> codes;
    TilePages ids;
    auto first = [&] {
      if (start >= len) return;
      ids.fetch(pages, start / kWeightKeys, len);
      request_keys<D>(p, ids, h, lane, codes);
      ids.fetch(pages, (start + kStride) / kWeightKeys, len);
    };
    first();
    for (int r = wave; r < kWeightRows; r += kStepWaves) {
      if (r < here) {
        const int row = row0 + r;
        // (a wavefront's row is turned over in its part of the logits' memory)
        const f32x2 v = put_query_row<D>(p, begin + (row >> shift), h * p.group + (row & (p.group - 1)), kept + 128 * wave, (uint16_t*)limbs, r, lane);
        if (lane == 0) info[r] = RowInfo{v.x, v.y, 0.f, 0.f};
      } else {
        put_no_row<D>(limbs, r, lane);
        if (lane == 0) info[r] = RowInfo{1.f, 0.f, 0.f, 0.f};
      }
    }
    __syncthreads();
    SharedQueries<D> tq;
    tq.limbs = limbs + lane;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      tq.scale[r] = info[4 * (lane >> 4) + r].scale;
      tq.sum_q[r] = info[4 * (lane >> 4) + r].sum_q;
    }
    const bool keep = (int64_t)here * len <= kKeptLogits;
    const CodeBits bits;
    // every step's logits, by rows 4 (lane / 16) + r and keys 16 t + lane % 16
    auto steps = [&](auto use) {
      for (int key0 = start; key0 < len; key0 += kStride) {
        const bool masked = key0 + kWeightKeys > min(first_hidden + (row0 >> shift), len);
        f32x4 x[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          u32x4 k[1][D / 32];
          const f32x2 pair[1] = {key_codes<D>(codes, bits, t, key0, len, lane, k[0])};
          f32x4 of[1];
          tile_logits16<D>(tq, k, pair, of);
          x[t] = of[0];
#pragma unroll
          for (int r = 0; r < 4; ++r) x[t][r] *= tq.scale[r];
          if (masked) hide(x[t], key0 + 16 * t + (lane & 15), len, first_hidden, shift, row0, lane);
          asm volatile("" ::: "memory");                                   // (or the limbs would be kept in registers after all)
        }
        if (key0 + kStride < len) {
          request_keys<D>(p, ids, h, lane, codes);
          ids.fetch(pages, (key0 + 2 * kStride) / kWeightKeys, len);
        }
        use(key0, x);
      }
    };
    float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (keep) {
      steps([&](int key0, const f32x4 (&x)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          m[r] = fmaxf(fmaxf(m[r], fmaxf(x[0][r], x[1][r])), fmaxf(x[2][r], x[3][r]));
          if (4 * (lane >> 4) + r < here) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const int key = key0 + 16 * t + (lane & 15);
              if (key < len) kept[(4 * (lane >> 4) + r) * len + key] = x[t][r];
            }
          }
        }
      });
    } else {
      steps([&](int, const f32x4 (&x)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float top = fmaxf(fmaxf(m[r], fmaxf(x[0][r], x[1][r])), fmaxf(x[2][r], x[3][r])), ref = top == -INFINITY ? 0.f : top;
          sum[r] = fmaf(sum[r], fast_exp2(m[r] - ref), (fast_exp2(x[0][r] - ref) + fast_exp2(x[1][r] - ref)) + (fast_exp2(x[2][r] - ref) + fast_exp2(x[3][r] - ref)));
          m[r] = top;
        }
      });
    }
    // rows' maxima, and sums so far, over all lanes and wavefronts
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float top = row_allmax(m[r]), part = row_allsum(sum[r] * fast_exp2(m[r] - (top == -INFINITY ? 0.f : top)));
      if ((lane & 15) == 0) stats[wave][4 * (lane >> 4) + r] = make_float2(top, part);
    }
    __syncthreads();
    if (threadIdx.x < kWeightRows) {
      float top = -INFINITY, all = 0.f;
#pragma unroll
      for (int w = 0; w < kStepWaves; ++w) top = fmaxf(top, stats[w][threadIdx.x].x);
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < kStepWaves; ++w) all += stats[w][threadIdx.x].y * fast_exp2(stats[w][threadIdx.x].x - ref);
      info[threadIdx.x].m = ref;
      info[threadIdx.x].inv = all == 0.f ? 0.f : 1.f / all;
    }
    __syncthreads();
    if (keep) {
      // weights in the logits' places and their sums, a row after the other
      for (int r = 0; r < here; ++r) {
        float part = 0.f;
        const float ref = info[r].m;
        for (int j = threadIdx.x; j < len; j += kThreads) {
          const float w = fast_exp2(kept[r * len + j] - ref);
          kept[r * len + j] = w;
          part += w;
        }
        part = add_xor32(add_xor16(row_allsum(part)));
        if (lane == 0) stats[wave][r].y = part;
      }
      __syncthreads();
      if ((int)threadIdx.x < here) {
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < kStepWaves; ++w) all += stats[w][threadIdx.x].y;
        info[threadIdx.x].inv = all == 0.f ? 0.f : all == all ? 1.f / all : 1.f;
        if (all != all) info[threadIdx.x].m = all;
      }
      __syncthreads();
      // (weights of a row whose sum is no number, as above)
      for (int r = 0; r < here; ++r)
        if (info[r].m != info[r].m)
          for (int j = threadIdx.x; j < min(len, first_hidden + ((row0 + r) >> shift)); j += kThreads) kept[r * len + j] = info[r].m;
      for (int j = threadIdx.x; j < len; j += kThreads) {
        float w = 0.f;
        for (int r = 0; r < here; ++r) w = fmaf(kept[r * len + j], info[r].inv, w);
        p.scores[record + j] = (prev ? prev[record + j] : 0.f) + w;
      }
    } else {
      first();
      int end[4];                                                          // positions that the rows see, also those whose logit is -infinity
#pragma unroll
      for (int r = 0; r < 4; ++r) end[r] = min(len, first_hidden + ((row0 + 4 * (lane >> 4) + r) >> shift));
      steps([&](int key0, const f32x4 (&x)[4]) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float w = 0.f;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * (lane >> 4) + r < here && key0 + 16 * t + (lane & 15) < end[r])
              w = fmaf(fast_exp2(x[t][r] - info[4 * (lane >> 4) + r].m), info[4 * (lane >> 4) + r].inv, w);
          w = add_xor32(add_xor16(w));
          const int key = key0 + 16 * t + lane;
          if (lane < 16 && key < len) p.scores[record + key] = (prev ? prev[record + key] : 0.f) + w;
        }
      });
    }
    prev = p.scores;
    __syncthreads();
  }
}

// How the passes are handed out: chunks of the keys, and what a block's wavefronts share out.  Its keys, 256 at a time, so that codes are turned
// into operands once; its row tiles where a sequence has four and more and there are few blocks of 256 keys (sharing keys and rows: 10 x 131
// tokens of 32 heads over 135 keys 89 us and 50, 24 x 60 over 74 89 and 61, 2 x 100 over 304 59 and 28, 1 x 185 over 3700 35 and 25; but 3 x
// 200 of 64 heads over 3800, 480 blocks, 174 and 184, 8 x 210 over 15000 214 and 258).
struct WeightPlan { int chunks, chunk_keys; bool share_rows; };
static WeightPlan weight_plan(int G, int Hkv, int64_t T, int B, int64_t bound) {
  const int64_t items = (int64_t)B * Hkv, tiles = T * G / ((int64_t)B * kWeightRows), wide = 4 * kWeightKeys;
  const bool share_rows = tiles >= 4 && items * ((bound + wide - 1) / wide) <= 256;
  const int64_t unit = share_rows ? kWeightKeys : wide, most = (bound + unit - 1) / unit;
  int64_t s = 2048 / items;
  if (s > most) s = most;
  if (s > 256) s = 256;
  if (s < 1) s = 1;
  return {(int)s, (int)(((bound + s - 1) / s + unit - 1) / unit * unit), share_rows};
}

size_t weights_bytes(int D, int Hq, int Hkv, int64_t T, int B, int64_t bound) {
  const int64_t tiles = row_tiles(T, Hq / Hkv, kWeightRows, B);
  const WeightPlan plan = weight_plan(Hq / Hkv, Hkv, T, B, bound);
  return 16 + (size_t)tiles * Hkv * (2 * (D / 32) * 64 * 16 + kWeightRows * (sizeof(RowInfo) + (size_t)plan.chunks * 8));
}

template <int D, bool SHARE_ROWS>
static void launch_passes(const PromptParams& p, int64_t tiles, const WeightPlan& plan, hipStream_t st) {
  const int wide = p.n_kv_heads * plan.chunks;
  if (p.T_q) {
    weight_query_kernel<D><<<dim3((unsigned)tiles, p.n_kv_heads), dim3(1024), 0, st>>>(p, tiles);
    // Which groups of row tiles a sequence has is known on the device alone.  As many blocks for each sequence as the whole batch has groups,
    // while that is few blocks, an empty one 0.4 ns; otherwise the blocks search for their sequence, some 4 us (10 x 131 tokens of 32 heads over 135
    // keys 52.6 us and 55, 24 x 60 over 75, 9216 blocks, 52.5 and 57.4; 64 x 200 over 3000 1965 and 1842, 1024 x 16 over 40 1720 and 649).
    const int64_t each = (tiles + kGroupTiles - 1) / kGroupTiles, groups = row_tiles(p.T_q, p.group, kGroupTiles * kWeightRows, p.B);
    const bool search = each * p.B * wide > 16384;
    const int64_t high = search ? (groups < 32768 ? groups : 32768) : p.B, deep = search ? (groups + high - 1) / high : each;
    weight_pass_kernel<D, true, SHARE_ROWS><<<dim3(wide, (unsigned)high, (unsigned)deep), dim3(256), 0, st>>>(p, tiles, plan.chunk_keys, search);
    weight_join_kernel<D><<<dim3((unsigned)tiles, p.n_kv_heads), dim3(256), 0, st>>>(p, tiles, plan.chunks);
  }
  weight_pass_kernel<D, false, SHARE_ROWS><<<dim3(wide, p.B), dim3(256), 0, st>>>(p, tiles, plan.chunk_keys, false);
}

// One launch where a sequence has about one query: short contexts, whose four launches take longer than a block of one compute unit for each
// (sequence, kv head) (8 kv heads; one launch and two passes: 1 x 1000 tokens 13.7 us and 15.5, 8 x 1000 14.2 and 16.4; 1 x 2000 19.1 and
// 15.5), or batches that fill the chip, the sooner if the logits fit shared memory (16 x 4000 35 and 44.6, 8 x 4000 33 and 27; 64 of 4000 to
// 10000, which do not, 201 and 250, 24 of 1000 to 8000 102 and 66).  Several queries a sequence are level at best (32 x 5 over 1000 tokens
// 36.5 and 37, 8 x 5 31 and 20).
static bool one_launch(const PromptParams& p) {
  const int64_t items = (int64_t)p.B * p.n_kv_heads;
  if (p.T_q > p.B) return false;
  return (int64_t)p.bound * p.group <= kKeptLogits ? items >= 128 || p.bound <= 1280 : items >= 256;
}

int launch_weights(const PromptParams& p, int D, hipStream_t st) {
  const int64_t tiles = row_tiles(p.T_q, p.group, kWeightRows, p.B);
  const WeightPlan plan = weight_plan(p.group, p.n_kv_heads, p.T_q, p.B, p.bound);
  // (grids: widths below 2^32 threads, groups of tiles below 2^16)
  if ((int64_t)p.n_kv_heads * plan.chunks * 256 > 0xffffffffLL || (tiles + kGroupTiles - 1) / kGroupTiles > 65535) return SAW_EINVAL;
  if (one_launch(p)) {
    const dim3 grid(p.n_kv_heads, p.B);
    if (D == 128) weight_step_kernel<128><<<grid, dim3(64 * kStepWaves), 0, st>>>(p);
    else weight_step_kernel<64><<<grid, dim3(64 * kStepWaves), 0, st>>>(p);
    return hipGetLastError() == hipSuccess ? SAW_OK : SAW_ELAUNCH;
  }
  if (D == 128) plan.share_rows ? launch_passes<128, true>(p, tiles, plan, st) : launch_passes<128, false>(p, tiles, plan, st);
  else plan.share_rows ? launch_passes<64, true>(p, tiles, plan, st) : launch_passes<64, false>(p, tiles, plan, st);
  return hipGetLastError() == hipSuccess ? SAW_OK : SAW_ELAUNCH;
}

}  // namespace saw
