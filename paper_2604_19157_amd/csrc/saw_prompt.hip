// Attention of packed queries: softmax(q K^T s) V with K and V of 16 bits or read from the INT4 pages.
#include "saw_prompt_tile.h"

namespace saw {

enum { kKvBf16, kKvF16, kKvInt4 };

// Channels of one vector that a lane holds: lane, lane + 64.
template <int D, int KV>
struct RowSource {
  const PromptParams& p;
  int b, h, k0, lane;
  __device__ void load(bool value, int j, float (&x)[D / 64]) const {
    if constexpr (KV == kKvInt4) {
      int page = p.page_table[(int64_t)b * p.max_pages + (j >> 4)];
      if (page < 0 || page >= p.num_pages) page = 0;
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

// q R and o R^T of one row in LDS (128 floats; of 64 channels the first half)
__device__ void rotate_row(const PromptParams& p, float* x, int D, int lane) {
  if (p.rot_k) {
    if (p.has_signs)
      for (int c = lane; c < D; c += 64) x[c] = apply_sign(p.signs, c, x[c]);
    wave_sync();
    wave_lds_fwht128<1>(x, p.had_block, lane);
    for (int c = lane; c < D; c += 64) x[c] *= had_norm(p.had_block);
    wave_sync();
  }
  if (p.dense_k) wave_lds_matvec128<1>(x, p.dense, lane);
}
__device__ void unrotate_row(const PromptParams& p, float* x, int D, int lane) {
  if (p.dense_v) wave_lds_matvec128<1>(x, p.dense + kDenseD * kDenseD, lane);
  if (p.rot_v) {
    wave_lds_fwht128<1>(x, p.had_block, lane);
    for (int c = lane; c < D; c += 64) x[c] = apply_sign(p.signs, c, x[c] * had_norm(p.had_block));
    wave_sync();
  }
}

template <typename M>
__device__ __forceinline__ float widen(uint16_t x);
template <> __device__ __forceinline__ float widen<MathBf16>(uint16_t x) { return bf16_to_f32(x); }
template <> __device__ __forceinline__ float widen<MathF16>(uint16_t x) { return f16_to_f32(x); }

// ---------------------------------------------------------------------------------------------------------------------------------
// Prompt attention over 16-bit keys and values.
// A block takes 32 rows per wavefront and goes over the keys in tiles of 64, which come from memory straight into a double buffer in
// shared memory (each transfer has a whole tile's products to arrive in); one barrier a tile.
template <int D, typename M, int NW>
__global__ __launch_bounds__(64 * NW, 2) void prompt_kernel(PromptParams p) {
  constexpr int R = 32 * NW, kRow = 2 * D, kTile = kTileKeys * kRow, kInstr = kTile / 1024, kRpi = 1024 / kRow;
  __shared__ __attribute__((aligned(1024))) char lds[2][2][kTile];       // [buffer][K, V]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % p.n_kv_heads;
  // (the last tiles of a causal sequence have the most keys and start first)
  const int64_t tile = (int64_t)gridDim.x / p.n_kv_heads - 1 - blockIdx.x / p.n_kv_heads;
  RowTile rt;
  if (!find_row_tile(p, tile, R, lane, rt)) return;
  int k0, len;
  packed_range(p.cu_k, rt.b, p.T_k, k0, len);
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
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    qf[ks] = *(const u32x4*)((const uint16_t*)p.q + token * p.q_stride + (int64_t)head * D + 16 * ks + 8 * (lane >> 5));
  RowState<D> st;
  st.m = -INFINITY; st.ref = 0.f; st.sum = 0.f;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.o[t][r] = 0.f;

  const uint16_t* const kp = (const uint16_t*)p.k + (int64_t)k0 * p.k_stride + (int64_t)h * D;
  const uint16_t* const vp = (const uint16_t*)p.v + (int64_t)k0 * p.v_stride + (int64_t)h * D;
  auto load = [&](int buf, int t) {
#pragma unroll
    for (int j = 0; j < kInstr / NW; ++j) {
      const int in = wave * (kInstr / NW) + j;                             // 1024 bytes: kRpi rows
      const int r = in * kRpi + lane / (D / 8), place = lane % (D / 8);
      const int64_t key = min(t * kTileKeys + r, len - 1);                 // (behind the end: the last key again, masked)
      __builtin_amdgcn_global_load_lds((const GLOBAL_AS void*)(kp + key * p.k_stride + 8 * k_place(r, place)), (LDS_AS void*)(lds[buf][0] + in * 1024), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const GLOBAL_AS void*)(vp + key * p.v_stride + 8 * v_place(r, place)), (LDS_AS void*)(lds[buf][1] + in * 1024), 16, 0, 0);
    }
  };
  if (t0 < t1) load(0, t0);
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    __builtin_amdgcn_s_waitcnt(0x0F70);                                   // vmcnt(0): this wavefront's part of tile t is there
    lds_barrier();                                                        // ... everybody's is, and nobody reads the other buffer any more
    if (t + 1 < t1) load(buf ^ 1, t + 1);
    if (t * kTileKeys < wend) {
      f32x16 s[2];
      u32x4 pf[4];
      tile_logits<D, M>(lds[buf][0], qf, s, lane);
      if ((t + 1) * kTileKeys > wfull) tile_mask(s, sees - t * kTileKeys, lane);
      tile_weights<D, M>(s, p.scale, st, pf);
      tile_values<D, M>(lds[buf][1], pf, st, lane);
    }
  }
  const float sum = add_xor32(st.sum);
  // Values that are no numbers: a masked key's weight is zero, but zero times infinity is not.  Rows of a wavefront that ended with one
  // are taken again, key by key, over the keys that each sees.
  float odd = 0.f;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd = fmaf(st.o[t][r], 0.f, odd);
  const bool split = gridDim.y > 1;
  float* const records = p.ws + (int64_t)blockIdx.y * p.T_q * p.n_q_heads * D;
  float2* const ml = (float2*)(p.ws + (int64_t)gridDim.y * p.T_q * p.n_q_heads * D) + (int64_t)blockIdx.y * p.T_q * p.n_q_heads;
  if (__any(odd != odd)) {
    constexpr int E = D / 64;
    for (int i = 0; i < 32 && w0 + i <= last; ++i) {
      const int64_t tok = rt.begin + ((w0 + i) >> shift);
      const int hd = h * p.group + ((w0 + i) & (p.group - 1));
      const int end = min(sees_of(w0 + i), t1 * kTileKeys);
      float q[E], acc[E], m = -INFINITY, den = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        q[e] = widen<M>(((const uint16_t*)p.q)[tok * p.q_stride + (int64_t)hd * D + lane + 64 * e]) * p.scale;
        acc[e] = 0.f;
      }
      for (int j = t0 * kTileKeys; j < end; ++j) {
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x = fmaf(q[e], widen<M>(kp[j * p.k_stride + lane + 64 * e]), x);
        x = add_xor32(add_xor16(row_allsum(x)));
        const float top = fmaxf(m, x), ref = top == -INFINITY ? 0.f : top;
        const float alpha = fast_exp2(m - ref), w = fast_exp2(x - ref);
        m = top;
        den = fmaf(den, alpha, w);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(acc[e], alpha, w * widen<M>(vp[j * p.v_stride + lane + 64 * e]));
      }
      const int64_t at = tok * p.n_q_heads + hd;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (split) records[at * D + lane + 64 * e] = acc[e];
        else store_elem(p.out, p.dtype, at * D + lane + 64 * e, den == 0.f ? 0.f : acc[e] / den);
      }
      if (split && lane == 0) ml[at] = make_float2(m, den);
    }
    return;
  }
  if (row > last) return;
  const int64_t at = token * p.n_q_heads + head;
  if (split) {
    if (lane < 32) ml[at] = make_float2(st.m, sum);
    if (sum != 0.f)
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *(f32x4*)(records + at * D + 32 * t + 2 * r + 4 * (lane >> 5)) = f32x4{st.o[t][r], st.o[t][r + 1], st.o[t][r + 2], st.o[t][r + 3]};
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *(u32x2*)((uint16_t*)p.out + at * D + 32 * t + 2 * r + 4 * (lane >> 5)) =
          u32x2{M::pack(st.o[t][r] * inv, st.o[t][r + 1] * inv), M::pack(st.o[t][r + 2] * inv, st.o[t][r + 3] * inv)};
}

// Joins the partial records of a row: one wavefront a row.
template <int D>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptParams p, int splits) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rows = p.T_q * p.n_q_heads, row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= rows) return;
  const int64_t token = row / p.n_q_heads;
  const int b = last_not_above(p.B, token, lane, [&](int i) { return clamped_offset(p.cu_q, i, p.T_q); });
  if (b < 0 || token >= clamped_offset(p.cu_q, b + 1, p.T_q)) return;
  const float2* const ml = (const float2*)(p.ws + (int64_t)splits * rows * D);
  float m = -INFINITY;
  for (int s = lane; s < splits; s += 64) m = fmaxf(m, ml[s * rows + row].x);
  m = max_xor32(max_xor16(row_allmax(m)));
  const float ref = m == -INFINITY ? 0.f : m;
  float den = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float2 r = ml[s * rows + row];
    if (r.y == 0.f) continue;                                             // (nothing seen there: no values were written)
    const float w = fast_exp2(r.x - ref);
    den = fmaf(w, r.y, den);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(w, p.ws[(s * rows + row) * D + E * lane + e], o[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) store_elem(p.out, p.dtype, row * D + E * lane + e, den == 0.f ? 0.f : o[e] / den);
}

// How a call is handed out: wavefronts of a block and splits of the keys.
struct PromptPlan { int waves, splits; };
static PromptPlan prompt_plan(int G, int Hkv, int64_t T, int B, int64_t max_k_len) {
  PromptPlan r = {4, 1};
  const int64_t blocks = row_tiles(T, G, 32 * r.waves, B) * Hkv;
  int64_t s = 512 / blocks, most = (max_k_len + 255) / 256;
  if (s > most) s = most;
  r.splits = s < 1 ? 1 : s > 64 ? 64 : (int)s;
  return r;
}
static size_t record_bytes(int D, int64_t rows, int splits) { return (size_t)rows * splits * (D + 2) * 4; }

template <int D, int KV>
__global__ __launch_bounds__(256) void attn_rows_kernel(PromptParams p) {
  constexpr int E = D / 64;
  __shared__ __attribute__((aligned(16))) float rows[4][128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= p.T_q * p.n_q_heads) return;
  const int64_t token = row / p.n_q_heads;
  const int head = (int)(row % p.n_q_heads);
  int b = -1, begin = 0, n = 0;
  for (int i = 0; i < p.B && b < 0; ++i) {
    packed_range(p.cu_q, i, p.T_q, begin, n);
    if (token >= begin && token < begin + n) b = i;
  }
  if (b < 0) return;
  int k0 = 0, len;
  if (KV == kKvInt4) len = min(max(p.seq_lens[b], 0), p.bound);
  else packed_range(p.cu_k, b, p.T_k, k0, len);
  const int i = (int)(token - begin);
  const int sees = p.causal ? min(len, len - n + i + 1) : len;
  const RowSource<D, KV> src = {p, b, head / p.group, k0, lane};
  float* const x = rows[wave];
  const uint16_t* const qr = (const uint16_t*)p.q + token * p.q_stride + (int64_t)head * D;
  if (E == 1) x[lane + 64] = 0.f;
  for (int e = 0; e < E; ++e) x[lane + 64 * e] = p.dtype == SAW_BF16 ? bf16_to_f32(qr[lane + 64 * e]) : f16_to_f32(qr[lane + 64 * e]);
  wave_sync();
  if (KV == kKvInt4) rotate_row(p, x, D, lane);
  float q[E], acc[E], m = -INFINITY, den = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) { q[e] = x[lane + 64 * e] * p.scale; acc[e] = 0.f; }
  for (int j = 0; j < sees; ++j) {
    float k[E], v[E], t = 0.f;
    src.load(false, j, k);
    src.load(true, j, v);
#pragma unroll
    for (int e = 0; e < E; ++e) t = fmaf(q[e], k[e], t);
    t = add_xor32(add_xor16(row_allsum(t)));
    const float top = fmaxf(m, t);
    const float ref = top == -INFINITY ? 0.f : top;
    const float alpha = fast_exp2(m - ref), w = fast_exp2(t - ref);
    m = top;
    den = fmaf(den, alpha, w);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(acc[e], alpha, w * v[e]);
  }
  wave_sync();
  for (int e = 0; e < E; ++e) x[lane + 64 * e] = den == 0.f ? 0.f : acc[e] / den;
  wave_sync();
  if (KV == kKvInt4) unrotate_row(p, x, D, lane);
  for (int e = 0; e < E; ++e) store_elem(p.out, p.dtype, row * D + lane + 64 * e, x[lane + 64 * e]);
}

// (max, sum) of every row's logits, for the weights
template <int D>
__global__ __launch_bounds__(256) void row_stats_kernel(PromptParams p) {
  constexpr int E = D / 64;
  __shared__ __attribute__((aligned(16))) float rows[4][128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= p.T_q * p.n_q_heads) return;
  const int64_t token = row / p.n_q_heads;
  const int head = (int)(row % p.n_q_heads);
  int b = -1, begin = 0, n = 0;
  for (int i = 0; i < p.B && b < 0; ++i) {
    packed_range(p.cu_q, i, p.T_q, begin, n);
    if (token >= begin && token < begin + n) b = i;
  }
  if (b < 0) return;
  const int len = min(max(p.seq_lens[b], 0), p.bound);
  const int sees = min(len, len - n + (int)(token - begin) + 1);
  const RowSource<D, kKvInt4> src = {p, b, head / p.group, 0, lane};
  float* const x = rows[wave];
  const uint16_t* const qr = (const uint16_t*)p.q + token * p.q_stride + (int64_t)head * D;
  if (E == 1) x[lane + 64] = 0.f;
  for (int e = 0; e < E; ++e) x[lane + 64 * e] = p.dtype == SAW_BF16 ? bf16_to_f32(qr[lane + 64 * e]) : f16_to_f32(qr[lane + 64 * e]);
  wave_sync();
  rotate_row(p, x, D, lane);
  float* const out = p.ws + row * (D + 2);
  float q[E], m = -INFINITY, den = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) { q[e] = x[lane + 64 * e] * p.scale; out[2 + lane + 64 * e] = q[e]; }
  for (int j = 0; j < sees; ++j) {
    float k[E], t = 0.f;
    src.load(false, j, k);
#pragma unroll
    for (int e = 0; e < E; ++e) t = fmaf(q[e], k[e], t);
    t = add_xor32(add_xor16(row_allsum(t)));
    const float top = fmaxf(m, t);
    const float ref = top == -INFINITY ? 0.f : top;
    den = fmaf(den, fast_exp2(m - ref), fast_exp2(t - ref));
    m = top;
  }
  if (lane == 0) { out[0] = m == -INFINITY ? 0.f : m; out[1] = den; }
}

// a wavefront per (sequence, kv head, position): the sum over the rows that see it
template <int D>
__global__ __launch_bounds__(256) void weights_kernel(PromptParams p) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = blockIdx.z, h = blockIdx.y, j = blockIdx.x * 4 + wave;
  const int len = min(max(p.seq_lens[b], 0), p.bound);
  if (j >= len) return;
  int begin, n;
  packed_range(p.cu_q, b, p.T_q, begin, n);
  const RowSource<D, kKvInt4> src = {p, b, h, 0, lane};
  float k[E], total = 0.f;
  src.load(false, j, k);
  for (int i = max(0, j - (len - n)); i < n; ++i)
    for (int g = 0; g < p.group; ++g) {
      const float* const r = p.ws + ((int64_t)(begin + i) * p.n_q_heads + h * p.group + g) * (D + 2);
      float t = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) t = fmaf(r[2 + lane + 64 * e], k[e], t);
      t = add_xor32(add_xor16(row_allsum(t)));
      if (r[1] != 0.f) total += fast_exp2(t - r[0]) / r[1];
    }
  const int64_t at = ((int64_t)b * p.n_kv_heads + h) * p.score_stride + j;
  if (lane == 0) p.scores[at] = (p.prev ? p.prev[at] : 0.f) + total;
}

template <int D, typename M>
static void launch_prompt16(const PromptParams& p, const PromptPlan& plan, hipStream_t st) {
  const dim3 grid((unsigned)(row_tiles(p.T_q, p.group, 32 * plan.waves, p.B) * p.n_kv_heads), plan.splits);
  prompt_kernel<D, M, 4><<<grid, dim3(256), 0, st>>>(p);
  if (plan.splits > 1) prompt_merge_kernel<D><<<dim3((unsigned)((p.T_q * p.n_q_heads + 3) / 4)), dim3(256), 0, st>>>(p, plan.splits);
}

int launch_prompt(const PromptParams& p, int D, bool int4, hipStream_t st) {
  const int64_t rows = p.T_q * p.n_q_heads;
  if (int4) {
    const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
    if (D == 128) attn_rows_kernel<128, kKvInt4><<<grid, block, 0, st>>>(p);
    else attn_rows_kernel<64, kKvInt4><<<grid, block, 0, st>>>(p);
  } else {
    const PromptPlan plan = prompt_plan(p.group, p.n_kv_heads, p.T_q, p.B, p.bound);
    if (D == 128) {
      if (p.dtype == SAW_BF16) launch_prompt16<128, MathBf16>(p, plan, st);
      else launch_prompt16<128, MathF16>(p, plan, st);
    } else {
      if (p.dtype == SAW_BF16) launch_prompt16<64, MathBf16>(p, plan, st);
      else launch_prompt16<64, MathF16>(p, plan, st);
    }
  }
  return hipGetLastError() == hipSuccess ? SAW_OK : SAW_ELAUNCH;
}

int launch_weights(const PromptParams& p, int D, hipStream_t st) {
  const int64_t rows = p.T_q * p.n_q_heads;
  const dim3 grid((unsigned)((rows + 3) / 4)), block(256), wgrid((p.bound + 3) / 4, p.n_kv_heads, p.B);
  if (D == 128) {
    if (rows) row_stats_kernel<128><<<grid, block, 0, st>>>(p);
    weights_kernel<128><<<wgrid, block, 0, st>>>(p);
  } else {
    if (rows) row_stats_kernel<64><<<grid, block, 0, st>>>(p);
    weights_kernel<64><<<wgrid, block, 0, st>>>(p);
  }
  return hipGetLastError() == hipSuccess ? SAW_OK : SAW_ELAUNCH;
}

size_t prompt_bytes(int D, int Hq, int Hkv, int64_t T, int B, int64_t max_k_len) {
  const PromptPlan plan = prompt_plan(Hq / Hkv, Hkv, T, B, max_k_len);
  return 16 + (plan.splits > 1 ? record_bytes(D, T * Hq, plan.splits) : 0);
}
size_t paged_prompt_bytes(int, int, int, int64_t, int, int64_t) { return 16; }
size_t weights_bytes(int D, int Hq, int, int64_t T, int, int64_t) { return 16 + (size_t)T * Hq * (D + 2) * 4; }

}  // namespace saw
