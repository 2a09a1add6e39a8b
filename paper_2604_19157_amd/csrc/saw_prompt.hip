// Attention of packed queries: softmax(q K^T s) V with K and V of 16 bits or read from the INT4 pages.
#include "saw_prompt.h"

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

int launch_prompt(const PromptParams& p, int D, bool int4, hipStream_t st) {
  const int64_t rows = p.T_q * p.n_q_heads;
  const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
  if (D == 128) {
    if (int4) attn_rows_kernel<128, kKvInt4><<<grid, block, 0, st>>>(p);
    else if (p.dtype == SAW_BF16) attn_rows_kernel<128, kKvBf16><<<grid, block, 0, st>>>(p);
    else attn_rows_kernel<128, kKvF16><<<grid, block, 0, st>>>(p);
  } else {
    if (int4) attn_rows_kernel<64, kKvInt4><<<grid, block, 0, st>>>(p);
    else if (p.dtype == SAW_BF16) attn_rows_kernel<64, kKvBf16><<<grid, block, 0, st>>>(p);
    else attn_rows_kernel<64, kKvF16><<<grid, block, 0, st>>>(p);
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

size_t prompt_bytes(int, int, int, int64_t, int, int64_t) { return 16; }
size_t paged_prompt_bytes(int, int, int, int64_t, int, int64_t) { return 16; }
size_t weights_bytes(int D, int Hq, int, int64_t T, int, int64_t) { return 16 + (size_t)T * Hq * (D + 2) * 4; }

}  // namespace saw
