// Eviction: which tokens of every (sequence, kv head) are kept, and the move of their bytes to other pages.
#include "saw_evict.h"

namespace saw {

// Order of the scores as unsigned numbers: larger score, larger key; -0 = +0; NaN below everything.
__device__ __forceinline__ uint32_t score_key(float f) {
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  if ((u & 0x7fffffffu) == 0u) return 0x80000000u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Kept positions of one (sequence, kv head), in ascending order: a block finds the key of the last score that is kept, 8 bits of it a
// pass, and then hands out the places in one scan over the positions; of equal keys the lowest positions are kept.
__global__ __launch_bounds__(1024) void evict_select_kernel(EvictParams p) {
  const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = min(max(p.seq_lens[b], 0), p.bound);
  const int64_t row = (int64_t)b * p.n_kv_heads + h;
  const float* const s = p.scores + row * p.score_stride;
  int32_t* const kept = p.kept + row * p.budget;
  float* const out = p.scores_out ? p.scores_out + row * p.score_out_stride : nullptr;
  const int n = min(len, p.budget), old = max(len - p.recent, 0);
  if (h == 0 && tid == 0) p.new_lens[b] = n;
  __shared__ int hist[256];
  __shared__ int pick[2];                       // digit, how many of it are still wanted
  __shared__ int sums[16][2];
  uint32_t prefix = 0;
  int want = n - (len - old);                   // of the old tokens
  const bool all = len <= p.budget;
  if (!all) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int j = tid; j < old; j += 1024) {
        const uint32_t key = score_key(s[j]);
        if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int left = want, d = 255;
        while (d > 0 && hist[d] < left) left -= hist[d--];
        pick[0] = d;
        pick[1] = left;
      }
      __syncthreads();
      prefix |= (uint32_t)pick[0] << shift;
      want = pick[1];
      __syncthreads();
    }
  }
  // `want` of the tokens whose key is `prefix` are kept, the lowest positions first
  int done = 0, ties = 0;
  for (int j0 = 0; j0 < len; j0 += 1024) {
    const int j = j0 + tid;
    bool above = false, tie = false;
    if (j < len) {
      if (all || j >= old) above = true;
      else {
        const uint32_t key = score_key(s[j]);
        above = n > len - old && key > prefix;
        tie = n > len - old && key == prefix;
      }
    }
    const uint64_t am = __ballot(above), tm = __ballot(tie), below = (1ull << lane) - 1;
    if (lane == 0) { sums[wave][0] = __popcll(am); sums[wave][1] = __popcll(tm); }
    __syncthreads();
    int t0 = ties, a0 = done, at, tt = ties;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) { t0 += sums[w][1]; a0 += sums[w][0]; }
      done += sums[w][0];
      tt += sums[w][1];
    }
    t0 += __popcll(tm & below);
    a0 += __popcll(am & below);
    at = a0 + min(t0, want) - 0;
    // (`done` counts what is above; kept ties are counted apart)
    if (above || (tie && t0 < want)) {
      kept[at] = j;
      if (out) out[at] = s[j];
    }
    ties = tt;
    __syncthreads();
  }
  for (int i = n + tid; i < p.budget; i += 1024) {
    kept[i] = -1;
    if (out) out[i] = 0.f;
  }
}

template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  constexpr int LPV = D / 32;                    // 16-byte pieces of a vector's codes
  const int t = blockIdx.x * (256 / LPV) + threadIdx.x / LPV, part = threadIdx.x % LPV;
  const int b = blockIdx.z, h = blockIdx.y;
  if (t >= min(min(max(p.seq_lens[b], 0), p.bound), p.budget)) return;
  const int j = p.kept[((int64_t)b * p.n_kv_heads + h) * p.budget + t];
  if (j < 0) return;
  const int from = p.page_table[(int64_t)b * p.max_pages + (j >> 4)], to = p.dst_table[(int64_t)b * p.dst_pages + (t >> 4)];
  if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) return;
  const int64_t src = ((int64_t)from * p.n_kv_heads + h) * 16 + (j & 15), dst = ((int64_t)to * p.n_kv_heads + h) * 16 + (t & 15);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    ((u32x4*)(p.codes[w] + dst * (D / 2)))[part] = ((const u32x4*)(p.codes[w] + src * (D / 2)))[part];
    if (part == w) ((u32x2*)p.meta[w])[dst] = ((const u32x2*)p.meta[w])[src];
  }
}

int launch_evict(const EvictParams& p, int B, int D, hipStream_t st) {
  evict_select_kernel<<<dim3(p.n_kv_heads, B), dim3(1024), 0, st>>>(p);
  const int per = 256 / (D / 32);
  const dim3 grid((p.budget + per - 1) / per, p.n_kv_heads, B);
  if (D == 128) evict_move_kernel<128><<<grid, dim3(256), 0, st>>>(p);
  else evict_move_kernel<64><<<grid, dim3(256), 0, st>>>(p);
  return hipGetLastError() == hipSuccess ? SAW_OK : SAW_ELAUNCH;
}

}  // namespace saw
