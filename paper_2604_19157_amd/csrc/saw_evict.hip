// Eviction: which tokens of every (sequence, kv head) are kept, and the move of their bytes to other pages.
#include "saw_evict.h"

namespace saw {

// Order of the scores as unsigned numbers: larger score, larger key; -0 = +0; NaN below everything.
__device__ __forceinline__ uint32_t score_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.f);                           // (-0 + 0 = +0)
  const uint32_t key = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return f == f ? key : 0u;
}
__device__ __forceinline__ float score_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

constexpr int kBins = 2048, kCopies = 4, kListed = 8192, kAtOnce = 16;

// The largest bin d such that the bins above it hold fewer than `want` entries, and how many are still wanted of it: by the first
// wavefront, 32 bins a lane.  (A single thread that walked the bins took 8 us a digit.)
__device__ __forceinline__ int bin_of(const int* hist, int d) {
  int n = 0;
#pragma unroll
  for (int c = 0; c < kCopies; ++c) n += hist[d * kCopies + c];
  return n;
}
__device__ __forceinline__ void pick_bin(const int* hist, int want, int lane, int (&pick)[3]) {
  constexpr int kMine = kBins / 64;
  int mine = 0;
#pragma unroll 8
  for (int i = 0; i < kMine; ++i) mine += bin_of(hist, lane * kMine + (i + lane) % kMine);
  int upto = mine;                               // entries of this lane's bins and of all lanes' above
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_down(upto, d);
    if (lane + d < 64) upto += v;
  }
  const uint64_t enough = __ballot(upto >= want);          // lanes 0 .. k
  const int k = enough ? 63 - __builtin_clzll(enough) : 0;
  // lane k's bins, one a lane, the highest first
  int left = want - __shfl(upto - mine, k);
  const int d = k * kMine + kMine - 1 - lane;
  const int of = lane < kMine ? bin_of(hist, d) : 0;
  int before = of;                               // of the bins down to this one
#pragma unroll
  for (int i = 1; i < kMine; i <<= 1) {
    const int v = __shfl_up(before, i);
    if (lane >= i) before += v;
  }
  const uint64_t reached = __ballot(lane < kMine && before >= left) | 1ull << (kMine - 1);
  if (lane == __builtin_ctzll(reached)) {
    pick[0] = d;
    pick[1] = left - (before - of);
    pick[2] = of;
  }
}

// f(position, score) for the positions of [j0, j1) that a thread of `threads` is given, kAtOnce loads in flight while there are as many
template <int N, typename F>
__device__ __forceinline__ int batch_scores(const float* s, int j, int j1, int thread, int threads, F f) {
  for (; j + (N - 1) * threads < j1; j += N * threads) {
    float x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) x[u] = s[min(j + u * threads + thread, j1 - 1)];
#pragma unroll
    for (int u = 0; u < N; ++u) f(j + u * threads + thread, x[u]);
  }
  return j;
}
template <typename F>
__device__ __forceinline__ void for_scores(const float* s, int j0, int j1, int thread, int threads, F f) {
  const int j = batch_scores<kAtOnce>(s, j0, j1, thread, threads, f);
  batch_scores<1>(s, batch_scores<4>(s, j, j1, thread, threads, f), j1, thread, threads, f);
}

// The last score that is kept: positions from `old` on and scores above it are, of its equals the first.  (Compared as floats, which agrees
// with the keys but for NaN: if that is the last that is kept, every number is above it.)
struct Last {
  float score;
  bool nan;
  int old;
  __device__ Last(uint32_t key, int old) : score(score_of(key)), nan(key == 0), old(old) {}
  __device__ bool above(int at, float f) const { return at >= old || (nan ? f == f : f > score); }
  __device__ bool tie(int at, float f) const { return at < old && (nan ? f != f : f == score); }
};

// Kept positions of those that each(f) calls f(position, score) with, ascending over the lanes and calls (from j1 on: none), by each of the
// block's 16 wavefronts: they count what they keep, then write it behind what the wavefronts in
// front of them keep, and the block behind `done` kept tokens with `tied` equals of the last among them.
template <typename E>
__device__ __forceinline__ void write_kept(E each, int j1, int wave, int lane, const Last& last, int want, int done, int tied,
                                           int2* sums, int32_t* kept, float* out) {
  int above = 0, ties = 0;
  each([&](int at, float f) {
    above += __popcll(__ballot(at < j1 && last.above(at, f)));
    ties += __popcll(__ballot(at < j1 && last.tie(at, f)));
  });
  if (lane == 0) sums[wave] = make_int2(above, ties);
  __syncthreads();
  for (int w = 0; w < wave; ++w) { done += sums[w].x; tied += sums[w].y; }
  each([&](int at, float f) {
    const bool over = at < j1 && last.above(at, f), tie = at < j1 && last.tie(at, f);
    const uint64_t om = __ballot(over), tm = __ballot(tie);
    if (om | tm) {
      int to = done + min(tied, want) + __builtin_amdgcn_mbcnt_hi((uint32_t)(om >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)om, 0));
      bool keep = over;
      if (tm) {
        const int t = tied + __builtin_amdgcn_mbcnt_hi((uint32_t)(tm >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)tm, 0));
        to += min(t, want) - min(tied, want);
        keep = over || (tie && t < want);
      }
      if (keep) {
        kept[to] = at;
        if (out) out[to] = f;
      }
      done += __popcll(om);
      tied += __popcll(tm);
    }
  });
}

// Keys of [0, n) whose first digit is that of `prefix`, appended to `list` by the block's threads; `count` starts at zero.
__device__ __forceinline__ void list_candidates(const float* s, int j0, int j1, int tid, int lane, uint32_t prefix, uint32_t* list, int* count) {
  const uint64_t below = (1ull << lane) - 1;
  for_scores(s, j0, j1, tid, 1024, [&](int j, float f) {
    const uint32_t key = score_key(f);
    const bool take = j < j1 && key >> 21 == prefix >> 21;
    const uint64_t m = __ballot(take);
    if (m) {                                      // (one addition a wavefront)
      int at = 0;
      if (lane == 0) at = atomicAdd(count, __popcll(m));
      at = __builtin_amdgcn_readfirstlane(at) + __popcll(m & below);
      if (take) list[at] = key;
    }
  });
}

// Kept positions of one (sequence, kv head), in ascending order, by one block.  The key of the last score that is kept is found 11, 11 and
// 10 bits at a time; scores that share its first digit are listed in shared memory on the way, so that they alone are looked at for the
// others (where more than 8192 do, all scores are read again).  Then each wavefront counts what it keeps of its share of the positions
// and writes it behind the wavefronts in front of it; of equal keys the lowest positions are kept.
// Bound by its chain of steps - three times clearing, counting and picking, a barrier behind each, and the scores read four times from L2
// (reading them once into shared memory is level) -: 48 sequences of 700 to 8000 tokens and 8 heads 23 us, 4 of 600 to 1100 10 us.
__global__ __launch_bounds__(1024, 8) void evict_select_kernel(EvictParams p) {
  const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = min(max(p.seq_lens[b], 0), p.bound);
  const int64_t row = (int64_t)b * p.n_kv_heads + h;
  const float* const s = p.scores + row * p.score_stride;
  int32_t* const kept = p.kept + row * p.budget;
  float* const out = p.scores_out ? p.scores_out + row * p.score_out_stride : nullptr;
  const int n = min(len, p.budget), old = max(len - p.recent, 0);
  for (int i = n + tid; i < p.budget; i += 1024) {
    kept[i] = -1;
    if (out) out[i] = 0.f;
  }
  if (len <= p.budget) {
    for (int i = tid; i < len; i += 1024) {
      kept[i] = i;
      if (out) out[i] = s[i];
    }
    return;
  }
  __shared__ int hist[kBins * kCopies];          // (four copies, by lane: scores of like size meet in few bins)
  __shared__ int pick[3];                       // digit, how many of it are still wanted, how many there are
  __shared__ uint32_t listed[kListed];
  __shared__ int count;
  __shared__ int2 sums[16];
  uint32_t prefix = 0;
  int want = p.budget - p.recent;               // of the tokens in front of `old`
  int candidates = -1;                          // listed keys; -1: not listed
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? 1024 : kBins;
    for (int i = tid; i < kBins * kCopies; i += 1024) hist[i] = 0;
    if (tid == 0) count = 0;
    __syncthreads();
    if (digit == 0 || candidates < 0) {
      const int above = digit == 0 ? 31 : digit == 1 ? 21 : 10;                // (bits in front of the digit; none of the first)
      for_scores(s, 0, old, tid, 1024, [&](int j, float f) {
        const uint32_t key = score_key(f);
        if (j < old && (digit == 0 || key >> above == prefix >> above)) atomicAdd(&hist[((key >> shift) & (bins - 1)) * kCopies + lane % kCopies], 1);
      });
    } else {
      for (int j = tid; j < candidates; j += 1024) {
        const uint32_t key = listed[j];
        if (digit == 1 || (key >> 10) == (prefix >> 10)) atomicAdd(&hist[((key >> shift) & (bins - 1)) * kCopies + lane % kCopies], 1);
      }
    }
    __syncthreads();
    if (wave == 0) pick_bin(hist, want, lane, pick);
    __syncthreads();
    prefix |= (uint32_t)pick[0] << shift;
    want = pick[1];
    if (digit == 0) {
      candidates = pick[2] <= kListed ? 0 : -1;
      if (candidates == 0) {
        list_candidates(s, 0, old, tid, lane, prefix, listed, &count);
        __syncthreads();
        candidates = count;
      }
    }
    __syncthreads();
  }
  // `want` of the tokens whose key is `prefix` are kept, the lowest positions first
  const Last last(prefix, old);
  const int share = (len + 1023) / 1024 * 64, j0 = wave * share, j1 = min(len, j0 + share);
  write_kept([&](auto f) { for_scores(s, j0, j1, lane, 64, f); }, j1, wave, lane, last, want, 0, 0, sums, kept, out);
}

// The same for few long rows, by a block for every 8192 positions in three launches: digits of the segments; candidates of the segments, whose
// first digit every block picks by itself from all segments' counts; the remaining digits, by every block from all segments' candidates, and
// the segment's kept positions.  (131072 tokens, 8 heads: 4.6, 8.4 and 13.7 us; one block a row took 120, bound by the instructions that a single compute unit
// issues.)
constexpr int kSegment = 8192;

struct SegmentSpace {
  int* hist;                // [row][segment][kBins]
  uint32_t* list;           // [row][segment][kSegment]
  int2* counts;             // [row][segment]: scores above the first digit of the last, candidates
  int2* first;              // [row]: that digit, how many of it are wanted
  int segments;
  __host__ __device__ SegmentSpace(void* ws, int64_t rows, int segments) : segments(segments) {
    hist = (int*)ws;
    list = (uint32_t*)(hist + rows * segments * kBins);
    counts = (int2*)(list + rows * segments * kSegment);
    first = counts + rows * segments;
  }
};

__device__ __forceinline__ void clear(int* hist, int tid) {
  for (int i = tid; i < kBins * kCopies; i += 1024) hist[i] = 0;
}

__global__ __launch_bounds__(1024) void evict_digit_kernel(EvictParams p, SegmentSpace ws) {
  const int b = blockIdx.z, h = blockIdx.y, seg = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int len = min(max(p.seq_lens[b], 0), p.bound), old = max(len - p.recent, 0);
  const int j0 = seg * kSegment, j1 = min(old, j0 + kSegment);
  if (len <= p.budget || j0 >= len) return;
  const int64_t row = (int64_t)b * p.n_kv_heads + h;
  __shared__ int hist[kBins * kCopies];
  clear(hist, tid);
  __syncthreads();
  for_scores(p.scores + row * p.score_stride, j0, j1, tid, 1024, [&](int j, float f) {
    if (j < j1) atomicAdd(&hist[(score_key(f) >> 21) * kCopies + lane % kCopies], 1);
  });
  __syncthreads();
  for (int d = tid; d < kBins; d += 1024) ws.hist[(row * ws.segments + seg) * kBins + d] = bin_of(hist, d);
}

// f(key) for the m keys of a list, by a wavefront, eight loads in flight
template <typename F>
__device__ __forceinline__ void each_listed(const uint32_t* list, int m, int lane, F f) {
  for (int i = lane; i < m; i += 64 * 8) {
    uint32_t key[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) key[u] = list[min(i + 64 * u, m - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i + 64 * u < m) f(key[u]);
  }
}

// first digit of the last key that is kept, from the segments' counts
__device__ __forceinline__ void pick_first(const SegmentSpace& ws, int64_t row, int segments, int want, int tid, int lane, int* hist, int (&pick)[3]) {
  // (two bins a thread, and sixteen segments' on their way at once: a load waits longer than it works)
  const int2* const from = (const int2*)(ws.hist + row * ws.segments * kBins) + tid;
  int2 n = make_int2(0, 0);
  for (int g0 = 0; g0 < segments; g0 += 16) {
    int2 v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = from[(int64_t)min(g0 + k, segments - 1) * (kBins / 2)];
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (g0 + k < segments) { n.x += v[k].x; n.y += v[k].y; }
  }
  static_assert(kBins == 2 * 1024 && kCopies == 4, "two bins a thread");
  ((int4*)hist)[2 * tid] = make_int4(n.x, 0, 0, 0);
  ((int4*)hist)[2 * tid + 1] = make_int4(n.y, 0, 0, 0);
  __syncthreads();
  if (tid < 64) pick_bin(hist, want, lane, pick);
  __syncthreads();
}

__global__ __launch_bounds__(1024, 8) void evict_list_kernel(EvictParams p, SegmentSpace ws) {
  const int b = blockIdx.z, h = blockIdx.y, seg = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int len = min(max(p.seq_lens[b], 0), p.bound), old = max(len - p.recent, 0);
  const int j0 = seg * kSegment, j1 = min(old, j0 + kSegment);
  if (len <= p.budget || j0 >= len) return;
  const int64_t row = (int64_t)b * p.n_kv_heads + h;
  __shared__ __attribute__((aligned(16))) int hist[kBins * kCopies];
  __shared__ int pick[3];
  __shared__ int count, above;
  if (tid == 0) count = above = 0;
  pick_first(ws, row, (len + kSegment - 1) / kSegment, p.budget - p.recent, tid, lane, hist, pick);
  if (seg == 0 && tid == 0) ws.first[row] = make_int2(pick[0], pick[1]);
  list_candidates(p.scores + row * p.score_stride, j0, j1, tid, lane, (uint32_t)pick[0] << 21, ws.list + (row * ws.segments + seg) * kSegment, &count);
  int mine = 0;                                  // scores of larger digits
  for (int d = tid; d < kBins; d += 1024)
    if (d > pick[0]) mine += ws.hist[(row * ws.segments + seg) * kBins + d];
  if (mine) atomicAdd(&above, mine);
  __syncthreads();
  if (tid == 0) ws.counts[row * ws.segments + seg] = make_int2(above, count);
}

__global__ __launch_bounds__(1024, 8) void evict_write_kernel(EvictParams p, SegmentSpace ws) {
  const int b = blockIdx.z, h = blockIdx.y, seg = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = min(max(p.seq_lens[b], 0), p.bound), old = max(len - p.recent, 0), n = min(len, p.budget);
  const int64_t row = (int64_t)b * p.n_kv_heads + h;
  const float* const s = p.scores + row * p.score_stride;
  int32_t* const kept = p.kept + row * p.budget;
  float* const out = p.scores_out ? p.scores_out + row * p.score_out_stride : nullptr;
  // (every block a part of what lies behind the kept tokens, or of a sequence that is kept whole)
  for (int64_t i = (len <= p.budget ? 0 : n) + seg * 1024 + tid; i < p.budget; i += 1024 * (int)gridDim.x) {      // (a step may pass 2^31)
    kept[i] = i < n ? (int32_t)i : -1;
    if (out) out[i] = i < n ? s[i] : 0.f;
  }
  const int j0 = seg * kSegment, j1 = min(len, j0 + kSegment);
  if (len <= p.budget || j0 >= len) return;
  __shared__ __attribute__((aligned(16))) int hist[kBins * kCopies];
  __shared__ int pick[3];
  __shared__ int2 sums[16];
  __shared__ int before[2];
  const int segments = (len + kSegment - 1) / kSegment;
  constexpr int kMine = kSegment / 1024;         // of the lane, requested before the steps that they wait for
  const int w0 = j0 + wave * (kSegment / 16);
  float mine[kMine];
#pragma unroll
  for (int u = 0; u < kMine; ++u) mine[u] = s[min(w0 + 64 * u + lane, j1 - 1)];
  if (tid == 0) before[0] = before[1] = 0;
  const int2 first = ws.first[row];
  uint32_t prefix = (uint32_t)first.x << 21;
  int want = first.y;
  for (int digit = 1; digit < 3; ++digit) {
    const int shift = digit == 1 ? 10 : 0, bins = digit == 1 ? kBins : 1024, above = digit == 1 ? 21 : 10;
    __syncthreads();
    clear(hist, tid);
    __syncthreads();
    for (int g = wave; g < segments; g += 16) {              // (a wavefront a list)
      const int64_t at = row * ws.segments + g;
      each_listed(ws.list + at * kSegment, ws.counts[at].y, lane, [&](uint32_t key) {
        if (key >> above == prefix >> above) atomicAdd(&hist[((key >> shift) & (bins - 1)) * kCopies + lane % kCopies], 1);
      });
    }
    __syncthreads();
    if (wave == 0) pick_bin(hist, want, lane, pick);
    __syncthreads();
    prefix |= (uint32_t)pick[0] << shift;
    want = pick[1];
  }
  // kept in front of the segment, and equals of the last among the candidates there
  for (int g = wave; g < seg; g += 16) {
    const int64_t at = row * ws.segments + g;
    const int2 c = ws.counts[at];
    int above = 0, ties = 0;
    each_listed(ws.list + at * kSegment, c.y, lane, [&](uint32_t key) {
      above += key > prefix;
      ties += key == prefix;
    });
    for (int d = 1; d < 64; d <<= 1) { above += __shfl_xor(above, d); ties += __shfl_xor(ties, d); }
    if (lane == 0) {
      // (positions from `old` on are kept; where a segment in front of this one reaches them its end does)
      atomicAdd(&before[0], above + c.x + max(0, min(len, (g + 1) * kSegment) - max(old, g * kSegment)));
      atomicAdd(&before[1], ties);
    }
  }
  __syncthreads();
  const Last last(prefix, old);
  write_kept([&](auto f) {
#pragma unroll
    for (int u = 0; u < kMine; ++u) f(w0 + 64 * u + lane, mine[u]);
  }, j1, wave, lane, last, want, before[0], before[1], sums, kept, out);
}

// The kept tokens' codes and pairs, a thread for 16 bytes of K and of V of four tokens: where a token lies takes three loads one after the
// other, so that four of these chains have to be under way at once.  Bound by the memory: reads of 64 bytes at a time, writes of whole
// tiles (48 sequences, 2048 tokens kept, 226 MB: 54 to 61 us where no cache holds them, 4.2 TB/s at best; a copy reaches 5.05).
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  constexpr int LPV = D / 32, kEach = 4, kStep = 256 / LPV;      // 16-byte pieces of a vector's codes; tokens of a thread; tokens at once
  const int t0 = blockIdx.x * (kEach * kStep) + threadIdx.x / LPV, part = threadIdx.x % LPV;
  const int b = blockIdx.z, h = blockIdx.y;
  const int n = min(min(max(p.seq_lens[b], 0), p.bound), p.budget);
  // (new_lens may be seq_lens itself: the kernels before this one need the whole length; n is the same before and after the write)
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) p.new_lens[b] = n;
  if (t0 >= n) return;
  const int32_t* const kept = p.kept + ((int64_t)b * p.n_kv_heads + h) * p.budget;
  int j[kEach], from[kEach], to[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) j[k] = kept[min(t0 + k * kStep, n - 1)];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    from[k] = p.page_table[(int64_t)b * p.max_pages + (max(j[k], 0) >> 4)];
    to[k] = p.dst_table[(int64_t)b * p.dst_pages + (min(t0 + k * kStep, n - 1) >> 4)];
  }
  u32x4 codes[kEach][2];
  u32x2 pair[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int page = from[k] >= 0 && from[k] < p.num_pages ? from[k] : 0;
    const int64_t src = ((int64_t)page * p.n_kv_heads + h) * 16 + (j[k] & 15);
    codes[k][0] = ((const u32x4*)(p.codes[0] + src * (D / 2)))[part];
    codes[k][1] = ((const u32x4*)(p.codes[1] + src * (D / 2)))[part];
    pair[k] = ((const u32x2*)(part == 0 ? p.meta[0] : p.meta[1]))[src];
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int t = t0 + k * kStep;
    if (t >= n || from[k] < 0 || from[k] >= p.num_pages || to[k] < 0 || to[k] >= p.num_pages) continue;
    const int64_t dst = ((int64_t)to[k] * p.n_kv_heads + h) * 16 + (t & 15);
    ((u32x4*)(p.codes[0] + dst * (D / 2)))[part] = codes[k][0];
    ((u32x4*)(p.codes[1] + dst * (D / 2)))[part] = codes[k][1];
    if (part < 2) ((u32x2*)p.meta[part])[dst] = pair[k];
  }
}

// Segments are worth their three launches while rows alone leave compute units without work and are long: 8 rows of 131072 tokens 136 us in
// all with a block a row; 8 of 16384 level.
static int evict_segments(int64_t rows, int64_t bound) { return rows < 128 && bound > 16384 ? (int)((bound + kSegment - 1) / kSegment) : 0; }
size_t evict_bytes(int64_t rows, int64_t bound) {
  const size_t segments = evict_segments(rows, bound);
  return segments * rows * (kBins * 4 + kSegment * 4 + 8) + (segments ? rows * 8 : 0);
}

int launch_evict(const EvictParams& p, int B, int D, void* ws, hipStream_t st) {
  const int64_t rows = (int64_t)B * p.n_kv_heads;
  const int segments = evict_segments(rows, p.bound);
  if (segments) {
    const SegmentSpace space(ws, rows, segments);
    const dim3 grid(segments, p.n_kv_heads, B);
    evict_digit_kernel<<<grid, dim3(1024), 0, st>>>(p, space);
    evict_list_kernel<<<grid, dim3(1024), 0, st>>>(p, space);
    evict_write_kernel<<<grid, dim3(1024), 0, st>>>(p, space);
  } else {
    evict_select_kernel<<<dim3(p.n_kv_heads, B), dim3(1024), 0, st>>>(p);
  }
  const int per = 4 * 256 / (D / 32);
  const dim3 grid((p.budget + per - 1) / per, p.n_kv_heads, B);
  if (D == 128) evict_move_kernel<128><<<grid, dim3(256), 0, st>>>(p);
  else evict_move_kernel<64><<<grid, dim3(256), 0, st>>>(p);
  return hipGetLastError() == hipSuccess ? SAW_OK : SAW_ELAUNCH;
}

}  // namespace saw
