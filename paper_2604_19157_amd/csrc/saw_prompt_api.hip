// C ABI entry points of packed queries (prompt attention, attention and attention weights over the INT4 pages) and of eviction:
// argument validation on the host, then kernel launches on the caller's stream.
#include <math.h>

#include "saw_check.h"
#include "saw_evict.h"
#include "saw_prompt.h"

namespace saw {

int launch_prompt(const PromptParams&, int D, bool int4, hipStream_t);
int launch_weights(const PromptParams&, int D, hipStream_t);
int launch_evict(const EvictParams&, int B, int D, hipStream_t);
size_t prompt_bytes(int D, int Hq, int Hkv, int64_t T, int B, int64_t max_k_len);
size_t paged_prompt_bytes(int D, int Hq, int Hkv, int64_t T, int B, int64_t max_k_len);
size_t weights_bytes(int D, int Hq, int Hkv, int64_t T, int B, int64_t max_k_len);

static bool group_ok(int n_q_heads, int n_kv_heads) {
  if (n_kv_heads < 1 || n_kv_heads > 65535 || n_q_heads < 1 || n_q_heads % n_kv_heads) return false;
  const int g = n_q_heads / n_kv_heads;
  return g == 1 || g == 2 || g == 4 || g == 8;
}
static bool tokens_ok(int64_t T, int B) { return T >= 0 && T <= 0x7fffffffLL && B >= 1 && B <= 65535; }
static bool aligned4(const void* p) { return (((uintptr_t)p) & 3u) == 0; }

static float log2_scale(float sm_scale, int head_dim) {
  return (sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)head_dim)) * 1.4426950408889634f;
}

// The arguments that the calls over the INT4 pages share; `bound`: the clamp of the lengths.
static int paged_args(const saw_cache_t* c, const void* q, int dtype, int64_t T, int64_t q_stride, int Hq, const int32_t* cu_q, int B,
                      const int32_t* pt, int max_pages, const int32_t* seq_lens, int32_t max_seq_len, float sm_scale, void* ws,
                      bool values, PromptParams* p) {
  if (!c) return SAW_ENULL;
  if (!shape_ok(c) || !block_ok(c)) return SAW_EINVAL;
  if (dtype != SAW_F16 && dtype != SAW_BF16) return SAW_EINVAL;
  if (!group_ok(Hq, c->n_kv_heads) || !tokens_ok(T, B) || max_pages < 1) return SAW_EINVAL;
  const int64_t cap = (int64_t)max_pages * c->page_size;
  if (cap > 0x7fffffffLL || max_seq_len > cap) return SAW_EINVAL;
  if (!isfinite(sm_scale)) return SAW_EINVAL;
  if (q_stride < (int64_t)Hq * c->head_dim || (q_stride & 7)) return SAW_EINVAL;
  if (!c->k_codes || !c->k_meta || (values && (!c->v_codes || !c->v_meta)) || !cu_q || !pt || !seq_lens || (T && (!q || !ws))) return SAW_ENULL;
  if (!aligned16(q) || !aligned16(ws) || !aligned16(c->k_codes) || !aligned16(c->k_meta) || !aligned4(cu_q) || !aligned4(pt) || !aligned4(seq_lens))
    return SAW_EINVAL;
  if (values && (!aligned16(c->v_codes) || !aligned16(c->v_meta))) return SAW_EINVAL;
  *p = {};
  p->q = q; p->q_stride = q_stride; p->T_q = T; p->cu_q = cu_q; p->B = B; p->n_q_heads = Hq; p->n_kv_heads = c->n_kv_heads;
  p->group = Hq / c->n_kv_heads; p->dtype = dtype; p->scale = log2_scale(sm_scale, c->head_dim); p->causal = 1;
  p->k_codes = c->k_codes; p->v_codes = c->v_codes; p->k_meta = c->k_meta; p->v_meta = c->v_meta;
  p->page_table = pt; p->seq_lens = seq_lens; p->max_pages = max_pages; p->num_pages = c->num_pages;
  p->bound = max_seq_len <= 0 ? (int32_t)cap : max_seq_len;
  p->had_block = c->had_block;
  p->rot_k = (c->rotate_mask & SAW_ROT_K) && c->had_block > 1;
  p->rot_v = (c->rotate_mask & SAW_ROT_V) && c->had_block > 1;
  for (int i = 0; i < 4; ++i) p->signs.w[i] = c->sign_bits[i];
  p->has_signs = (p->signs.w[0] | p->signs.w[1] | p->signs.w[2] | p->signs.w[3]) != 0;
  p->dense = (const float*)c->dense_rot;
  p->dense_k = p->dense && (c->rotate_mask & SAW_ROT_K);
  p->dense_v = p->dense && (c->rotate_mask & SAW_ROT_V);
  p->ws = (float*)ws;
  return SAW_OK;
}

}  // namespace saw

using namespace saw;

extern "C" {

size_t saw_prompt_workspace_bytes(int32_t head_dim, int32_t n_q_heads, int32_t n_kv_heads, int64_t T_q, int32_t B, int64_t max_k_len) {
  if ((head_dim != 64 && head_dim != 128) || !group_ok(n_q_heads, n_kv_heads) || !tokens_ok(T_q, B) || max_k_len < 0 || max_k_len > 0x7fffffffLL) return 0;
  return prompt_bytes(head_dim, n_q_heads, n_kv_heads, T_q, B, max_k_len);
}

int saw_prompt_attn(const void* q, const void* k, const void* v, int32_t dtype, int32_t head_dim, int32_t n_q_heads, int32_t n_kv_heads,
                    int64_t T_q, int64_t T_k, int64_t q_stride, int64_t k_stride, int64_t v_stride, const int32_t* cu_q,
                    const int32_t* cu_k, int32_t B, int64_t max_k_len, int32_t causal, float sm_scale, void* out, void* workspace,
                    size_t workspace_bytes, saw_stream_t stream) {
  if (dtype != SAW_F16 && dtype != SAW_BF16) return SAW_EINVAL;
  if ((head_dim != 64 && head_dim != 128) || !group_ok(n_q_heads, n_kv_heads) || !tokens_ok(T_q, B) || !tokens_ok(T_k, B)) return SAW_EINVAL;
  if (!isfinite(sm_scale)) return SAW_EINVAL;
  const int64_t kv = (int64_t)n_kv_heads * head_dim;
  if (q_stride < (int64_t)n_q_heads * head_dim || k_stride < kv || v_stride < kv || ((q_stride | k_stride | v_stride) & 7)) return SAW_EINVAL;
  if (T_q == 0) return SAW_OK;
  if (!q || (T_k && (!k || !v)) || !cu_q || !cu_k || !out || !workspace) return SAW_ENULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(workspace) || !aligned4(cu_q) || !aligned4(cu_k)) return SAW_EINVAL;
  PromptParams p = {};
  p.q = q; p.k = k; p.v = v; p.dtype = dtype; p.n_q_heads = n_q_heads; p.n_kv_heads = n_kv_heads; p.group = n_q_heads / n_kv_heads;
  p.T_q = T_q; p.T_k = T_k; p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.cu_q = cu_q; p.cu_k = cu_k; p.B = B;
  p.causal = causal != 0; p.scale = log2_scale(sm_scale, head_dim); p.out = out; p.ws = (float*)workspace;
  p.bound = (int32_t)(max_k_len <= 0 || max_k_len > T_k ? T_k : max_k_len);
  if (workspace_bytes < prompt_bytes(head_dim, n_q_heads, n_kv_heads, T_q, B, p.bound)) return SAW_EWORKSPACE;
  return launch_prompt(p, head_dim, false, (hipStream_t)stream);
}

size_t saw_paged_prompt_workspace_bytes(const saw_cache_t* c, int32_t n_q_heads, int64_t T, int32_t B, int64_t max_seq_len) {
  if (!c || !shape_ok(c) || !group_ok(n_q_heads, c->n_kv_heads) || !tokens_ok(T, B) || max_seq_len < 1 || max_seq_len > 0x7fffffffLL) return 0;
  return paged_prompt_bytes(c->head_dim, n_q_heads, c->n_kv_heads, T, B, max_seq_len);
}

int saw_paged_prompt_attn(const saw_cache_t* c, const void* q, int32_t dtype, int64_t T, int64_t q_stride, int32_t n_q_heads,
                          const int32_t* cu_q, int32_t B, const int32_t* page_table, int32_t max_pages_per_seq,
                          const int32_t* seq_lens, int32_t max_seq_len, float sm_scale, void* out, void* workspace,
                          size_t workspace_bytes, saw_stream_t stream) {
  PromptParams p;
  const int rc = paged_args(c, q, dtype, T, q_stride, n_q_heads, cu_q, B, page_table, max_pages_per_seq, seq_lens, max_seq_len, sm_scale,
                            workspace, true, &p);
  if (rc != SAW_OK) return rc;
  if (T == 0) return SAW_OK;
  if (!out) return SAW_ENULL;
  if (!aligned16(out)) return SAW_EINVAL;
  if (workspace_bytes < paged_prompt_bytes(c->head_dim, n_q_heads, c->n_kv_heads, T, B, p.bound)) return SAW_EWORKSPACE;
  p.out = out;
  return launch_prompt(p, c->head_dim, true, (hipStream_t)stream);
}

size_t saw_attn_weights_workspace_bytes(const saw_cache_t* c, int32_t n_q_heads, int64_t T, int32_t B, int64_t max_seq_len) {
  if (!c || !shape_ok(c) || !group_ok(n_q_heads, c->n_kv_heads) || !tokens_ok(T, B) || max_seq_len < 1 || max_seq_len > 0x7fffffffLL) return 0;
  return weights_bytes(c->head_dim, n_q_heads, c->n_kv_heads, T, B, max_seq_len);
}

int saw_paged_attn_weights(const saw_cache_t* c, const void* q, int32_t dtype, int64_t T, int64_t q_stride, int32_t n_q_heads,
                           const int32_t* cu_q, int32_t B, const int32_t* page_table, int32_t max_pages_per_seq,
                           const int32_t* seq_lens, int32_t max_seq_len, float sm_scale, const float* prev, float* scores,
                           int64_t score_stride, void* workspace, size_t workspace_bytes, saw_stream_t stream) {
  PromptParams p;
  const int rc = paged_args(c, q, dtype, T, q_stride, n_q_heads, cu_q, B, page_table, max_pages_per_seq, seq_lens, max_seq_len, sm_scale,
                            workspace, false, &p);
  if (rc != SAW_OK) return rc;
  if (!scores || !workspace) return SAW_ENULL;
  if (!aligned4(prev) || !aligned4(scores) || score_stride < p.bound) return SAW_EINVAL;
  if (workspace_bytes < weights_bytes(c->head_dim, n_q_heads, c->n_kv_heads, T, B, p.bound)) return SAW_EWORKSPACE;
  p.prev = prev; p.scores = scores; p.score_stride = score_stride;
  return launch_weights(p, c->head_dim, (hipStream_t)stream);
}

int saw_evict_pages(const saw_cache_t* c, const float* scores, int64_t score_stride, const int32_t* page_table,
                    int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t B, int32_t max_seq_len, int32_t budget, int32_t recent,
                    const int32_t* dst_table, int32_t dst_pages_per_seq, int32_t* new_lens, int32_t* kept, float* scores_out,
                    int64_t score_out_stride, saw_stream_t stream) {
  if (!c) return SAW_ENULL;
  if (!shape_ok(c) || c->n_kv_heads > 65535 || B < 1 || B > 65535 || max_pages_per_seq < 1 || dst_pages_per_seq < 1) return SAW_EINVAL;
  const int64_t cap = (int64_t)max_pages_per_seq * c->page_size;
  if (cap > 0x7fffffffLL || max_seq_len > cap) return SAW_EINVAL;
  const int32_t bound = max_seq_len <= 0 ? (int32_t)cap : max_seq_len;
  if (budget < 1 || recent < 0 || recent > budget || (int64_t)dst_pages_per_seq * c->page_size < budget) return SAW_EINVAL;
  if (score_stride < bound || (scores_out && score_out_stride < budget)) return SAW_EINVAL;
  if (!c->k_codes || !c->v_codes || !c->k_meta || !c->v_meta || !scores || !page_table || !seq_lens || !dst_table || !new_lens || !kept)
    return SAW_ENULL;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || (((uintptr_t)c->k_meta) & 7u) || (((uintptr_t)c->v_meta) & 7u)) return SAW_EINVAL;
  if (!aligned4(scores) || !aligned4(page_table) || !aligned4(seq_lens) || !aligned4(dst_table) || !aligned4(new_lens) || !aligned4(kept) || !aligned4(scores_out))
    return SAW_EINVAL;
  EvictParams p = {};
  p.codes[0] = c->k_codes; p.codes[1] = c->v_codes; p.meta[0] = c->k_meta; p.meta[1] = c->v_meta;
  p.scores = scores; p.score_stride = score_stride; p.page_table = page_table; p.seq_lens = seq_lens; p.dst_table = dst_table;
  p.max_pages = max_pages_per_seq; p.dst_pages = dst_pages_per_seq; p.num_pages = c->num_pages; p.n_kv_heads = c->n_kv_heads;
  p.bound = bound; p.budget = budget; p.recent = recent; p.new_lens = new_lens; p.kept = kept;
  p.scores_out = scores_out; p.score_out_stride = score_out_stride;
  return launch_evict(p, B, c->head_dim, (hipStream_t)stream);
}

}  // extern "C"
