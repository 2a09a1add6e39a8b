"""Argument marshalling of the binding's hot calls through ctypes: what ``csrc/marshal.cpp`` does, for a tree whose native module was
not built (it needs the headers of Python and torch, which the library itself does not).  A call takes 10 to 15 us longer on the
host.  Functions return the C call's code; a failed check raises AssertionError."""
from __future__ import annotations

import ctypes

import torch

from . import binding as b


def _rows(t):
    return t.dim() == 2 and t.is_contiguous()


def store(cache, K, V, page_table, slots):
    T = K.shape[0]
    assert K.dim() == 3 and K.dtype == V.dtype and K.shape == V.shape and K.stride(2) == 1 and K.stride(1) == cache.head_dim
    assert V.stride() == K.stride() and page_table.dtype == torch.int32 and slots.dtype == torch.int32
    assert _rows(page_table) and slots.is_contiguous() and slots.shape == (T, 2)
    st = cache.struct()
    return b.lib().saw_rotate_quant_store(ctypes.byref(st), b._ptr(K), b._ptr(V), b._DT[K.dtype], T,
                                          K.stride(0) if T > 1 else cache.n_kv_heads * cache.head_dim, b._ptr(page_table),
                                          page_table.shape[0], page_table.shape[1], b._ptr(slots), b._stream())


def store_layers(caches, Ks, Vs, page_table, slots):
    n = len(caches)
    c0, K0 = caches[0], Ks[0]
    T = K0.shape[0]
    stride = K0.stride(0) if T > 1 else c0.n_kv_heads * c0.head_dim
    assert len(Ks) == n == len(Vs) and K0.dim() == 3
    for K, V in zip(Ks, Vs):
        assert K.dtype == K0.dtype and K.shape == K0.shape == V.shape and K.stride(2) == 1 and K.stride(1) == c0.head_dim
        assert V.stride() == K.stride() and (T <= 1 or K.stride(0) == stride)
    assert _rows(page_table) and slots.is_contiguous() and slots.shape == (T, 2)
    sts = (b.SawCacheStruct * n)(*[c.struct() for c in caches])
    kp = (ctypes.c_void_p * n)(*[K.data_ptr() for K in Ks])
    vp = (ctypes.c_void_p * n)(*[V.data_ptr() for V in Vs])
    return b.lib().saw_rotate_quant_store_layers(sts, kp, vp, n, b._DT[K0.dtype], T, stride, b._ptr(page_table), page_table.shape[0],
                                                 page_table.shape[1], b._ptr(slots), b._stream())


def _hints(order, B):
    if order is None:
        return b.SawHints(None)
    assert order.dtype == torch.int32 and order.numel() == B and order.is_contiguous()
    return b.SawHints(order.data_ptr())


def decode(cache, q, page_table, seq_lens, max_seq_len, sm_scale, out, workspace, num_splits, order):
    B, Hq, _ = q.shape
    assert q.is_contiguous() and _rows(page_table) and seq_lens.dtype == torch.int32
    st, hints = cache.struct(), _hints(order, B)
    return b.lib().saw_paged_decode_attn_hinted(ctypes.byref(st), b._ptr(q), b._DT[q.dtype], B, Hq, b._ptr(page_table),
                                                page_table.shape[1], b._ptr(seq_lens), max_seq_len, float(sm_scale), b._ptr(out),
                                                b._DT[out.dtype], b._ptr(workspace), workspace.numel(), num_splits,
                                                ctypes.byref(hints), b._stream())


def append(cache, K_new, V_new, q, page_table, seq_lens, max_seq_len, sm_scale, out, workspace, order):
    B, Hq, _ = q.shape
    assert q.is_contiguous() and K_new.is_contiguous() and V_new.is_contiguous() and K_new.dtype == V_new.dtype
    assert _rows(page_table) and seq_lens.dtype == torch.int32
    st, hints = cache.struct(), _hints(order, B)
    return b.lib().saw_append_decode_attn_hinted(ctypes.byref(st), b._ptr(K_new), b._ptr(V_new), b._DT[K_new.dtype], b._ptr(q),
                                                 b._DT[q.dtype], B, Hq, b._ptr(page_table), page_table.shape[1], b._ptr(seq_lens),
                                                 max_seq_len, float(sm_scale), b._ptr(out), b._DT[out.dtype], b._ptr(workspace),
                                                 workspace.numel(), ctypes.byref(hints), b._stream())


def flatten(cache, page_table, seq, pos_begin, pos_end, unrotate, k_out, v_out):
    ref = k_out if k_out is not None else v_out
    stride = ref.stride(0) if pos_end > pos_begin else cache.n_kv_heads * cache.head_dim
    st = cache.struct()
    return b.lib().saw_flatten_dequant(ctypes.byref(st), b._ptr(page_table), page_table.shape[1], seq, pos_begin, pos_end,
                                       int(bool(unrotate)), b._DT[ref.dtype], b._ptr(k_out), b._ptr(v_out), stride, b._stream())


def kv16_decode(cache, q, page_table, seq_lens, max_seq_len, sm_scale, out, workspace, num_splits):
    B, Hq, _ = q.shape
    st = cache.struct()
    return b.lib().saw_kv16_paged_decode_attn(ctypes.byref(st), b._ptr(cache.k_pages), b._ptr(cache.v_pages), b._DT[cache.dtype],
                                              b._ptr(q), b._DT[q.dtype], B, Hq, b._ptr(page_table), page_table.shape[1],
                                              b._ptr(seq_lens), max_seq_len, float(sm_scale), b._ptr(out), b._DT[out.dtype],
                                              b._ptr(workspace), workspace.numel(), num_splits, b._stream())


def _on_this_gpu(*tensors):
    assert all(t.is_cuda for t in tensors), "every tensor is on the GPU"
    assert all(t.get_device() == torch.cuda.current_device() for t in tensors), "every tensor is on the current device"


def _pools(cache):
    return [t for t in (cache.k_codes, cache.v_codes, cache.k_meta, cache.v_meta, cache.dense_rot) if t is not None]


def _heads_dense(t):
    return t.dim() == 3 and (t.shape[2] <= 1 or t.stride(2) == 1) and (t.shape[1] <= 1 or t.stride(1) == t.shape[2])


def _token_stride(t):
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def _vector(t, n):
    return t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous() and t.numel() == n


def _table(t, rows):
    return t.dtype == torch.int32 and _rows(t) and t.shape[0] == rows


def _record(t, B, heads):
    return t.dtype == torch.float32 and t.dim() == 3 and t.is_contiguous() and t.shape[0] == B and t.shape[1] == heads


def _counts(*values):
    assert all(-2**31 <= v < 2**31 for v in values), "a count is beyond 32 bits"


def _like(out, q):
    return out.is_contiguous() and out.dtype == q.dtype and out.shape == q.shape


def prompt(q, k, v, cu_q, cu_k, max_k_len, causal, sm_scale, out, workspace):
    assert _heads_dense(q) and _heads_dense(k) and _heads_dense(v) and q.dtype == k.dtype == v.dtype
    assert k.shape == v.shape and q.shape[2] == k.shape[2] and _like(out, q) and cu_q.numel() >= 2
    assert _vector(cu_q, cu_q.numel()) and _vector(cu_k, cu_q.numel()) and workspace.is_contiguous()
    _on_this_gpu(q, k, v, cu_q, cu_k, out, workspace)
    return b.lib().saw_prompt_attn(b._ptr(q), b._ptr(k), b._ptr(v), b._DT[q.dtype], q.shape[2], q.shape[1], k.shape[1], q.shape[0],
                                   k.shape[0], _token_stride(q), _token_stride(k), _token_stride(v), b._ptr(cu_q), b._ptr(cu_k),
                                   cu_q.numel() - 1, max_k_len, int(bool(causal)), float(sm_scale), b._ptr(out), b._ptr(workspace),
                                   workspace.nbytes, b._stream())


def paged_prompt(cache, q, cu_q, page_table, seq_lens, max_seq_len, sm_scale, out, workspace):
    B = seq_lens.numel()
    _counts(max_seq_len)
    assert _heads_dense(q) and q.shape[2] == cache.head_dim and _like(out, q)
    assert _vector(cu_q, B + 1) and _vector(seq_lens, B) and _table(page_table, B) and workspace.is_contiguous()
    _on_this_gpu(q, cu_q, page_table, seq_lens, out, workspace, *_pools(cache))
    st = cache.struct()
    return b.lib().saw_paged_prompt_attn(ctypes.byref(st), b._ptr(q), b._DT[q.dtype], q.shape[0], _token_stride(q), q.shape[1], b._ptr(cu_q),
                                         B, b._ptr(page_table), page_table.shape[1], b._ptr(seq_lens), max_seq_len, float(sm_scale),
                                         b._ptr(out), b._ptr(workspace), workspace.nbytes, b._stream())


def attn_weights(cache, q, cu_q, page_table, seq_lens, prev, scores, max_seq_len, sm_scale, workspace):
    B = seq_lens.numel()
    _counts(max_seq_len)
    assert _heads_dense(q) and q.shape[2] == cache.head_dim and _record(scores, B, cache.n_kv_heads)
    assert prev is None or (_record(prev, B, cache.n_kv_heads) and prev.shape == scores.shape)
    assert _vector(cu_q, B + 1) and _vector(seq_lens, B) and _table(page_table, B) and workspace.is_contiguous()
    _on_this_gpu(q, cu_q, page_table, seq_lens, scores, workspace, *([] if prev is None else [prev]), *_pools(cache))
    st = cache.struct()
    return b.lib().saw_paged_attn_weights(ctypes.byref(st), b._ptr(q), b._DT[q.dtype], q.shape[0], _token_stride(q), q.shape[1],
                                          b._ptr(cu_q), B, b._ptr(page_table), page_table.shape[1], b._ptr(seq_lens), max_seq_len,
                                          float(sm_scale), b._ptr(prev), b._ptr(scores), scores.shape[2], b._ptr(workspace),
                                          workspace.nbytes, b._stream())


def evict(cache, scores, page_table, seq_lens, dst_table, budget, recent, max_seq_len, new_lens, kept, scores_out, workspace):
    B = seq_lens.numel()
    _counts(budget, recent, max_seq_len)
    assert _record(scores, B, cache.n_kv_heads) and (scores_out is None or _record(scores_out, B, cache.n_kv_heads))
    assert kept.dtype == torch.int32 and kept.is_contiguous() and kept.shape == (B, cache.n_kv_heads, budget)
    assert _vector(seq_lens, B) and _vector(new_lens, B) and _table(page_table, B) and _table(dst_table, B)
    _on_this_gpu(scores, page_table, seq_lens, dst_table, new_lens, kept, *(x for x in (scores_out, workspace) if x is not None), *_pools(cache))
    assert workspace is None or workspace.is_contiguous()
    st = cache.struct()
    return b.lib().saw_evict_pages(ctypes.byref(st), b._ptr(scores), scores.shape[2], b._ptr(page_table), page_table.shape[1],
                                   b._ptr(seq_lens), B, max_seq_len, budget, recent, b._ptr(dst_table), dst_table.shape[1],
                                   b._ptr(new_lens), b._ptr(kept), b._ptr(scores_out), 0 if scores_out is None else scores_out.shape[2],
                                   b._ptr(workspace), 0 if workspace is None else workspace.nbytes, b._stream())
