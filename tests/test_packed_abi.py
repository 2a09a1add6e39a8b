"""Refusals of the calls of packed queries and of eviction, without a GPU: every one is turned down on the host before anything is launched."""
import ctypes
import math
import warnings

import pytest
import torch


@pytest.fixture(scope="module")
def saw():
    import os
    from paper_2604_19157_amd import binding, build
    if not os.path.exists(build.LIB):
        build.build_library()
    binding.lib()
    return binding


A = 1 << 20                                      # an aligned address that is never looked at
EINVAL, ENULL, EWORKSPACE = -1, -2, -3


def _cache(saw, **kw):
    f = dict(k_codes=A, v_codes=A, k_meta=A, v_meta=A, num_pages=64, n_kv_heads=8, page_size=16, head_dim=128, had_block=128, rotate_mask=3,
             sign_bits=(ctypes.c_uint32 * 4)(), dense_rot=None)
    f.update(kw)
    return saw.SawCacheStruct(**f)


PROMPT = dict(q=A, k=A, v=A, dtype=2, head_dim=128, n_q_heads=32, n_kv_heads=8, T_q=100, T_k=100, q_stride=4096, k_stride=1024, v_stride=1024, cu_q=A, cu_k=A,
              B=2, max_k_len=0, causal=1, sm_scale=0.0, out=A, workspace=A, workspace_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), EINVAL), (dict(dtype=0), EINVAL), (dict(head_dim=96), EINVAL), (dict(n_q_heads=24), EINVAL), (dict(n_q_heads=20), EINVAL),
    (dict(n_kv_heads=0), EINVAL), (dict(n_q_heads=0), EINVAL), (dict(T_q=-1), EINVAL), (dict(T_k=-1), EINVAL), (dict(T_q=1 << 31), EINVAL), (dict(T_q=1 << 26), EINVAL), (dict(T_k=(1 << 31) - 1), EINVAL), (dict(B=0), EINVAL),
    (dict(B=65536), EINVAL), (dict(q_stride=4088), EINVAL), (dict(q_stride=4100), EINVAL), (dict(k_stride=1016), EINVAL), (dict(v_stride=1020), EINVAL),
    (dict(k_stride=1028), EINVAL), (dict(sm_scale=math.nan), EINVAL), (dict(sm_scale=math.inf), EINVAL), (dict(q=None), ENULL), (dict(k=None), ENULL),
    (dict(v=None), ENULL), (dict(cu_q=None), ENULL), (dict(cu_k=None), ENULL), (dict(out=None), ENULL), (dict(workspace=None), ENULL), (dict(q=A + 8), EINVAL),
    (dict(k=A + 2), EINVAL), (dict(v=A + 8), EINVAL), (dict(out=A + 8), EINVAL), (dict(workspace=A + 4), EINVAL), (dict(cu_q=A + 2), EINVAL), (dict(cu_k=A + 1), EINVAL),
    (dict(workspace_bytes=15), EWORKSPACE), (dict(T_q=4, T_k=1 << 20, workspace_bytes=1 << 12), EWORKSPACE), (dict(T_q=0, q=None, out=None), 0)], ids=str)
def test_prompt_refusals(saw, change, code):
    assert saw.lib().saw_prompt_attn(*{**PROMPT, **change}.values()) == code


PAGED = dict(cache=None, q=A, dtype=2, T=100, q_stride=4096, n_q_heads=32, cu_q=A, B=2, page_table=A, max_pages=100, seq_lens=A, max_seq_len=0, sm_scale=0.0,
             out=A, workspace=A, workspace_bytes=1 << 40, stream=None)
SHARED = [(dict(dtype=3), EINVAL), (dict(n_q_heads=12), EINVAL), (dict(n_q_heads=128), EINVAL), (dict(T=-1), EINVAL), (dict(T=1 << 26), EINVAL), (dict(max_pages=(1 << 27) - 1), EINVAL), (dict(q_stride=4095), EINVAL),
          (dict(q_stride=4104 - 4), EINVAL), (dict(B=0), EINVAL), (dict(B=65536), EINVAL), (dict(max_pages=0), EINVAL), (dict(max_pages=1 << 28), EINVAL),
          (dict(max_seq_len=1601), EINVAL), (dict(sm_scale=math.nan), EINVAL), (dict(q=None), ENULL), (dict(cu_q=None), ENULL), (dict(page_table=None), ENULL),
          (dict(seq_lens=None), ENULL), (dict(workspace=None), ENULL), (dict(q=A + 8), EINVAL), (dict(workspace=A + 8), EINVAL), (dict(workspace_bytes=8), EWORKSPACE)]
CACHES = [(dict(head_dim=96), EINVAL), (dict(page_size=32), EINVAL), (dict(had_block=8), EINVAL), (dict(had_block=128, head_dim=64), EINVAL), (dict(rotate_mask=4), EINVAL),
          (dict(num_pages=0), EINVAL), (dict(k_codes=None), ENULL), (dict(k_meta=None), ENULL), (dict(k_codes=A + 4), EINVAL), (dict(k_meta=A + 8), EINVAL),
          (dict(dense_rot=A, head_dim=64, had_block=64), EINVAL)]


@pytest.mark.parametrize("change,code", SHARED + [(dict(out=None), ENULL), (dict(out=A + 8), EINVAL)], ids=str)
def test_paged_prompt_refusals(saw, change, code):
    c = _cache(saw)
    assert saw.lib().saw_paged_prompt_attn(*{**PAGED, "cache": ctypes.byref(c), **change}.values()) == code


@pytest.mark.parametrize("change,code", CACHES + [(dict(v_codes=None), ENULL), (dict(v_meta=A + 8), EINVAL)], ids=str)
def test_paged_prompt_refuses_caches(saw, change, code):
    c = _cache(saw, **change)
    assert saw.lib().saw_paged_prompt_attn(*{**PAGED, "cache": ctypes.byref(c)}.values()) == code
    assert saw.lib().saw_paged_prompt_attn(*PAGED.values()) == ENULL


WEIGHTS = dict(cache=None, q=A, dtype=2, T=100, q_stride=4096, n_q_heads=32, cu_q=A, B=2, page_table=A, max_pages=100, seq_lens=A, max_seq_len=0, sm_scale=0.0,
               prev=A, scores=A, score_stride=1600, workspace=A, workspace_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,code", SHARED + [(dict(scores=None), ENULL), (dict(score_stride=1599), EINVAL), (dict(prev=A + 2), EINVAL), (dict(scores=A + 1), EINVAL)], ids=str)
def test_weights_refusals(saw, change, code):
    c = _cache(saw)
    assert saw.lib().saw_paged_attn_weights(*{**WEIGHTS, "cache": ctypes.byref(c), **change}.values()) == code


@pytest.mark.parametrize("scale", [3e38, -math.inf, math.inf, math.nan])
def test_logit_scales_beyond_fp32_are_refused(saw, scale):
    """Logits are taken in log2 units: the scale times log2(e) has to be a number, or a logit of zero would be none."""
    r = ctypes.byref(_cache(saw))
    assert saw.lib().saw_prompt_attn(*{**PROMPT, "sm_scale": scale}.values()) == EINVAL
    assert saw.lib().saw_paged_prompt_attn(*{**PAGED, "cache": r, "sm_scale": scale}.values()) == EINVAL
    assert saw.lib().saw_paged_attn_weights(*{**WEIGHTS, "cache": r, "sm_scale": scale}.values()) == EINVAL


def test_grids_beyond_32_bits_are_refused(saw):
    """Launches are counted in 32 bits of threads, and the weights' groups of rows in 16."""
    wide = dict(n_kv_heads=1024, n_q_heads=1024, T_q=1, q_stride=1024 * 128, k_stride=1024 * 128, v_stride=1024 * 128, B=65535)
    assert saw.lib().saw_prompt_attn(*{**PROMPT, **wide}.values()) == EINVAL
    many = _cache(saw, n_kv_heads=1024)
    assert saw.lib().saw_paged_prompt_attn(*{**PAGED, "cache": ctypes.byref(many), "n_q_heads": 1024, "q_stride": 1024 * 128, "T": 1, "B": 65535}.values()) == EINVAL
    c = _cache(saw)
    assert saw.lib().saw_paged_attn_weights(*{**WEIGHTS, "cache": ctypes.byref(c), "T": 1 << 22}.values()) == EINVAL


@pytest.mark.parametrize("change,code", CACHES, ids=str)
def test_weights_refuse_caches(saw, change, code):
    c = _cache(saw, **change)
    assert saw.lib().saw_paged_attn_weights(*{**WEIGHTS, "cache": ctypes.byref(c)}.values()) == code


EVICT = dict(cache=None, scores=A, score_stride=1600, page_table=A, max_pages=100, seq_lens=A, B=2, max_seq_len=0, budget=500, recent=10, dst=A, dst_pages=32, new_lens=A,
             kept=A, scores_out=A, score_out_stride=500, workspace=None, workspace_bytes=0, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(score_stride=1599), EINVAL), (dict(max_pages=0), EINVAL), (dict(B=0), EINVAL), (dict(B=65536), EINVAL), (dict(max_seq_len=1601), EINVAL), (dict(budget=0), EINVAL),
    (dict(recent=-1), EINVAL), (dict(recent=501), EINVAL), (dict(dst_pages=31), EINVAL), (dict(score_out_stride=499), EINVAL), (dict(scores=None), ENULL),
    (dict(page_table=None), ENULL), (dict(seq_lens=None), ENULL), (dict(dst=None), ENULL), (dict(new_lens=None), ENULL), (dict(kept=None), ENULL), (dict(scores=A + 2), EINVAL),
    (dict(kept=A + 2), EINVAL), (dict(scores_out=A + 2), EINVAL), (dict(workspace=A + 8), EINVAL), (dict(max_pages=2000, score_stride=32000), ENULL),
    (dict(max_pages=2000, score_stride=32000, workspace=A, workspace_bytes=100), EWORKSPACE)], ids=str)
def test_evict_refusals(saw, change, code):
    c = _cache(saw)
    assert saw.lib().saw_evict_pages(*{**EVICT, "cache": ctypes.byref(c), **change}.values()) == code


@pytest.mark.parametrize("change,code", [(dict(head_dim=96), EINVAL), (dict(page_size=8), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(v_codes=None), ENULL),
                                         (dict(k_codes=A + 8), EINVAL), (dict(v_meta=A + 4), EINVAL)], ids=str)
def test_evict_refuses_caches(saw, change, code):
    c = _cache(saw, **change)
    assert saw.lib().saw_evict_pages(*{**EVICT, "cache": ctypes.byref(c)}.values()) == code


@pytest.mark.parametrize("budget,code", [((1 << 31) - 1, EINVAL), (0x7fff0001, EINVAL)])
def test_budgets_beyond_the_counters_are_refused(saw, budget, code):
    """Positions and kept tokens are counted in 32 bits in steps of a block, as lengths are."""
    c = _cache(saw)
    wide = dict(budget=budget, dst_pages=1 << 27, score_out_stride=1 << 32)
    assert saw.lib().saw_evict_pages(*{**EVICT, "cache": ctypes.byref(c), **wide}.values()) == code


def test_workspaces(saw):
    L, c = saw.lib(), _cache(saw)
    r = ctypes.byref(c)
    assert L.saw_prompt_workspace_bytes(128, 32, 8, 1000, 4, 1000) > 0
    for bad in [(96, 32, 8, 10, 1, 10), (128, 24, 8, 10, 1, 10), (128, 32, 0, 10, 1, 10), (128, 32, 8, -1, 1, 10), (128, 32, 8, 10, 0, 10), (128, 32, 8, 10, 1, -1)]:
        assert L.saw_prompt_workspace_bytes(*bad) == 0
    # a few queries over a long context are split, many are not
    assert L.saw_prompt_workspace_bytes(128, 32, 8, 16, 1, 100000) > L.saw_prompt_workspace_bytes(128, 32, 8, 16, 1, 200)
    assert L.saw_prompt_workspace_bytes(128, 32, 8, 8192, 1, 8192) == 16
    for f in (L.saw_paged_prompt_workspace_bytes, L.saw_attn_weights_workspace_bytes):
        assert f(r, 32, 100, 4, 1000) > 0 and f(None, 32, 100, 4, 1000) == 0 and f(r, 24, 100, 4, 1000) == 0 and f(r, 32, 100, 4, 0) == 0 and f(r, 32, -1, 4, 10) == 0
    assert L.saw_evict_workspace_bytes(r, 1, 131072) > 0 and L.saw_evict_workspace_bytes(r, 4, 1000) == 0 and L.saw_evict_workspace_bytes(None, 1, 1000) == 0


def test_the_binding_sizes_scratch_for_every_bound_that_the_call_takes(saw):
    """<= 0 stands for all keys; a bound above their number, whatever its size, for their number."""
    q, k = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(5000, 2, 128, dtype=torch.bfloat16)
    need = saw.prompt_workspace_bytes(q, k, 1, 5000)
    assert need > 16
    for bound in (0, -1, -(1 << 40), 5001, 1 << 31, 1 << 40):
        assert saw.prompt_workspace_bytes(q, k, 1, bound) == need
    assert saw.prompt_workspace_bytes(q, k, 1, 400) < need


def test_scratch_is_asked_for_where_it_is_used(saw):
    """Records of split keys or for a learned rotation of V, rotated queries for one of K; nothing of rows otherwise."""
    L = saw.lib()
    rows, record, query = 2048 * 32, 130 * 4, 128 * 2 + 4
    for kw, each in ((dict(), 0), (dict(dense_rot=A), record + query), (dict(dense_rot=A, rotate_mask=1), query), (dict(dense_rot=A, rotate_mask=2), record),
                     (dict(dense_rot=A, rotate_mask=0), 0)):
        need = L.saw_paged_prompt_workspace_bytes(ctypes.byref(_cache(saw, **kw)), 32, 2048, 1, 18432)
        assert rows * each < need <= rows * each + 64, kw
    r = ctypes.byref(_cache(saw))
    assert L.saw_paged_prompt_workspace_bytes(r, 32, 160, 32, 4096) >= 2 * 160 * 32 * record       # (few rows: split)
    assert L.saw_paged_prompt_attn(*{**PAGED, "cache": r, "T": 2048, "B": 1, "max_pages": 1152, "workspace_bytes": 31}.values()) == EWORKSPACE


def test_workspaces_without_queries(saw):
    L, r = saw.lib(), ctypes.byref(_cache(saw))
    for B in (1, 7, 65535):
        assert L.saw_prompt_workspace_bytes(128, 32, 8, 0, B, 1000) == 16
        assert 0 < L.saw_paged_prompt_workspace_bytes(r, 32, 0, B, 1000) <= 64 and L.saw_attn_weights_workspace_bytes(r, 32, 0, B, 1000) > 0
    assert L.saw_prompt_attn(*{**PROMPT, "T_q": 0}.values()) == 0


@pytest.fixture(params=["native", "ctypes"])
def marshal(request, saw):
    if request.param == "ctypes":
        from paper_2604_19157_amd import marshal_ctypes
        return marshal_ctypes
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        try:
            return saw._marshal()
        except Warning:
            pytest.skip("the native module is not built")


def test_the_binding_turns_down_tensors_it_cannot_pass_on(saw, marshal):
    """Types, shapes, layouts and places of tensors; each call below would be answered if the change were not there and the tensors were on a GPU."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, k = torch.zeros(6, 4, 128, dtype=torch.bfloat16), torch.zeros(6, 2, 128, dtype=torch.bfloat16)
    ws, cu, lens, pt = torch.zeros(1 << 12, dtype=torch.uint8), i32(3), i32(2), i32(2, 8)
    cache = saw.Cache(8, 2, 128, 128, device="cpu")
    rec = torch.zeros(2, 2, 128)

    def refused(call, args, changes):
        for at, x in [(None, None), *changes]:
            a = list(args)
            if at is not None:
                a[at] = x
            with pytest.raises((AssertionError, TypeError, KeyError)):
                call(*a)

    strided = torch.zeros(6, 128, 4, dtype=torch.bfloat16).transpose(1, 2)
    refused(marshal.prompt, (q, k, k, cu, cu, 0, True, 0.0, torch.zeros_like(q), ws),
            [(0, strided), (1, k.half()), (2, k[:5]), (3, cu.long()), (4, i32(4)), (3, i32(1)), (8, torch.zeros(6, 4, 128)), (8, strided), (9, torch.zeros(64, 64)[:, :8])])
    refused(marshal.paged_prompt, (cache, q, cu, pt, lens, 0, 0.0, torch.zeros_like(q), ws),
            [(1, q[..., :64]), (2, i32(4)), (3, i32(3, 8)), (3, i32(2, 16)[:, ::2]), (4, lens.long()), (5, 1 << 33), (7, q.float())])
    refused(marshal.attn_weights, (cache, q, cu, pt, lens, None, rec, 0, 0.0, ws),
            [(5, rec[..., :64]), (5, torch.zeros(2, 2, 64)), (6, rec.double()), (6, torch.zeros(2, 3, 128)), (2, i32(2)), (7, -(1 << 40))])
    refused(marshal.evict, (cache, rec, pt, lens, i32(2, 2), 20, 0, 0, i32(2), i32(2, 2, 20), None, None),
            [(1, rec.half()), (4, i32(3, 2)), (5, (1 << 32) + 20), (8, i32(3)), (9, i32(2, 2, 21)), (10, torch.zeros(2, 2, 20, dtype=torch.float64)), (11, torch.zeros(8, 8)[:, :2])])


def test_both_ways_to_marshal_have_the_same_calls(saw):
    from paper_2604_19157_amd import marshal_ctypes
    native = saw._marshal()
    for name in ("prompt", "paged_prompt", "attn_weights", "evict"):
        assert callable(getattr(native, name)) and callable(getattr(marshal_ctypes, name))
