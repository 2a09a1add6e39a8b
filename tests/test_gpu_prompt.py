"""saw_prompt_attn against attention in 64 bits, within bounds worked out per output (packed_cases)."""
import numpy as np
import pytest
import torch

import packed_cases as pc

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def saw():
    from paper_2604_19157_amd import binding
    binding.lib()
    return binding


def _run(saw, n_q, n_k, Hkv, G, d, dtype, causal=True, seed=0, sm_scale=0.0):
    cu_q, cu_k = pc.offsets(n_q), pc.offsets(n_k)
    q, k, v = pc.rand((cu_q[-1], Hkv * G, d), seed, dtype), pc.rand((cu_k[-1], Hkv, d), seed + 1, dtype), pc.rand((cu_k[-1], Hkv, d), seed + 2, dtype)
    got = saw.prompt_attn(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(cu_q).cuda(), torch.from_numpy(cu_k).cuda(), causal=causal, sm_scale=sm_scale)
    torch.cuda.synchronize()
    want, tol = pc.prompt_reference(q, k, v, cu_q, cu_k, causal, sm_scale or None)
    pc.check(got, want, tol)


LENGTHS = [[1], [2, 1, 3], [0, 5, 0, 33], [64, 65, 63], [31, 32, 33, 127], [257], [130, 400, 1, 0]]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_causal(saw, lengths, G, d, dtype):
    _run(saw, lengths, lengths, 2, G, d, dtype, seed=len(lengths))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 8), (128, 1)])
def test_every_query_sees_every_key(saw, d, G, dtype):
    _run(saw, [1, 40, 0, 129], [7, 201, 5, 64], 2, G, d, dtype, causal=False)


@pytest.mark.parametrize("n_q,n_k", [([5, 1, 17], [700, 513, 64]), ([40, 9], [1, 0]), ([100, 3, 65], [37, 3, 66]), ([2], [2500]), ([130, 1], [1999, 1024])], ids=str)
@pytest.mark.parametrize("d,G", [(128, 4), (64, 2), (128, 8)])
def test_more_and_fewer_keys_than_queries(saw, n_q, n_k, d, G):
    """A prefix without queries in front; queries in front of all keys, whose rows are zero."""
    _run(saw, n_q, n_k, 2, G, d, BF)
    _run(saw, n_q, n_k, 1, G, d, FP)


def test_rows_that_see_nothing_are_zero(saw):
    cu_q, cu_k = pc.offsets([6, 3]), pc.offsets([2, 0])
    q, k = pc.rand((9, 4, 128), 1, BF).cuda(), pc.rand((2, 2, 128), 2, BF).cuda()
    out = torch.full_like(q, 7.0)
    saw.prompt_attn(q, k, k, torch.from_numpy(cu_q).cuda(), torch.from_numpy(cu_k).cuda(), out=out)
    assert torch.count_nonzero(out[:4]) == 0 and torch.count_nonzero(out[6:]) == 0 and torch.count_nonzero(out[4:6]) > 0


@pytest.mark.parametrize("scale", [0.03, 0.5])
def test_logit_scale(saw, scale):
    _run(saw, [70], [70], 2, 2, 128, FP, sm_scale=scale)


@pytest.mark.parametrize("d,G", [(128, 4), (64, 1)])
def test_tokens_at_a_stride(saw, d, G):
    """Queries, keys and values as slices of one projection's output."""
    Hkv, cu = 2, pc.offsets([50, 0, 77])
    x = pc.rand((127, (G + 2) * Hkv * d + 8), 5, BF).cuda()
    q = x[:, :G * Hkv * d].unflatten(1, (G * Hkv, d))
    k, v = (x[:, (G + i) * Hkv * d:(G + i + 1) * Hkv * d].unflatten(1, (Hkv, d)) for i in (0, 1))
    cq = torch.from_numpy(cu).cuda()
    got = saw.prompt_attn(q, k, v, cq)
    want, tol = pc.prompt_reference(q.cpu().contiguous(), k.cpu().contiguous(), v.cpu().contiguous(), cu, cu, True)
    pc.check(got, want, tol)
    assert torch.equal(got, saw.prompt_attn(q.contiguous(), k.contiguous(), v.contiguous(), cq))


def test_strides_beyond_32_bits(saw):
    """Tokens 2^21 elements apart: the last lie behind 2^32 elements."""
    far = torch.empty((2100, 1 << 21), dtype=BF, device="cuda")
    x = [pc.rand((2100, h, 128), 7 + i, BF).cuda() for i, h in enumerate((4, 2, 2))]
    views, at = [], 64
    for t in x:
        v = far[:, at:at + t[0].numel()].unflatten(1, t.shape[1:])
        v.copy_(t)
        views.append(v)
        at += t[0].numel()
    cu = torch.tensor([0, 2000, 2100], dtype=torch.int32, device="cuda")
    assert torch.equal(saw.prompt_attn(*views, cu), saw.prompt_attn(*x, cu))


@pytest.mark.parametrize("d", [128, 64])
def test_rows_of_no_sequence_are_left_as_they_were(saw, d):
    q, k = pc.rand((200, 8, d), 3, BF).cuda(), pc.rand((200, 2, d), 4, BF).cuda()
    out = torch.full_like(q, 3.0)
    cu = np.array([10, 60, 150], np.int32)
    saw.prompt_attn(q, k, k, torch.from_numpy(cu).cuda(), out=out)
    want, tol = pc.prompt_reference(q.cpu(), k.cpu(), k.cpu(), cu, cu, True)
    pc.check(out[10:150], want[10:150], tol[10:150])
    assert bool((out[:10] == 3).all()) and bool((out[150:] == 3).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,d,G", [(BF, 128, 4), (FP, 64, 2), (FP, 128, 8)])
def test_masked_keys_and_values_count_for_nothing(saw, bad, dtype, d, G):
    """Whatever stands in keys and values that a query does not see, also in its neighbours' sequences, its row is the same."""
    n = [20, 150, 33]
    cu = pc.offsets(n)
    q, k, v = pc.rand((203, 2 * G, d), 1, dtype), pc.rand((203, 2, d), 2, dtype), pc.rand((203, 2, d), 3, dtype)
    cq = torch.from_numpy(cu).cuda()
    clean = saw.prompt_attn(q.cuda(), k.cuda(), v.cuda(), cq)
    for at in (60, 120, 169):                         # of the second sequence, whose later rows see them
        for which in (0, 1):
            k2, v2 = k.clone(), v.clone()
            (k2, v2)[which][at] = bad
            got = saw.prompt_attn(q.cuda(), k2.cuda(), v2.cuda(), cq)
            same = torch.ones(203, dtype=torch.bool)
            same[at:170] = False
            want, tol = pc.prompt_reference(q, k, v, cu, cu, True)
            pc.check(got[same.cuda()], want[same.numpy()], tol[same.numpy()], (at, which))
            if which == 1 or bad != -float("inf"):
                assert not torch.isfinite(got[at:170].float()).all(-1).any() or which == 0
    assert torch.isfinite(clean.float()).all()


def test_an_infinite_value_shows_where_it_is_seen(saw):
    q, k, v = (pc.rand((90, 2, 128), s, BF).cuda() for s in (1, 2, 3))
    v[30, :, 5] = float("inf")
    out = saw.prompt_attn(q, k, v, torch.tensor([0, 90], dtype=torch.int32).cuda())
    assert torch.isfinite(out[:30].float()).all() and torch.isinf(out[30:, :, 5]).all()
    assert torch.isfinite(out[30:, :, :5].float()).all() and torch.isfinite(out[30:, :, 6:].float()).all()


def test_a_row_of_minus_infinities_is_zero(saw):
    """Logits of -infinity have no weight; a row that has no others is zero."""
    q, k, v = torch.ones((3, 2, 64), dtype=BF).cuda(), pc.rand((3, 2, 64), 2, BF).cuda(), pc.rand((3, 2, 64), 3, BF).cuda()
    k[0] = -float("inf")
    out = saw.prompt_attn(q, k, v, torch.tensor([0, 3], dtype=torch.int32).cuda())
    assert torch.count_nonzero(out[0]) == 0
    want, tol = pc.prompt_reference(q[1:2].cpu(), k[1:2].cpu(), v[1:2].cpu(), [0, 1], [0, 1], True)
    pc.check(out[1:2], want, tol)


@pytest.mark.parametrize("shift", [0.0, 60.0, -60.0])
def test_large_logits_of_either_sign(saw, shift):
    """A common part of every logit of a row changes nothing but the maximum: keys are k + shift c along q's common channel."""
    d = 64
    q, k, v = pc.rand((65, 2, d), 1, FP), pc.rand((65, 2, d), 2, FP), pc.rand((65, 2, d), 3, FP)
    q[..., 0], k[..., 0] = 2.0, shift
    got = saw.prompt_attn(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, 65], dtype=torch.int32).cuda())
    want, tol = pc.prompt_reference(q, k, v, [0, 65], [0, 65], True)
    pc.check(got, want, tol)


def test_offsets_outside_the_tensors_are_clamped(saw):
    q, k = pc.rand((40, 4, 128), 1, BF).cuda(), pc.rand((40, 2, 128), 2, BF).cuda()
    out = torch.full_like(q, 3.0)
    cu = torch.tensor([-5, 30, 90], dtype=torch.int32).cuda()
    saw.prompt_attn(q, k, k, cu, out=out)
    want, tol = pc.prompt_reference(q.cpu(), k.cpu(), k.cpu(), [0, 30, 40], [0, 30, 40], True)
    pc.check(out, want, tol)


@pytest.mark.parametrize("n_q,n_k", [([33, 200, 1], [33, 200, 1]), ([4, 2], [1500, 900])], ids=str)
def test_captured_and_replayed_on_another_stream(saw, n_q, n_k):
    cu_q, cu_k = (torch.from_numpy(pc.offsets(n)).cuda() for n in (n_q, n_k))
    q, k, v = pc.rand((sum(n_q), 8, 128), 1, BF).cuda(), pc.rand((sum(n_k), 2, 128), 2, BF).cuda(), pc.rand((sum(n_k), 2, 128), 3, BF).cuda()
    ws = torch.empty(saw.prompt_workspace_bytes(q, k, len(n_q)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    saw.prompt_attn(q, k, v, cu_q, cu_k, out=out, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        saw.prompt_attn(q, k, v, cu_q, cu_k, out=out, workspace=ws)
    for i in range(3):
        q.copy_(pc.rand(q.shape, 10 + i, BF))
        ws.fill_(0xff)
        out.fill_(9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        again = saw.prompt_attn(q, k, v, cu_q, cu_k)
        assert torch.equal(out, again)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = saw.prompt_attn(q, k, v, cu_q, cu_k)
    here = saw.prompt_attn(q, k, v, cu_q, cu_k)
    torch.cuda.synchronize()
    assert torch.equal(other, here)


@pytest.mark.parametrize("d,G,Hkv,n,n_k", [(128, 8, 2, 5120, 5120), (64, 8, 16, 600, 630)])
def test_long_prompts(saw, d, G, Hkv, n, n_k):
    """Long enough for the large blocks: rows at the ends and around a block's border, of the first and last heads."""
    q, k, v = pc.rand((n, Hkv * G, d), 1, BF), pc.rand((n_k, Hkv, d), 2, BF), pc.rand((n_k, Hkv, d), 3, BF)
    got = saw.prompt_attn(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([0, n_k], dtype=torch.int32).cuda()).cpu()
    for g in (0, Hkv - 1):
        heads = slice(g * G, (g + 1) * G)
        for i in [0, 1, 31, 32, 33, 63, 64, n // 2 + 5, n - 33, n - 1]:
            L = n_k - n + i + 1
            want, tol = pc.prompt_reference(q[i:i + 1, heads], k[:L, g:g + 1], v[:L, g:g + 1], [0, 1], [0, L], True)
            pc.check(got[i:i + 1, heads], want, tol, (g, i))


def test_no_queries_is_a_no_op(saw):
    q, k = torch.empty((0, 4, 128), dtype=BF, device="cuda"), pc.rand((5, 2, 128), 1, BF).cuda()
    assert saw.prompt_attn(q, k, k, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor([0, 5], dtype=torch.int32).cuda()).shape == (0, 4, 128)


@pytest.mark.parametrize("causal", [True, False])
def test_no_keys_at_all(saw, causal):
    q, k = pc.rand((7, 4, 128), 1, BF).cuda(), torch.empty((0, 2, 128), dtype=BF, device="cuda")
    cu = torch.tensor([0, 3, 7], dtype=torch.int32, device="cuda")
    assert torch.count_nonzero(saw.prompt_attn(q, k, k, cu, torch.zeros_like(cu), causal=causal, out=torch.full_like(q, 4.0))) == 0


@pytest.mark.parametrize("bound", [-1, 10 ** 12])
def test_bounds_below_zero_and_beyond_the_keys(saw, bound):
    """They stand for the number of keys."""
    q, k, v = pc.rand((3, 4, 128), 1, BF).cuda(), pc.rand((5000, 2, 128), 2, BF).cuda(), pc.rand((5000, 2, 128), 3, BF).cuda()
    cu_q, cu_k = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, 5000], dtype=torch.int32, device="cuda")
    assert torch.equal(saw.prompt_attn(q, k, v, cu_q, cu_k, max_k_len=bound), saw.prompt_attn(q, k, v, cu_q, cu_k))


def test_many_sequences(saw):
    rng = np.random.default_rng(3)
    n = rng.integers(0, 9, 300).tolist()
    _run(saw, n, [x + int(e) for x, e in zip(n, rng.integers(0, 40, 300))], 1, 4, 64, BF)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,n,L,d", [(300, 1, 4000, 64), (2, 1, 4000, 128), (300, 40, 2000, 128), (1, 6000, 6000, 64)])
def test_many_small_weights(saw, B, n, L, d, dtype):
    """One key of nearly all the weight and no value, thousands of 2^-25.2 of its weight each: the output is what they give.  Off by the roundings of
    output and weight and, fp16, by 2^-32 of the largest weight for each key (logits are exact: 17.5, 0)."""
    sink, tail = 17.5, 4.0
    q, k = torch.zeros((B * n, 8, d), dtype=dtype, device="cuda"), torch.zeros((B * L, 1, d), dtype=dtype, device="cuda")
    v = torch.full_like(k, tail)
    q[..., 0] = 1
    k[::L, :, 0] = sink
    v[::L] = 0
    cu_q, cu_k = (torch.arange(0, B * x + 1, x, dtype=torch.int32, device="cuda") for x in (n, L))
    got = saw.prompt_attn(q, k, v, cu_q, cu_k, sm_scale=1.0).double().cpu().numpy()
    seen = np.tile(np.arange(L - n, L), B).astype(np.float64)[:, None, None]
    small = np.exp(-sink)
    want = tail * seen * small / (1 + seen * small)
    # (fp16 outputs below 2^-14: half of fp16's smallest step)
    tol = want * (2 * pc.U[dtype] + 2.0 ** -18 + L * 2.0 ** -22) * 1.01 + tail * L * 2.0 ** -32 + (2.0 ** -25 if dtype == FP else 0)
    assert (np.abs(got - want) <= tol).all(), np.nanmax(np.abs(got - want) / tol)


def _odd_values(v, seed, count):
    """v with `count` elements that are no numbers, and what is left of it with zeros there."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randint(v.numel(), (count,), generator=g)
    odd = v.clone()
    odd.view(-1)[at] = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=v.dtype)[torch.randint(3, (count,), generator=g)]
    return odd, torch.where(torch.isfinite(odd), odd, torch.zeros_like(odd))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 8), (128, 1)])
@pytest.mark.parametrize("n_q,n_k,causal", [([20, 150, 33], [20, 150, 33], True), ([300], [300], True), ([3, 70], [2500, 90], True), ([40, 9], [200, 70], False)], ids=str)
def test_values_that_are_no_numbers_show_where_they_are_seen(saw, n_q, n_k, causal, d, G, dtype):
    cu_q, cu_k = pc.offsets(n_q), pc.offsets(n_k)
    q, k, v = pc.rand((cu_q[-1], 2 * G, d), 1, dtype), pc.rand((cu_k[-1], 2, d), 2, dtype), pc.rand((cu_k[-1], 2, d), 3, dtype)
    for count in (1, 40, 2000):
        odd, rest = _odd_values(v, count, count)
        got = saw.prompt_attn(q.cuda(), k.cuda(), odd.cuda(), torch.from_numpy(cu_q).cuda(), torch.from_numpy(cu_k).cuda(), causal=causal)
        want, tol = pc.prompt_reference(q, k, rest, cu_q, cu_k, causal)
        pc.check_odd(got, want, tol, odd.double().numpy(), cu_q, cu_k, causal, G, count)


def test_an_infinite_value_of_hardly_any_weight(saw):
    """Its channel is infinite whatever the weight is rounded to."""
    q, k = torch.ones((8, 2, 64), dtype=FP).cuda(), torch.zeros((100, 1, 64), dtype=FP).cuda()
    v = pc.rand((100, 1, 64), 3, FP).cuda()
    k[7, :, 0] = 300
    v[50, :, 9], v[51, :, 10] = float("inf"), -float("inf")
    out = saw.prompt_attn(q, k, v, torch.tensor([0, 8], dtype=torch.int32).cuda(), torch.tensor([0, 100], dtype=torch.int32).cuda(), sm_scale=1.0)
    assert bool((out[..., 9] == float("inf")).all()) and bool((out[..., 10] == -float("inf")).all())
    rest = [c for c in range(64) if c not in (9, 10)]
    assert torch.equal(out[..., rest], v[7, 0, rest].expand(8, 2, 62))


def test_rows_that_see_a_key_that_is_no_number(saw):
    """Rows that see a key of NaN, or one whose logit is +infinity, are NaN; a logit of -infinity has no weight; the other rows are what they were."""
    n, G, d = [20, 150, 33], 2, 64
    cu = pc.offsets(n)
    for dtype in (BF, FP):
        q, k, v = pc.rand((203, 2 * G, d), 1, dtype), pc.rand((203, 2, d), 2, dtype), pc.rand((203, 2, d), 3, dtype)
        q[..., 0] = q[..., 0].abs() + 0.5
        want, tol = pc.prompt_reference(q, k, v, cu, cu, True)
        for at in (60, 120, 169):                     # of the second sequence
            # without the key: the sequence's rows behind it over the other keys (the first of these rows sees one key less than its successor)
            rest = [20 + i for i in range(150) if 20 + i != at]
            less, less_tol = pc.prompt_reference(q[at:170], k[rest], v[rest], [0, 170 - at], [0, 149], True)
            for bad in (float("nan"), float("inf"), -float("inf")):
                k2 = k.clone()
                k2[at, :, 0] = bad
                got = saw.prompt_attn(q.cuda(), k2.cuda(), v.cuda(), torch.from_numpy(cu).cuda())
                pc.check(got[:at], want[:at], tol[:at], (at, bad))
                pc.check(got[170:], want[170:], tol[170:], (at, bad))
                if bad == -float("inf"):
                    pc.check(got[at:170], less, less_tol, at)
                else:
                    assert bool(torch.isnan(got[at:170]).all()), (at, bad)


def test_sums_of_large_values_that_do_not_overflow(saw):
    """Values of 1e36: weights 2^7.5 of the first tile's would carry a sum past fp32's range on its way."""
    q, k = torch.zeros((2, 4, 64), dtype=BF), torch.zeros((130, 2, 64), dtype=BF)
    v = (pc.rand((130, 2, 64), 3, BF).float().sign() * 1e36).to(BF)
    q[..., 0] = 1
    k[64:, :, 0] = 5.1875
    cu_q, cu_k = pc.offsets([2]), pc.offsets([130])
    got = saw.prompt_attn(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(cu_q).cuda(), torch.from_numpy(cu_k).cuda(), sm_scale=1.0)
    want, tol = pc.prompt_reference(q, k, v, cu_q, cu_k, True, 1.0)
    pc.check(got, want, tol)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_no_number_does_not_take_the_call_apart(saw, bad):
    """Seen by every row of a head, it costs a few readings of the values, not a pass key by key."""
    n = 2048
    q, k, v = pc.rand((n, 32, 128), 1, BF).cuda(), pc.rand((n, 8, 128), 2, BF).cuda(), pc.rand((n, 8, 128), 3, BF).cuda()
    cu, ws, out = torch.tensor([0, n], dtype=torch.int32).cuda(), torch.empty(1 << 26, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    call = lambda: saw.prompt_attn(q, k, v, cu, out=out, workspace=ws)  # noqa: E731
    clean = pc.milliseconds(call)
    v[0, :, 5] = bad
    odd = pc.milliseconds(call)
    assert odd < 20 * clean + 1
