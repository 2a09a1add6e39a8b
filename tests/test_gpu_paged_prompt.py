"""saw_paged_prompt_attn and saw_paged_attn_weights against attention in 64 bits over the dequantised cache, within bounds worked out per
output (packed_cases)."""
import numpy as np
import pytest
import torch

import gpu_cases as gc
import packed_cases as pc
from oracle import saw_oracle as O
from paper_2604_19157_amd import synth

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def saw():
    from paper_2604_19157_amd import binding
    binding.lib()
    return binding


class Case:
    def __init__(self, saw, n, lens, Hkv=2, G=4, d=128, h=128, mask=3, dtype=BF, signs=False, dense=False, seed=0, offsets=True):
        """A cache of random codes, scales and zero-points (any number is a stored value), queries scaled so that logits spread over a few units."""
        rng = np.random.default_rng(seed)
        self.n, self.lens, self.h, self.mask, self.d, self.G, self.Hkv = n, np.asarray(lens, np.int32), h, mask, d, G, Hkv
        pages = [(x + 15) // 16 for x in lens]
        num = sum(pages) + 3
        perm = rng.permutation(num).astype(np.int32)
        self.pt = np.full((len(lens), max(max(pages), 1)), num + 99, np.int32)
        at = 0
        for b, p in enumerate(pages):
            self.pt[b, :p] = perm[at:at + p]
            at += p
        self.ref = O.new_cache(num, Hkv, 16, d)
        for w in "kv":
            self.ref[w + "_codes"][...] = rng.integers(0, 256, self.ref[w + "_codes"].shape)
            m = self.ref[w + "_meta"]
            m[..., 0] = rng.uniform(0.02, 0.3, m.shape[:-1])
            m[..., 1] = np.where(rng.random(m.shape[:-1]) < (0.1 if offsets else 0), rng.integers(-60, 80, m.shape[:-1]), rng.integers(4, 12, m.shape[:-1]))
        self.signs = synth.random_signs(d, seed + 1) if signs else None
        self.dense = synth.random_orthogonal(d, seed + 2) if dense else None
        self.cu = pc.offsets(n)
        self.q = pc.rand((self.cu[-1], Hkv * G, d), seed + 3, dtype, 0.5)
        self.cache = saw.Cache(num, Hkv, d, h, mask, signs=self.signs, dense=self.dense)
        for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
            t = getattr(self.cache, name)
            t.copy_(torch.from_numpy(np.ascontiguousarray(self.ref[name])).reshape(t.shape))
        self.args = (self.q.cuda(), torch.from_numpy(self.cu).cuda(), torch.from_numpy(self.pt).cuda(), torch.from_numpy(self.lens).cuda())

    def weights(self):
        """(b, rows, kv head, query head, weights, largest |q||k| sum and |logit| of each row)"""
        rot = self.mask & 1
        for b, (n, L) in enumerate(zip(self.n, self.lens.tolist())):
            if n == 0 or L == 0:
                continue
            rows = slice(self.cu[b], self.cu[b + 1])
            q = self.q[rows].double().numpy()
            if rot:
                q = O.rotate(q, self.h, self.signs, self.dense)
            k = O._gather(self.ref, "k", self.pt[b], 0, L)
            for j in range(self.q.shape[1]):
                yield (b, rows, j // self.G, j) + pc.weights64(q[:, j], k[:, j // self.G], pc.visible(n, L), self.d ** -0.5)

    def step(self, which, b, g, L):
        """s (|z| + 15) of every token"""
        pos = np.arange(L)
        m = self.ref[which + "_meta"][self.pt[b][pos // 16], g, pos % 16].astype(np.float64)
        return m[:, 0] * (np.abs(m[:, 1]) + 15)

    def attention(self):
        u = pc.U[self.q.dtype]
        out, tol = np.zeros(self.q.shape), np.zeros(self.q.shape)
        for b, rows, g, j, w, top, big in self.weights():
            L = int(self.lens[b])
            v = O._gather(self.ref, "v", self.pt[b], 0, L)[:, g]
            o, A = w @ v, w @ np.abs(v)
            # (the weights' part of the bound in the rotated space: rotating back mixes a block's channels, |x R^T| <= |x| sqrt(channels mixed))
            mix = self.d if self.dense is not None else self.h
            if self.mask & 2:
                blocks = A.reshape(len(A), -1, mix) if mix > 1 else A[..., None]
                A = np.repeat(np.sqrt((blocks ** 2).sum(-1)), mix, axis=-1).reshape(A.shape)
                o = O.unrotate(o, self.h, self.signs, self.dense)
            out[rows, j] = o
            # (a value is c s - s z with the product s z rounded to fp32 and the difference once more: off by at most
            # 2^-24 s |z| + 2^-24 |x| <= 2^-23 s (|z| + 15) before it is rounded to 16 bits, also where c = z)
            off = [2.0 ** -23 * self.step(x, b, g, L) for x in "kv"]
            q = np.sqrt(self.d) * np.linalg.norm(self.q[rows, j].double().numpy(), axis=1) * self.d ** -0.5    # scale sum |q~| at most
            tol[rows, j] = pc.bound(o, A, top, big, L, self.d, u, 2.0 ** -10, 2.0 ** -10 + 2.0 ** -18, q * off[0].max())
            # (and fp16's smallest step: a weight of less than 2^-14 of the row's largest is off by 2^-25 of it, a value by 2^-31 of the largest)
            least = (2.0 ** -25 * w.max(1) * np.abs(v).max(1).sum() + 2.0 ** -31 * self.step("v", b, g, L).max())[:, None]
            tol[rows, j] += 1.01 * np.sqrt(max(mix, 1) if self.mask & 2 else 1) * ((w @ off[1])[:, None] + least)
        return out, tol


SHAPES = [([1], [1]), ([1, 1, 1], [70, 1, 200]), ([3, 0, 5], [40, 9, 5]), ([33, 64], [100, 64]), ([130], [333]), ([2, 17], [900, 1030]), ([5, 5, 5], [513, 640, 64])]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,G", [(128, 1), (128, 4), (128, 8), (64, 2), (64, 8)])
@pytest.mark.parametrize("n,lens", SHAPES, ids=str)
def test_attention(saw, n, lens, d, G, dtype):
    c = Case(saw, n, lens, G=G, d=d, h=d, dtype=dtype, seed=len(n) + d)
    want, tol = c.attention()
    pc.check(saw.paged_prompt_attn(c.cache, *c.args), want, tol)


@pytest.mark.parametrize("n,lens", [([1, 5], [200, 333]), ([150], [400])], ids=str)
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,h", [(128, 128), (64, 16), (128, 1)])
def test_attention_over_ordinary_codes(saw, d, h, dtype, n, lens):
    """Zero-points inside the codes' range, as the store writes them for values of both signs: the roundings are small against the values, so
    that the mean error is held to one and a half half steps of fp16 on top of the output's own (roundings of query, key, weight and value of like size)."""
    c = Case(saw, n, lens, d=d, h=h, dtype=dtype, seed=11, offsets=False)
    want, tol = c.attention()
    got = saw.paged_prompt_attn(c.cache, *c.args)
    pc.check(got, want, tol)
    off = np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)
    assert off < pc.U[dtype] + 1.5 * 2.0 ** -11 * max(1.0, np.abs(want).max() / np.abs(want).mean()) ** 0.5


def _half(x):
    """x as fp16 times a power of two for each row of the last axis: no number is subnormal that is not far below the largest."""
    top = np.abs(x).max(-1, keepdims=True)
    unit = 2.0 ** np.floor(np.log2(np.where(top > 0, top, 1)) - 14)
    return (x / unit).astype(np.float16).astype(np.float64) * unit


@pytest.mark.parametrize("d,h", [(128, 128), (64, 16), (128, 1)])
@pytest.mark.parametrize("n,lens,limbs", [([1, 5], [200, 333], True), ([150], [400], False), ([1], [3000], True)], ids=str)
def test_fp16_outputs_are_off_by_the_roundings_that_they_are_said_to_have(saw, n, lens, limbs, d, h):
    """Logits of a standard deviation of several units: no more than weights and values, and the queries of long chunks, as fp16 give in 64 bits.  (Norms of thousands of numbers, which vary by a few hundredths; 1.25 is not reached by chance.)"""
    c = Case(saw, n, lens, d=d, h=h, dtype=FP, seed=31, offsets=False)
    c.q.mul_(3)
    c.args[0].mul_(3)
    want, stated = np.zeros(c.q.shape), np.zeros(c.q.shape)
    for b, L in enumerate(lens):
        rows = slice(c.cu[b], c.cu[b + 1])
        q = O.rotate(c.q[rows].double().numpy(), h)
        k, v = (O._gather(c.ref, x, c.pt[b], 0, L) for x in "kv")
        for j in range(c.q.shape[1]):
            for out, qj, vj, half in ((want, q[:, j], v[:, j // 4], False), (stated, q[:, j] if limbs else _half(q[:, j]), _half(v[:, j // 4].ravel()).reshape(L, d), True)):
                w = pc.weights64(qj, k[:, j // 4], pc.visible(n[b], L), d ** -0.5)[0]
                o = O.unrotate((_half(w) if half else w) @ vj, h)
                out[rows, j] = o.astype(np.float16) if half else o
    got = saw.paged_prompt_attn(c.cache, *c.args).double().cpu().numpy()
    off, said = (np.linalg.norm(x - want) / np.linalg.norm(want) for x in (got, stated))
    assert off < 1.25 * said, (off, said)


OPTIONS = [dict(h=1), dict(h=16), dict(h=32, mask=1), dict(h=64, mask=2), dict(h=128, signs=True), dict(h=128, dense=True),
           dict(h=1, dense=True), dict(h=64, dense=True, signs=True, mask=1), dict(d=64, h=16), dict(d=64, h=64, signs=True), dict(d=64, h=1)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("options", OPTIONS, ids=str)
def test_rotations(saw, options, dtype):
    c = Case(saw, [7, 1, 40], [60, 300, 40], dtype=dtype, seed=4, **options)
    want, tol = c.attention()
    pc.check(saw.paged_prompt_attn(c.cache, *c.args), want, tol)


@pytest.mark.parametrize("options", [dict(h=128, signs=True), dict(h=1), dict(h=64, mask=1), dict(h=16, mask=2)], ids=str)
def test_many_rows_under_a_learned_rotation(saw, options):
    """Several rows at once, the last ones and those of no sequence among them."""
    c = Case(saw, [700, 0, 401], [760, 5, 430], seed=13, dense=True, **options)
    want, tol = c.attention()
    q = torch.cat([c.args[0], pc.rand((5, 8, 128), 2, BF).cuda()])
    out = torch.full_like(q, 7.0)
    saw.paged_prompt_attn(c.cache, q, *c.args[1:], out=out)
    pc.check(out[:1101], want, tol)
    assert bool((out[1101:] == 7).all())


def test_a_long_chunk(saw):
    """Blocks of 256 rows."""
    c = Case(saw, [1024], [1100], Hkv=16, G=4, seed=8)
    want, tol = c.attention()
    pc.check(saw.paged_prompt_attn(c.cache, *c.args), want, tol)


def test_queries_in_front_of_all_tokens_and_empty_sequences(saw):
    """More queries than tokens: the first rows see nothing and are zero; rows of no sequence stay as they were."""
    c = Case(saw, [6, 4, 0, 2], [2, 0, 7, 2])
    q = torch.cat([c.args[0], pc.rand((3, 8, 128), 9, BF).cuda()])
    out = torch.full_like(q, 5.0)
    saw.paged_prompt_attn(c.cache, q, *c.args[1:], out=out)
    want, tol = c.attention()
    pc.check(out[:12], want, tol)
    assert torch.count_nonzero(out[:4]) == 0 and torch.count_nonzero(out[6:10]) == 0 and bool((out[12:] == 5).all())


@pytest.mark.parametrize("n", [3, 80])
def test_scales_of_very_different_size(saw, n):
    """Scales over forty powers of two within a sequence, growing and shrinking along it; zero vectors between them."""
    for power in (1e-12, 1e9):
        c = Case(saw, [n], [400], d=128, h=1, seed=6)
        steps = np.geomspace(1, power, 400).astype(np.float32)
        for pos in range(400):
            page, slot = c.pt[0, pos // 16], pos % 16
            for w in "kv":
                c.ref[w + "_meta"][page, :, slot, 0] *= steps[pos] if w == "v" else np.float32(1e-3) * steps[pos] ** np.float32(0.25)
            if pos % 50 == 7:
                c.ref["v_meta"][page, :, slot] = (1, 0)
                c.ref["v_codes"][page, :, slot] = 0
        for name in ("k_meta", "v_meta", "v_codes"):
            t = getattr(c.cache, name)
            t.copy_(torch.from_numpy(np.ascontiguousarray(c.ref[name])).reshape(t.shape))
        want, tol = c.attention()
        pc.check(saw.paged_prompt_attn(c.cache, *c.args), want, tol, power)


def test_agrees_with_the_decode_call(saw):
    """One query a sequence is a decode step: both are within their bounds of the same numbers."""
    c = Case(saw, [1] * 6, [1, 15, 16, 333, 800, 64])
    want, tol = c.attention()
    got = saw.paged_prompt_attn(c.cache, *c.args)
    pc.check(got, want, tol)
    dec = saw.paged_decode_attn(c.cache, c.args[0], c.args[2].clamp(max=c.cache.num_pages - 1), c.args[3], out_dtype=BF)
    pc.check(dec, want, tol)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_slots_and_pages_that_are_not_seen_count_for_nothing(saw, bad):
    """Slots behind a sequence's end hold anything; tokens that a query does not see too."""
    c = Case(saw, [40, 3], [50, 21])
    want, tol = c.attention()
    clean = saw.paged_prompt_attn(c.cache, *c.args)
    for pool in (c.cache.k_meta, c.cache.v_meta):
        pool[c.pt[0, 3], :, 2:] = bad               # positions 50 on
        pool[c.pt[1, 1], :, 5:] = bad
    assert torch.equal(saw.paged_prompt_attn(c.cache, *c.args), clean)
    for pool in (c.cache.k_meta, c.cache.v_meta):
        keep = pool.clone()
        pool[c.pt[0, 2], :, 8] = bad                # position 40: rows 30 .. 39 see it
        got = saw.paged_prompt_attn(c.cache, *c.args)
        pc.check(got[:30], want[:30], tol[:30])
        pc.check(got[40:], want[40:], tol[40:])
        assert not torch.isfinite(got[30:40].float()).any()
        pool.copy_(keep)


@pytest.mark.parametrize("size", [1e-30, 1e4, 1e12, 1e30])
@pytest.mark.parametrize("n,lens", [([40, 3], [50, 21]), ([40, 3], [330, 21]), ([5, 3], [50, 21]), ([5, 3], [330, 700]), ([5], [4000]), ([300], [300])], ids=str)
def test_the_size_of_tokens_that_are_not_seen_counts_for_nothing(saw, n, lens, size):
    """A token of any finite scale: the queries in front of it give what they give without it."""
    c = Case(saw, n, lens, h=1)
    want, tol = c.attention()
    first = int(c.cu[1]) // 2                       # of sequence 0: queries from here on see the token at its end
    at = lens[0] - n[0] + first
    for pool in (c.cache.k_meta, c.cache.v_meta):
        keep = pool.clone()
        pool[c.pt[0, at // 16], :, at % 16, 0] = size
        got = saw.paged_prompt_attn(c.cache, *c.args)
        pc.check(got[:first], want[:first], tol[:first])
        pc.check(got[n[0]:], want[n[0]:], tol[n[0]:])
        pool.copy_(keep)


@pytest.mark.parametrize("size", [1e-30, 1e4, 1e30])
@pytest.mark.parametrize("d,h", [(128, 1), (128, 128), (64, 16)])
@pytest.mark.parametrize("n,lens", [([40, 3], [330, 21]), ([5, 3], [330, 700]), ([300], [300])], ids=str)
def test_the_size_of_tokens_that_are_not_seen_counts_for_nothing_in_fp16(saw, n, lens, d, h, size):
    c = Case(saw, n, lens, d=d, h=h, dtype=FP, signs=h > 1)
    want, tol = c.attention()
    first = int(c.cu[1]) // 2
    at = lens[0] - n[0] + first
    for pool in (c.cache.k_meta, c.cache.v_meta):
        keep = pool.clone()
        pool[c.pt[0, at // 16], :, at % 16, 0] = size
        got = saw.paged_prompt_attn(c.cache, *c.args)
        pc.check(got[:first], want[:first], tol[:first])
        pc.check(got[n[0]:], want[n[0]:], tol[n[0]:])
        pool.copy_(keep)


@pytest.mark.parametrize("n,lens", [([3], [50]), ([40], [330]), ([1], [5000])], ids=str)
def test_tokens_that_are_numbers_in_some_channels(saw, n, lens):
    """Codes far from the zero-point overflow fp32 and are infinite, those beside it are large numbers (bf16 has the exponents for both)."""
    c = Case(saw, n, lens, h=1, seed=23)
    at = lens[0] - n[0]                               # seen by every query
    for ref in (c.ref["v_meta"], c.cache.v_meta):
        ref[c.pt[0, at // 16], :, at % 16] = torch.tensor([1e38, 8.0]) if ref is c.cache.v_meta else (1e38, 8.0)
    with np.errstate(over="ignore"):
        v = O._gather(c.ref, "v", c.pt[0], 0, lens[0]).astype(np.float32).astype(np.float64)
    want, tol = np.zeros(c.q.shape), np.zeros(c.q.shape)
    rest = np.where(np.isfinite(v), v, 0)
    for b, rows, g, j, w, top, big in c.weights():
        want[rows, j] = w @ rest[:, g]
        # (half a step of the output, of the query and of nothing else: these rows are worked out in fp32)
        tol[rows, j] = pc.bound(want[rows, j], w @ np.abs(rest[:, g]), top, big, lens[0], c.d, pc.U[BF], 2.0 ** -10, 2.0 ** -10 + 2.0 ** -18)
    pc.check_odd(saw.paged_prompt_attn(c.cache, *c.args), want, tol, v, c.cu, pc.offsets(lens), True, c.G)


def test_page_ids_out_of_range_read_page_0(saw):
    c = Case(saw, [20], [60])
    pt = c.args[2].clone()
    pt[0, 1] = -7
    pt[0, 2] = 1 << 30
    got = saw.paged_prompt_attn(c.cache, c.args[0], c.args[1], pt, c.args[3])
    pt[0, 1:3] = 0
    assert torch.equal(got, saw.paged_prompt_attn(c.cache, c.args[0], c.args[1], pt, c.args[3]))


def test_bound_of_the_lengths(saw):
    """Lengths are clamped to max_seq_len, queries stay the last tokens of what is left."""
    c = Case(saw, [5, 2], [100, 30])
    got = saw.paged_prompt_attn(c.cache, *c.args, max_seq_len=48)
    c.lens = np.minimum(c.lens, 48)
    want, tol = c.attention()
    pc.check(got, want, tol)


def test_queries_at_a_stride(saw):
    c = Case(saw, [9, 31], [60, 31])
    wide = torch.zeros((40, 8 * 128 + 64), dtype=BF, device="cuda")
    view = wide[:, 32:32 + 8 * 128].unflatten(1, (8, 128))
    view.copy_(c.args[0])
    assert torch.equal(saw.paged_prompt_attn(c.cache, view, *c.args[1:]), saw.paged_prompt_attn(c.cache, *c.args))


def test_captured_and_replayed(saw):
    c = Case(saw, [5, 5, 33], [700, 64, 90])
    q = c.args[0].clone()
    ws = torch.empty(max(saw.paged_prompt_workspace_bytes(c.cache, q, 3, 704), saw.attn_weights_workspace_bytes(c.cache, q, 3, 704)), dtype=torch.uint8, device="cuda")
    out, scores, prev = torch.empty_like(q), torch.zeros((3, 2, 704), device="cuda"), torch.rand((3, 2, 704), device="cuda")

    def both():
        saw.paged_prompt_attn(c.cache, q, *c.args[1:], max_seq_len=704, out=out, workspace=ws)
        saw.paged_attn_weights(c.cache, q, *c.args[1:], prev=prev, scores=scores, max_seq_len=704, workspace=ws)

    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for i in range(3):
        q.copy_(pc.rand(q.shape, 20 + i, BF, 0.5))
        ws.fill_(0xff)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), scores.clone()
        both()
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(scores, got[1])


def _same_pages(saw, B, n, L, d, dtype, sink, tail):
    """B sequences of the same L tokens: the first has logit `sink` and value 0, the others logit 0 and the value `tail` in every channel."""
    Hkv, pages = 8, (L + 15) // 16
    cache = saw.Cache(pages, Hkv, d, 1)
    cache.k_codes.fill_(0x88)
    cache.v_codes.fill_(0xff)
    cache.k_codes[0, :, 0, 0] = 0x8f                 # channel 0 of the first token: 7 scales
    cache.v_codes[0, :, 0] = 0x88
    for pool, scale in ((cache.k_meta, sink / 7), (cache.v_meta, tail / 7)):
        pool[..., 0], pool[..., 1] = scale, 8
    q = torch.zeros((B * n, Hkv * 4, d), dtype=dtype, device="cuda")
    q[..., 0] = 1
    pt = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(B, 1)
    cu = torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda")
    return cache, q, cu, pt, torch.full((B,), L, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,n", [(70, 1), (70, 20), (1, 3), (1, 20), (16, 520)])
def test_many_small_weights(saw, B, n, d, dtype):
    """One token of nearly all the weight and no value, 20000 of 2^-25.2 of its weight each: the output is what they give.  Off by the roundings of
    output, weight and value and by 2^-32 of the largest weight for each token (logits are exact: 17.5, 0)."""
    L, sink, tail = 20000, 17.5, 3.5
    got = saw.paged_prompt_attn(*_same_pages(saw, B, n, L, d, dtype, sink, tail), sm_scale=1.0).double().cpu().numpy()
    seen = np.tile(np.arange(L - n, L), B).astype(np.float64)[:, None, None]           # tokens of the tail that a query sees
    small = np.exp(-sink)
    want = tail * seen * small / (1 + seen * small)
    tol = want * (pc.U[dtype] + 2.0 ** -10 + 2.0 ** -18 + L * 2.0 ** -22) * 1.01 + tail * L * 2.0 ** -32
    assert (np.abs(got - want) <= tol).all(), np.abs(got / want - 1).max()


@pytest.mark.parametrize("n,lens", [([3], [40]), ([1], [3000]), ([60], [100]), ([1], [200])], ids=str)
@pytest.mark.parametrize("options", [dict(h=1), dict(h=128), dict(h=1, dense=True)], ids=str)
def test_every_kind_of_nan_shows(saw, n, lens, options):
    """Also the one with all bits set, which memory that was never written may hold."""
    for pool in ("k_meta", "v_meta"):
        c = Case(saw, n, lens, **options)
        getattr(c.cache, pool)[c.pt[0, 0], :, 3].view(torch.int32).fill_(-1)
        assert bool(torch.isnan(saw.paged_prompt_attn(c.cache, *c.args)).all())
        if n == [1]:
            assert bool(torch.isnan(saw.paged_decode_attn(c.cache, c.args[0], c.args[2].clamp(max=c.cache.num_pages - 1), c.args[3], out_dtype=BF)).all())


@pytest.mark.parametrize("n,lens", [([7, 1], [60, 3000]), ([150], [400]), ([1300, 3], [1300, 900])], ids=str)
@pytest.mark.parametrize("options", [dict(h=128), dict(h=128, dense=True), dict(h=64, dense=True, mask=1), dict(h=64, dense=True, mask=2)], ids=str)
def test_scratch_of_the_size_asked_for(saw, options, n, lens):
    """Nothing behind it is written, and nothing of what it held counts."""
    c = Case(saw, n, lens, seed=21, **options)
    q = c.args[0]
    need = saw.paged_prompt_workspace_bytes(c.cache, q, len(n), c.pt.shape[1] * 16)
    got = []
    for fill in (0, 0xff):
        ws = torch.full((need + 4096,), fill, dtype=torch.uint8, device="cuda")
        got.append(saw.paged_prompt_attn(c.cache, *c.args, workspace=ws[:need]))
        assert bool((ws[need:] == fill).all())
    assert torch.equal(*got)
    want, tol = c.attention()
    pc.check(got[0], want, tol)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("n,lens", [([3, 5], [50, 900]), ([40, 150], [50, 160]), ([1], [6000]), ([100], [3000])], ids=str)
def test_values_that_are_no_numbers_show_where_they_are_seen(saw, n, lens, d, G, dtype):
    """Scales that are NaN or infinite: without a rotation a code above the zero-point is +infinity, one below -infinity, one at it NaN."""
    c = Case(saw, n, lens, d=d, G=G, h=1, dtype=dtype, seed=17)
    want, tol = c.attention()
    for seed, count in ((1, 1), (2, 2), (3, 12)):
        rng = np.random.default_rng(seed)
        ref = c.ref["v_meta"].copy()
        rest = c.ref["v_meta"].copy()
        for _ in range(count):
            b = rng.integers(len(n))
            at, g = rng.integers(max(0, lens[b] - 2 * n[b] - 20), lens[b]), rng.integers(2)
            ref[c.pt[b, at // 16], g, at % 16, 0] = rng.choice([np.nan, np.inf, -np.inf])
            rest[c.pt[b, at // 16], g, at % 16, 0] = 0
        keep = c.ref["v_meta"]
        c.ref["v_meta"] = rest
        want, tol = c.attention()
        c.ref["v_meta"] = ref
        with np.errstate(invalid="ignore"):
            values = np.concatenate([O._gather(c.ref, "v", c.pt[b], 0, L) for b, L in enumerate(lens)])
        c.ref["v_meta"] = keep
        c.cache.v_meta.copy_(torch.from_numpy(ref).reshape(c.cache.v_meta.shape))
        got = saw.paged_prompt_attn(c.cache, *c.args)
        pc.check_odd(got, want, tol, values, c.cu, pc.offsets(lens), True, G, count)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n,lens", [([3, 1], [50, 900]), ([40, 150], [50, 160]), ([1], [6000])], ids=str)
@pytest.mark.parametrize("pair", [(np.inf, 8.0), (-np.inf, 3.0), (np.nan, 8.0), (0.1, np.inf)], ids=str)
def test_keys_that_are_no_numbers_show_where_they_are_seen(saw, pair, n, lens, dtype):
    """A key of infinities of both signs, as queries of both signs meet them, has no logit: the rows that see it are NaN, the others what they were."""
    c = Case(saw, n, lens, dtype=dtype, seed=19)
    want, tol = c.attention()
    for back in (1, n[0] // 2 + 1):
        at = lens[0] - back                           # seen by the last `back` queries of the first sequence
        keep = c.cache.k_meta.clone()
        c.cache.k_meta[c.pt[0, at // 16], :, at % 16] = torch.tensor(pair, device="cuda")
        got = saw.paged_prompt_attn(c.cache, *c.args)
        c.cache.k_meta.copy_(keep)
        assert bool(torch.isnan(got[n[0] - back:n[0]]).all())
        pc.check(got[:n[0] - back], want[:n[0] - back], tol[:n[0] - back])
        pc.check(got[n[0]:], want[n[0]:], tol[n[0]:])


@pytest.mark.parametrize("n", [3, 80])
@pytest.mark.parametrize("size", [1.0, 1e-30])
def test_queries_of_zeros(saw, n, size):
    """A padded batch's: every token that they see weighs the same, however small the keys are."""
    c = Case(saw, [n], [300], h=1, seed=3)
    c.q.zero_()
    c.args[0].zero_()
    c.cache.k_meta[..., 0] *= size
    c.ref["k_meta"][..., 0] *= np.float32(size)
    want, tol = c.attention()
    pc.check(saw.paged_prompt_attn(c.cache, *c.args), want, tol)


@pytest.mark.parametrize("n", [8, 512])
def test_a_value_that_is_no_number_does_not_take_the_call_apart(saw, n):
    c = Case(saw, [n], [8192], Hkv=8, G=4, seed=3)
    ws, out = torch.empty(1 << 27, dtype=torch.uint8, device="cuda"), torch.empty_like(c.args[0])
    call = lambda: saw.paged_prompt_attn(c.cache, *c.args, out=out, workspace=ws)  # noqa: E731
    clean = pc.milliseconds(call)
    c.cache.v_meta[c.pt[0, 0], :, 0] = float("nan")
    odd = pc.milliseconds(call)
    assert odd < 20 * clean + 1


# ---- accumulated weights ----
def _scores(c, prev):
    """(scores, bound): a weight is off by at most w (exp(2 e) - 1 + 2^-20 + n 2^-22); then sums of as many terms as there are rows, in fp32."""
    out, tol = prev.astype(np.float64), np.zeros(prev.shape)
    rows = 1
    for b, at, g, j, w, top, big in c.weights():
        L = int(c.lens[b])
        e = top * (c.d * 2.0 ** -23 + 2.0 ** -21) + big * 2.0 ** -22
        out[b, g, :L] += w.sum(0)
        tol[b, g, :L] += (w * (np.expm1(2 * e) + 2.0 ** -20 + L * 2.0 ** -22)[:, None]).sum(0)
        rows = max(rows, c.G * (at.stop - at.start))
    return out, (tol + np.abs(out) * (rows + 2) * 2.0 ** -24) * 1.01 + 1e-30


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,G", [(128, 1), (128, 4), (128, 8), (64, 2), (64, 8)])
@pytest.mark.parametrize("n,lens", SHAPES, ids=str)
def test_weights(saw, n, lens, d, G, dtype):
    c = Case(saw, n, lens, G=G, d=d, h=d, dtype=dtype, seed=len(n) + d)
    prev = np.random.default_rng(1).random((len(n), 2, max(lens) + 21)).astype(np.float32)
    want, tol = _scores(c, prev)
    start = torch.full(prev.shape, 11.0, device="cuda")
    got = saw.paged_attn_weights(c.cache, *c.args, prev=torch.from_numpy(prev).cuda(), scores=start, max_seq_len=max(lens)).cpu()
    for b, L in enumerate(lens):
        pc.check(got[b, :, :L], want[b, :, :L], tol[b, :, :L], b)
        assert bool((got[b, :, L:] == 11).all())


@pytest.mark.parametrize("options", OPTIONS, ids=str)
def test_weights_under_rotations(saw, options):
    c = Case(saw, [7, 1, 40], [60, 300, 40], seed=4, **options)
    prev = np.zeros((3, 2, 304), np.float32)
    want, tol = _scores(c, prev)
    got = saw.paged_attn_weights(c.cache, *c.args, max_seq_len=304)
    pc.check(got, want, tol)


@pytest.mark.parametrize("n", [[1] * 40, [0, 3, 0, 1, 36] + [0] * 35], ids=["one each", "uneven"])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 8), (128, 1)])
def test_weights_of_a_decode_step(saw, n, d, G):
    """Batches that fill the chip: one launch, whose shared memory holds the logits of some sequences and not of others."""
    lens = [1, 16, 5000, 40, 300] + list(range(100, 2200, 60))
    c = Case(saw, n, lens, Hkv=8, G=G, d=d, h=d, seed=3)
    prev = np.random.default_rng(1).random((40, 8, 5003)).astype(np.float32)
    want, tol = _scores(c, prev)
    start = torch.from_numpy(prev).cuda()
    got = saw.paged_attn_weights(c.cache, *c.args, prev=start, scores=start, max_seq_len=5000).cpu()
    for b, L in enumerate(lens):
        pc.check(got[b, :, :L], want[b, :, :L], tol[b, :, :L], b)
        assert np.array_equal(got[b, :, L:].numpy(), prev[b, :, L:])


def test_weights_add_up_in_place_and_to_the_number_of_rows(saw):
    """Every row's weights sum to one; a second call on the record itself doubles it."""
    c = Case(saw, [4, 1, 0, 3], [300, 17, 9, 2])
    scores = torch.zeros((4, 2, 304), device="cuda")
    saw.paged_attn_weights(c.cache, *c.args, prev=scores, scores=scores, max_seq_len=304)
    once = scores.clone()
    total = once.double().sum(-1).cpu().numpy()
    # (the last sequence's first query sees nothing)
    assert np.abs(total - np.array([[16, 16], [4, 4], [0, 0], [8, 8]])).max() < 1e-4
    saw.paged_attn_weights(c.cache, *c.args, prev=scores, scores=scores, max_seq_len=304)
    assert torch.allclose(scores, 2 * once, rtol=2.0 ** -23, atol=0)


def test_weights_without_queries_keep_the_record(saw):
    c = Case(saw, [0, 0], [30, 5])
    prev = torch.rand((2, 2, 32), device="cuda")
    got = saw.paged_attn_weights(c.cache, *c.args, prev=prev, max_seq_len=32)
    assert torch.equal(got[0, :, :30], prev[0, :, :30]) and torch.equal(got[1, :, :5], prev[1, :, :5])
    assert torch.count_nonzero(got[1, :, 5:]) == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_weights_of_slots_that_are_not_seen(saw, bad):
    c = Case(saw, [3], [21])
    clean = saw.paged_attn_weights(c.cache, *c.args, max_seq_len=32)
    c.cache.k_meta[c.pt[0, 1], :, 5:] = bad
    assert torch.equal(saw.paged_attn_weights(c.cache, *c.args, max_seq_len=32), clean)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("lens", [[60, 30], [5000, 30], [60] + [30] * 40, [5000] + [30] * 40], ids=len)
def test_weights_of_a_query_that_is_no_number(saw, bad, lens):
    """It shows at the positions that it sees and nowhere else."""
    n = [10, 2] + [0] * (len(lens) - 2)
    c = Case(saw, n, lens, Hkv=8, seed=5)
    want, tol = _scores(c, np.zeros((len(n), 8, max(lens)), np.float32))
    only = Case(saw, [5, 2] + n[2:], lens, Hkv=8, seed=5)                  # the queries behind the fifth, alone
    only.q = torch.cat([c.q[5:10], c.q[10:]])
    behind, tol_behind = _scores(only, np.zeros((len(n), 8, max(lens)), np.float32))
    c.args[0][4] = bad
    got = saw.paged_attn_weights(c.cache, *c.args, max_seq_len=max(lens)).cpu()
    sees = lens[0] - 5                                                     # positions that query 4 of 10 sees
    assert bool(torch.isnan(got[0, :, :sees]).all())
    pc.check(got[0, :, sees:lens[0]], behind[0, :, sees:lens[0]], tol_behind[0, :, sees:lens[0]])
    pc.check(got[1:], want[1:], tol[1:])


@pytest.mark.parametrize("lens", [[60, 30], [5000, 30], [60] + [30] * 40, [5000] + [30] * 40], ids=len)
def test_weights_of_a_row_that_is_no_number_beside_an_infinite_key(saw, lens):
    """A token whose logit is -infinity is a token that the row sees: its weight is no number either."""
    n = [2] + [0] * (len(lens) - 1)
    c = Case(saw, n, lens, Hkv=8, h=1, seed=5)
    c.args[0].fill_(1)
    at = [lens[0] - 3, 1]                             # in the last tile, and in front
    for j in at:
        c.cache.k_codes[c.pt[0, j // 16], :, j % 16] = 0
        c.cache.k_meta[c.pt[0, j // 16], :, j % 16] = torch.tensor([float("inf"), 8.0], device="cuda")
    j = lens[0] - 4
    c.cache.k_meta[c.pt[0, j // 16], :, j % 16] = float("nan")
    got = saw.paged_attn_weights(c.cache, *c.args, max_seq_len=max(lens))
    assert bool(torch.isnan(got[0, :, :lens[0]]).all())


@pytest.mark.parametrize("n", [1, 2, 7])
@pytest.mark.parametrize("lens", [[60, 30], [5000, 30], [60] + [30] * 40, [5000] + [30] * 40], ids=len)
def test_weights_of_a_key_of_minus_infinity(saw, lens, n):
    """Its logits have no weight; the other positions get what they get without it."""
    c = Case(saw, [n] + [0] * (len(lens) - 1), lens, Hkv=8, h=1, seed=5)
    c.args[0].fill_(1)
    c.q.fill_(1)
    for j in (0, 17, lens[0] - n):                   # seen by every query
        where = c.pt[0, j // 16], slice(None), j % 16
        c.cache.k_codes[where] = 0
        c.cache.k_meta[where] = torch.tensor([float("inf"), 8.0], device="cuda")
        c.ref["k_codes"][where] = 0
        c.ref["k_meta"][where] = (1e4, 8.0)           # a weight of zero
    want, tol = _scores(c, np.zeros((len(lens), 8, max(lens)), np.float32))
    got = saw.paged_attn_weights(c.cache, *c.args, max_seq_len=max(lens))
    pc.check(got[0, :, :lens[0]], want[0, :, :lens[0]], tol[0, :, :lens[0]])


@pytest.mark.parametrize("n,lens,G", [([1, 1], [5000, 9000], 4), ([1], [20000], 8), ([2, 33], [7000, 3001], 2), ([1] * 40, list(range(100, 1300, 30)), 4)], ids=str)
def test_long_contexts_split(saw, n, lens, G):
    c = Case(saw, n, lens, G=G, seed=2)
    want, tol = c.attention()
    pc.check(saw.paged_prompt_attn(c.cache, *c.args), want, tol)
    prev = np.zeros((len(n), 2, max(lens)), np.float32)
    want, tol = _scores(c, prev)
    pc.check(saw.paged_attn_weights(c.cache, *c.args, prev=torch.from_numpy(prev).cuda(), max_seq_len=max(lens)), want, tol)


@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("n,lens", [([70, 0, 33], [75, 9, 300]), ([200], [1900]), ([17, 150, 64, 1], [17, 131, 640, 5])], ids=str)
def test_weights_of_many_queries_over_few_keys(saw, n, lens, d, G):
    """Wavefronts share out the rows."""
    c = Case(saw, n, lens, G=G, d=d, h=d, seed=7)
    prev = np.random.default_rng(2).random((len(n), 2, max(lens) + 5)).astype(np.float32)
    want, tol = _scores(c, prev)
    got = saw.paged_attn_weights(c.cache, *c.args, prev=torch.from_numpy(prev).cuda(), max_seq_len=max(lens)).cpu()
    for b, L in enumerate(lens):
        pc.check(got[b, :, :L], want[b, :, :L], tol[b, :, :L], b)


def test_weights_of_many_sequences_take_time_with_their_number(saw):
    """Four times the sequences: not sixteen times the blocks.  (Four times the work; eight leaves room for the clock.)"""
    took = []
    for B in (512, 2048):
        c = Case(saw, [16] * B, [40] * B, G=8, seed=2)
        ws = torch.empty(saw.attn_weights_workspace_bytes(c.cache, c.args[0], B, 48), dtype=torch.uint8, device="cuda")
        scores = torch.zeros((B, 2, 48), device="cuda")
        took.append(pc.milliseconds(lambda: saw.paged_attn_weights(c.cache, *c.args, scores=scores, max_seq_len=48, workspace=ws)))
        total = scores[..., :40].double().sum(-1)
        assert bool((total - 16 * 8).abs().max() < 1e-3)          # every row's weights sum to one
    assert took[1] < 8 * took[0], took


def test_weights_of_many_queries_over_one_long_sequence(saw):
    """A single head: wavefronts that share out the rows go over several steps of keys."""
    c = Case(saw, [90], [20000], Hkv=1, G=8, seed=9)
    prev = np.zeros((1, 1, 20000), np.float32)
    want, tol = _scores(c, prev)
    got = saw.paged_attn_weights(c.cache, *c.args, prev=torch.from_numpy(prev).cuda(), max_seq_len=20000)
    pc.check(got, want, tol)


# ---- the calls together ----
def test_pools_beyond_32_bits(saw):
    """Pages at the end of pools of 4.9 GiB of codes each: what they give at the front."""
    c = Case(saw, [5, 90], [700, 333], Hkv=8)
    num, used = 640000, c.cache.num_pages
    big = saw.Cache(num, 8, 128, 128, 3)
    for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
        getattr(big, name)[num - used:].copy_(getattr(c.cache, name))
    q, cu, pt, lens = c.args
    far = torch.where(pt < used, pt + (num - used), pt + num)
    assert torch.equal(saw.paged_prompt_attn(big, q, cu, far, lens), saw.paged_prompt_attn(c.cache, *c.args))
    scores = saw.paged_attn_weights(c.cache, *c.args)
    assert torch.equal(saw.paged_attn_weights(big, q, cu, far, lens), scores)
    dst = torch.arange(num // 2, num // 2 + 2 * 16, dtype=torch.int32, device="cuda").view(2, 16)
    _, kept, _ = saw.evict_pages(big, scores, far, lens, dst, 256, 20)
    for b in range(2):
        for g in (0, 7):
            j = kept[b, g].long()
            for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
                old, new = getattr(c.cache, name), getattr(big, name)
                assert torch.equal(new[dst[b].long(), g].flatten(0, 1), old[pt[b].long()[j // 16], g, j % 16])


def test_two_streams_at_once(saw):
    """Calls with workspaces of their own do not meet."""
    cases = [Case(saw, [5] * 8, [900 + 40 * i for i in range(8)], Hkv=8, seed=s) for s in (1, 2)]
    want = [(saw.paged_prompt_attn(c.cache, *c.args), saw.paged_attn_weights(c.cache, *c.args)) for c in cases]
    ws = [(torch.empty(saw.paged_prompt_workspace_bytes(c.cache, c.args[0], 8, c.pt.shape[1] * 16), dtype=torch.uint8, device="cuda"),
           torch.empty(saw.attn_weights_workspace_bytes(c.cache, c.args[0], 8, c.pt.shape[1] * 16), dtype=torch.uint8, device="cuda")) for c in cases]
    got = [(torch.zeros_like(a), torch.zeros_like(b)) for a, b in want]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s, w, g in zip(cases, streams, ws, got):
            with torch.cuda.stream(s):
                saw.paged_prompt_attn(c.cache, *c.args, out=g[0], workspace=w[0])
                saw.paged_attn_weights(c.cache, *c.args, scores=g[1], workspace=w[1])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])
