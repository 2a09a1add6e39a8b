"""saw_evict_pages: kept tokens against a plain selection, bytes as they were, and a run of a prompt, its weights, eviction and decode."""
import numpy as np
import pytest
import torch

import packed_cases as pc
from oracle import saw_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def saw():
    from paper_2604_19157_amd import binding
    binding.lib()
    return binding


class Case:
    def __init__(self, saw, lens, budget, recent, Hkv=2, d=128, seed=0, scores=None, width=None):
        rng = np.random.default_rng(seed)
        self.lens, self.budget, self.recent, self.Hkv = lens, budget, recent, Hkv
        B, src, dst = len(lens), [(x + 15) // 16 for x in lens], (budget + 15) // 16
        num = sum(src) + B * dst + 2
        perm = rng.permutation(num).astype(np.int32)
        self.pt = np.full((B, max(max(src), 1)), -1, np.int32)
        at = 0
        for b, p in enumerate(src):
            self.pt[b, :p] = perm[at:at + p]
            at += p
        self.dst = perm[at:at + B * dst].reshape(B, dst).copy()
        self.cache = saw.Cache(num, Hkv, d, 1)
        for name in ("k_codes", "v_codes"):
            t = getattr(self.cache, name)
            t.copy_(torch.from_numpy(rng.integers(0, 256, tuple(t.shape), np.uint8)))
        for name in ("k_meta", "v_meta"):
            t = getattr(self.cache, name)
            t.copy_(torch.from_numpy(rng.normal(size=tuple(t.shape)).astype(np.float32)))
        self.before = self.pools()
        self.scores = rng.random((B, Hkv, width or max(max(lens), 1))).astype(np.float32) if scores is None else scores
        self.args = (torch.from_numpy(self.scores).cuda(), torch.from_numpy(self.pt).cuda(), torch.from_numpy(np.asarray(lens, np.int32)).cuda(),
                     torch.from_numpy(self.dst).cuda())

    def pools(self):
        return {n: getattr(self.cache, n).cpu().numpy().copy() for n in ("k_codes", "v_codes", "k_meta", "v_meta")}

    def run(self, saw, **kw):
        got = saw.evict_pages(self.cache, *self.args, self.budget, recent=self.recent, max_seq_len=max(max(self.lens), 1), **kw)
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in got]

    def check(self, got):
        new_lens, kept, scores = got
        want = {n: p.copy() for n, p in self.before.items()}
        for b, L in enumerate(self.lens):
            n = min(L, self.budget)
            assert new_lens[b] == n
            for h in range(self.Hkv):
                at = O.evict_kept(self.scores[b, h], L, self.budget, self.recent)
                assert np.array_equal(kept[b, h, :n], at) and (kept[b, h, n:] == -1).all(), (b, h)
                assert np.array_equal(scores[b, h, :n], self.scores[b, h, at], equal_nan=True) and not scores[b, h, n:self.budget].any()
                to = np.arange(n)
                for name, pool in want.items():
                    pool[self.dst[b, to // 16], h, to % 16] = self.before[name][self.pt[b, at // 16], h, at % 16]
        for name, pool in self.pools().items():
            assert np.array_equal(pool.view(np.uint8), want[name].view(np.uint8)), name


@pytest.mark.parametrize("lens,budget,recent", [([1], 1, 0), ([40, 0, 17], 16, 4), ([100, 33, 34], 33, 33), ([2000, 1024, 1025, 5], 1000, 100),
                                                 ([64], 100, 10), ([5000, 4999], 1, 1), ([3000, 700], 65, 0), ([20000], 7777, 1234)], ids=str)
@pytest.mark.parametrize("d", [128, 64])
def test_kept_tokens_and_their_bytes(saw, lens, budget, recent, d):
    c = Case(saw, lens, budget, recent, d=d, Hkv=3, seed=budget)
    c.check(c.run(saw))


@pytest.mark.parametrize("kind", ["constant", "few", "zeros of both signs", "nan", "infinite", "negative", "tiny", "all nan"])
def test_scores_of_every_kind(saw, kind):
    rng = np.random.default_rng(5)
    s = rng.normal(size=(2, 2, 700)).astype(np.float32)
    if kind == "constant":
        s[:] = 0.25
    elif kind == "few":
        s = rng.integers(0, 4, s.shape).astype(np.float32)
    elif kind == "zeros of both signs":
        s = np.where(rng.random(s.shape) < 0.5, np.float32(0), np.float32(-0.0))
        s[:, :, ::7] = -1
    elif kind == "nan":
        s[rng.random(s.shape) < 0.6] = np.nan
    elif kind == "infinite":
        s[rng.random(s.shape) < 0.3] = np.inf
        s[rng.random(s.shape) < 0.3] = -np.inf
    elif kind == "negative":
        s = -np.abs(s)
    elif kind == "tiny":
        s = (s * np.float32(1e-40)).astype(np.float32)
    else:
        s[:] = np.nan
    c = Case(saw, [700, 651], 300, 20, scores=s.astype(np.float32))
    c.check(c.run(saw))


@pytest.mark.parametrize("lens,budget,recent", [([40000], 5000, 700), ([20000, 0, 8192, 8193, 30], 8192, 0), ([30000, 17000], 9000, 8999), ([16385], 1, 0),
                                                 ([50000], 30000, 20000)], ids=str)
@pytest.mark.parametrize("kind", ["random", "few", "constant", "nan"])
def test_long_rows(saw, lens, budget, recent, kind):
    """Few long rows are selected from by several blocks each."""
    rng = np.random.default_rng(budget)
    s = rng.random((len(lens), 2, max(lens) + 3)).astype(np.float32)
    if kind == "few":
        s = rng.integers(0, 5, s.shape).astype(np.float32)
    elif kind == "constant":
        s[:] = -2.5
    elif kind == "nan":
        s[rng.random(s.shape) < 0.7] = np.nan
    c = Case(saw, lens, budget, recent, scores=s)
    assert saw.evict_workspace_bytes(c.cache, len(lens), max(lens)) > 0
    c.check(c.run(saw))


@pytest.mark.parametrize("lens,budget", [([3000, 700, 90], 600), ([3000] * 300, 100), ([40000, 17000], 5000)], ids=["few", "many", "long"])
def test_lengths_replaced_in_place(saw, lens, budget):
    """new_lens is seq_lens: every head selects from the old length, whenever its block starts."""
    c = Case(saw, lens, budget, 10, Hkv=4)
    c.check(c.run(saw, new_lens=c.args[2]))
    assert c.args[2].tolist() == [min(x, budget) for x in lens]


@pytest.mark.parametrize("lens,Hkv", [([12000, 16384, 8193, 8192], 2), ([17000] + [30] * 64, 2)], ids=["middle", "many rows"])
@pytest.mark.parametrize("kind", ["random", "few", "constant", "nan", "all nan", "low digits"])
def test_many_scores_of_like_size_in_one_block(saw, lens, Hkv, kind):
    """Rows that a single block selects from, of which more scores share the first digit than its list holds: they are all read again."""
    rng = np.random.default_rng(9)
    s = rng.random((len(lens), Hkv, max(lens))).astype(np.float32)
    if kind == "few":
        s = rng.integers(1, 3, s.shape).astype(np.float32) / 8 + 1
    elif kind == "constant":
        s[:] = 0.25
    elif kind == "nan":
        s[rng.random(s.shape) < 0.9] = np.nan
    elif kind == "all nan":
        s[:] = np.nan
    elif kind == "low digits":                        # one in the first 11 bits of the key, many in the next and the last
        s = (1 + s / 16).astype(np.float32)
    for budget, recent in ((5000, 700), (1, 0), (8000, 8000)):
        c = Case(saw, lens, budget, recent, Hkv=Hkv, scores=s)
        assert saw.evict_workspace_bytes(c.cache, len(lens), max(lens)) == 0
        c.check(c.run(saw))


def test_rows_further_apart_than_needed(saw):
    c = Case(saw, [300, 200], 100, 10, width=517)
    out = torch.full((2, 2, 333), 8.0, device="cuda")
    got = c.run(saw, scores_out=out)
    c.check([got[0], got[1], got[2][..., :100]])
    assert (got[2][..., 100:] == 8).all()


def test_pages_out_of_range_are_not_copied(saw):
    c = Case(saw, [64], 48, 0)
    c.pt[0, 1], c.dst[0, 2] = 1 << 29, -3
    c.args = (c.args[0], torch.from_numpy(c.pt).cuda(), c.args[2], torch.from_numpy(c.dst).cuda())
    new_lens, kept, _ = c.run(saw)
    at = O.evict_kept(c.scores[0, 0], 64, 48, 0)
    assert new_lens[0] == 48 and np.array_equal(kept[0, 0], at)
    want = {n: p.copy() for n, p in c.before.items()}
    for h in range(2):
        at = O.evict_kept(c.scores[0, h], 64, 48, 0)
        for t, j in enumerate(at):
            if j // 16 != 1 and t // 16 != 2:
                for n in want:
                    want[n][c.dst[0, t // 16], h, t % 16] = c.before[n][c.pt[0, j // 16], h, j % 16]
    for n, pool in c.pools().items():
        assert np.array_equal(pool.view(np.uint8), want[n].view(np.uint8))


def test_two_sequences_may_share_the_pages_they_are_read_from(saw):
    """A common prefix: both sequences list the same source pages, each keeps its own choice of them."""
    c = Case(saw, [160, 160], 50, 8)
    c.pt[1] = c.pt[0]
    c.args = (c.args[0], torch.from_numpy(c.pt).cuda(), *c.args[2:])
    c.check(c.run(saw))


def test_captured_and_replayed(saw):
    c = Case(saw, [500, 90, 30], 64, 5)
    new_lens, kept, out = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((3, 2, 64), dtype=torch.int32, device="cuda"), torch.zeros((3, 2, 64), device="cuda")

    def run():
        saw.evict_pages(c.cache, *c.args, 64, recent=5, max_seq_len=500, new_lens=new_lens, kept=kept, scores_out=out)

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(3):
        c.scores = np.random.default_rng(50 + i).random(c.scores.shape).astype(np.float32)
        c.args[0].copy_(torch.from_numpy(c.scores))
        kept.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.check([new_lens.cpu().numpy(), kept.cpu().numpy(), out.cpu().numpy()])


def test_long_rows_captured_and_replayed_with_lengths_in_place(saw):
    """The launches of few long rows in a graph, lengths replaced by each replay and set back before the next."""
    lens, budget = [40000, 17000, 300], 2000
    c = Case(saw, lens, budget, 100)
    ws = torch.empty(saw.evict_workspace_bytes(c.cache, 3, 40000), dtype=torch.uint8, device="cuda")
    kept, out = torch.zeros((3, 2, budget), dtype=torch.int32, device="cuda"), torch.zeros((3, 2, budget), device="cuda")

    def run():
        saw.evict_pages(c.cache, *c.args, budget, recent=100, max_seq_len=40000, new_lens=c.args[2], kept=kept, scores_out=out, workspace=ws)

    old = c.args[2].clone()
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(3):
        c.scores = np.random.default_rng(60 + i).random(c.scores.shape).astype(np.float32)
        c.args[0].copy_(torch.from_numpy(c.scores))
        c.args[2].copy_(old)
        ws.fill_(0xff)
        kept.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.check([c.args[2].cpu().numpy(), kept.cpu().numpy(), out.cpu().numpy()])


@pytest.mark.parametrize("d,dtype", [(128, torch.bfloat16), (64, torch.float16)])
def test_prompt_weights_eviction_and_decode_together(saw, d, dtype):
    """Prompts are attended to and stored, a chunk of new tokens follows, its weights decide what is kept, decode goes on over the kept
    tokens: the last step against attention in 64 bits over the tokens that the record of kept positions names."""
    Hkv, G, h = 2, 4, 64
    n, extra, budget, recent = [150, 61, 20], [9, 16, 1], 48, 12
    B, width = 3, 12
    pt = torch.randperm(B * width, generator=torch.Generator().manual_seed(1)).to(torch.int32).reshape(B, width).cuda()
    dst = (torch.randperm(B * 4, generator=torch.Generator().manual_seed(2)).to(torch.int32).reshape(B, 4) + B * width).cuda()
    cache = saw.Cache(B * width + B * 4, Hkv, d, h)
    cu = torch.from_numpy(pc.offsets(n)).cuda()
    q, k, v = (pc.rand((sum(n), H, d), s, dtype).cuda() for H, s in ((Hkv * G, 1), (Hkv, 2), (Hkv, 3)))
    out = saw.prompt_attn(q, k, v, cu)
    want, tol = pc.prompt_reference(q.cpu(), k.cpu(), v.cpu(), pc.offsets(n), pc.offsets(n), True)
    pc.check(out, want, tol)
    slots = torch.tensor([(b, i) for b in range(B) for i in range(n[b])], dtype=torch.int32).cuda()
    saw.rotate_quant_store(cache, k, v, pt, slots)
    # a chunk: its tokens are stored first
    q2, k2, v2 = (pc.rand((sum(extra), H, d), s, dtype).cuda() for H, s in ((Hkv * G, 4), (Hkv, 5), (Hkv, 6)))
    slots = torch.tensor([(b, n[b] + i) for b in range(B) for i in range(extra[b])], dtype=torch.int32).cuda()
    saw.rotate_quant_store(cache, k2, v2, pt, slots)
    lens = [a + b for a, b in zip(n, extra)]
    sl, cu2 = torch.tensor(lens, dtype=torch.int32).cuda(), torch.from_numpy(pc.offsets(extra)).cuda()
    saw.paged_prompt_attn(cache, q2, cu2, pt, sl)
    scores = saw.paged_attn_weights(cache, q2, cu2, pt, sl)
    before = cache.k_codes.clone()
    new_lens, kept, _ = saw.evict_pages(cache, scores, pt, sl, dst, budget, recent)
    assert new_lens.tolist() == [min(x, budget) for x in lens]
    assert torch.equal(before[pt.long().flatten()], cache.k_codes[pt.long().flatten()])
    s = scores.cpu().numpy()
    q3 = pc.rand((B, Hkv * G, d), 7, dtype).cuda()
    got = saw.paged_decode_attn(cache, q3, dst, new_lens, max_seq_len=budget).double().cpu().numpy()
    for b in range(B):
        kf, vf = (x.double().cpu().numpy() for x in saw.dequant_pages(cache, pt, b, 0, lens[b], unrotate=True))
        for g in range(Hkv):
            at = O.evict_kept(s[b, g], lens[b], budget, recent)
            assert kept[b, g, :len(at)].tolist() == at.tolist()
            qg = q3[b, g * G:(g + 1) * G].double().cpu().numpy()
            o = O._softmax_rows(qg @ kf[at, g].T / np.sqrt(d)) @ vf[at, g]
            assert np.abs(got[b, g * G:(g + 1) * G] - o).max() < 1e-4 * np.abs(vf[at, g]).max()
