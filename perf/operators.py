"""Prompt attention and cache eviction: the calls that stand before and between the decode steps.

Four operators, as a serving program makes their calls for one layer:

  prompt   attention of packed prompts over their own 16-bit keys and values, causal, with grouped heads
           (``binding.prompt_attn``); a sequence may have more keys than queries, as with a dense prefix in front
  chunk    attention of a few or many new tokens of every sequence over the INT4 pages, which hold the new tokens
           already (``binding.paged_prompt_attn``): draft tokens to verify, chunks of a prompt
  weights  the attention weight that every cached token gets from such queries, summed over queries and the query heads
           of a kv head and added to what it had (``binding.paged_attn_weights``)
  evict    keeps the heaviest and the newest tokens of every kv head and moves their bytes to other pages
           (``binding.evict_pages``)

Plain forms are torch operations in 32 bits over padded batches.  Pools are filled with the codes and (scale, zero) pairs that
the quantiser gives for normal values with a few outlier channels.  Evicted tokens' bytes are moved and never quantised again,
so pools are returned as the whole numbers they hold.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, op, **kw):
    # lo..hi: new tokens of a sequence (evict: tokens cached); ctx_lo..ctx_hi: tokens in front of them
    c = {"name": name, "op": op, "n_q": 32, "n_kv": 8, "d": 128, "dtype": "bf16"}
    if op == "prompt":
        c.update(causal=True, ctx_lo=0, ctx_hi=0)
    else:
        c.update(h=128, mask=3, signs=False, learned=False)
    c.update(kw)
    return c


def listed():
    return [
        # Four short fp16 prompts of a chat: latency and launches.
        _case("prompt_short", "prompt", B=4, lo=37, hi=251, dtype="f16"),
        # One long document, the largest product here.
        _case("prompt_8192", "prompt", B=1, lo=8192, hi=8192),
        # A packed batch of prompts of different lengths.
        _case("prompt_packed", "prompt", B=19, lo=60, hi=1437),
        # A chunk of a prompt behind a dense prefix read back from the cache; 64-channel heads, eight to a kv head.
        _case("prompt_prefix_d64", "prompt", B=2, lo=1000, hi=1000, ctx_lo=9001, ctx_hi=15001, n_q=64, d=64, dtype="f16"),
        # Five draft tokens of every sequence to verify against the cache.
        _case("chunk_verify", "chunk", B=32, lo=5, hi=5, ctx_lo=512, ctx_hi=4096, h=64),
        # A chunk of 2048 tokens of a long prompt.
        _case("chunk_2048", "chunk", B=1, lo=2048, hi=2048, ctx_lo=16384, ctx_hi=16384),
        # Chunks of several prompts at once, fp16, randomised Hadamard on 64-channel heads.
        _case("chunk_ragged_d64", "chunk", B=7, lo=17, hi=700, ctx_lo=100, ctx_hi=5000, d=64, h=64, dtype="f16", signs=True),
        # A decode step's queries: every step adds its weights to the record.
        _case("weights_decode", "weights", B=64, lo=1, hi=1, ctx_lo=512, ctx_hi=4096),
        # The last tokens of two long prompts, which decide what is kept of them; eight query heads to a kv head.
        _case("weights_window", "weights", B=2, lo=32, hi=32, ctx_lo=12000, ctx_hi=16001, n_q=64),
        # Four chats cut back to 512 tokens.
        _case("evict_small", "evict", B=4, lo=600, hi=1100, budget=512, recent=64),
        # A server's ragged batch, some of it below the budget.
        _case("evict_ragged", "evict", B=48, lo=700, hi=8000, budget=2048, recent=256),
        # A long document cut to an eighth.
        _case("evict_long", "evict", B=1, lo=131072, hi=131072, budget=16384, recent=1000),
    ]


#: the most logits a drawn case may have in its padded form, and the most bytes
MOST_LOGITS, MOST_BYTES = 0.8e9, 0.4e9


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "chunk", "chunk", "weights", "weights", "evict", "evict"])
    d = rng.choice([128, 128, 64])
    n_kv = rng.choice([1, 2, 4, 8, 8])
    c = {"op": op, "n_kv": n_kv, "n_q": n_kv * rng.choice([1, 2, 4, 4, 8]), "d": d, "dtype": rng.choice(["bf16", "f16"]), "B": _log(rng, 1, 64)}
    if op != "prompt":
        c.update(h=rng.choice([h for h in (1, 16, 32, 64, 128) if h <= d]), mask=rng.choice([3, 3, 1]), signs=rng.random() < 0.25,
                 learned=d == 128 and rng.random() < 0.2)
    if op == "evict":
        c["hi"] = _log(rng, 20, min(131072, int(MOST_BYTES / (c["B"] * n_kv * (d + 16)))))
        c["budget"] = max(1, int(c["hi"] * rng.uniform(0.05, 0.8)))
        c["recent"] = int(c["budget"] * rng.choice([0.0, 0.1, 0.5, 1.0]))
        c["lo"] = max(1, int(c["hi"] * rng.uniform(0.1, 1.0)))
        return c
    each = MOST_LOGITS / (c["B"] * c["n_q"])
    if op == "prompt":
        c["causal"] = rng.random() < 0.8
        c["hi"] = _log(rng, 1, min(6000, int(math.sqrt(each))))
        ctx = rng.choice([0, 0, 1])
    else:
        c["hi"] = _log(rng, 1, min(3000 if op == "chunk" else 256, int(math.sqrt(each)))) if rng.random() < 0.6 else rng.randrange(1, 9)
        ctx = 1
    c["lo"] = max(1, int(c["hi"] * rng.uniform(0.05, 1.0)))
    most = min(40000, int(each / c["hi"]) - c["hi"], int(MOST_BYTES / (c["B"] * n_kv * 4 * d)))
    c["ctx_hi"] = _log(rng, 1, max(1, most)) if ctx else 0
    c["ctx_lo"] = int(c["ctx_hi"] * rng.uniform(0.05, 1.0))
    return c


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi, seed):
    """Quantiles of a uniform distribution over [lo, hi], dealt out in a seeded order."""
    v = [lo + int((hi - lo) * (i + 0.5) / n) for i in range(n)]
    return [v[i] for i in torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()]


def _offsets(n):
    return torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32).cuda()


def _rotation(c, seed):
    """(signs, learned matrix, whole rotation in 64 bits: diag(signs), block Hadamard, learned)"""
    d, h = c["d"], c["h"]
    g = torch.Generator().manual_seed(seed + 29)
    signs = [1.0 if x else -1.0 for x in torch.randint(0, 2, (d,), generator=g).tolist()] if c["signs"] else None
    learned = None
    if c["learned"]:
        Q, R = torch.linalg.qr(torch.randn((d, d), generator=g, dtype=torch.float64))
        learned = (Q * torch.sign(torch.diagonal(R))).float()
    H = torch.ones((1, 1), dtype=torch.float64)
    while H.shape[0] < h:
        H = torch.cat([torch.cat([H, H], 1), torch.cat([H, -H], 1)], 0)
    M = torch.block_diag(*([H / math.sqrt(h)] * (d // h)))
    if h > 1 and signs is not None:
        M = torch.tensor(signs, dtype=torch.float64)[:, None] * M
    if learned is not None:
        M = M @ learned.double()
    return signs, learned, M.cuda()


def _channel_scales(c, seed):
    """One per (kv head, channel): four channels of a head are 20 times as large, as keys have them."""
    g = torch.Generator().manual_seed(seed + 37)
    s = torch.ones((2, c["n_kv"], c["d"]))
    for t in range(2):
        for k in range(c["n_kv"]):
            s[t, k, torch.randperm(c["d"], generator=g)[:4]] = 20.0
    return s.cuda()


def _pools(c, pages, seed, M):
    """Code and (scale, zero) pools of one layer, every slot quantised from its own values."""
    n_kv, d = c["n_kv"], c["d"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    scales = _channel_scales(c, seed)
    got = {}
    for t, name in enumerate("kv"):
        codes = torch.empty((pages, n_kv, PAGE, d // 2), dtype=torch.uint8, device="cuda")
        meta = torch.empty((pages, n_kv, PAGE, 2), dtype=torch.float32, device="cuda")
        step = max(1, (1 << 26) // (n_kv * PAGE * d))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            y = torch.randn((n, n_kv, PAGE, d), generator=g, device="cuda") * scales[t][:, None, :]
            if c["mask"] >> t & 1:
                y = (y.reshape(-1, d) @ M.float()).reshape(y.shape)
            mn = y.amin(-1)
            s = (y.amax(-1) - mn) / 15
            z = torch.round(-mn / s)
            q = (torch.round(y / s[..., None]) + z[..., None]).clamp_(0, 15).to(torch.uint8)
            codes[p:p + n] = q[..., 0::2] | q[..., 1::2] << 4
            meta[p:p + n, ..., 0] = s
            meta[p:p + n, ..., 1] = z
        got[name + "_codes"], got[name + "_meta"] = codes, meta
    return got


def _tables(need, seed, width=0):
    """Page tables (one for each list of needed pages) out of one shuffled pool with a few pages to spare."""
    pool = sum(map(sum, need)) + 8
    perm = torch.randperm(pool, generator=torch.Generator().manual_seed(seed + 41)).to(torch.int32)
    at, tables = 0, []
    for pages in need:
        pt = torch.zeros((len(pages), max(max(pages), width)), dtype=torch.int32)
        for b, n in enumerate(pages):
            pt[b, :n] = perm[at:at + n]
            at += n
        tables.append(pt.cuda())
    return tables, pool


def _pages(n):
    return (n + PAGE - 1) // PAGE


def prepare(case, seed):
    c, d, B = case, case["d"], case["B"]
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    s = {"c": c}
    new = _spread(B, c["lo"], c["hi"], seed + 17)
    if c["op"] == "evict":
        budget = c["budget"]
        s["lens"], s["max_len"] = torch.tensor(new, dtype=torch.int32).cuda(), max(new)
        (s["pt"], s["dst"]), pool = _tables([[_pages(n) for n in new], [_pages(budget)] * B], seed)
        # accumulated weights: spread over orders of magnitude, some tokens never looked at
        x = torch.exp(2 * torch.randn((B, c["n_kv"], max(new)), generator=g, device="cuda") - 4)
        s["scores"] = torch.where(torch.rand(x.shape, generator=g, device="cuda") < 0.03, 0.0, x)
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["kept"] = torch.zeros((B, c["n_kv"], budget), dtype=torch.int32, device="cuda")
        s["scores_out"] = torch.zeros((B, c["n_kv"], budget), dtype=torch.float32, device="cuda")
    else:
        ctx = _spread(B, c["ctx_lo"], c["ctx_hi"], seed + 19)
        lens = [a + b for a, b in zip(ctx, new)]
        s["new"], s["max_new"], s["max_len"] = new, max(new), c["hi"] + c["ctx_hi"]  # (a bound, whichever sequence meets which context)
        s["cu_q"], s["lens"] = _offsets(new), torch.tensor(lens, dtype=torch.int32).cuda()
        s["q"] = torch.randn((sum(new), c["n_q"], d), generator=g, device="cuda").to(DTYPES[c["dtype"]])
        if c["op"] == "prompt":
            sc = _channel_scales(c, seed)
            s["cu_k"] = _offsets(lens)
            s["k"], s["v"] = ((torch.randn((sum(lens), c["n_kv"], d), generator=g, device="cuda") * sc[t].sqrt()).to(DTYPES[c["dtype"]]) for t in range(2))
        else:
            (s["pt"],), pool = _tables([[_pages(n) for n in lens]], seed, _pages(s["max_len"]))
        if c["op"] == "weights":
            s["prev"] = torch.rand((B, c["n_kv"], s["max_len"]), generator=g, device="cuda")
            s["scores"] = torch.zeros_like(s["prev"])
    if c["op"] != "prompt":
        s["signs"], s["learned"], s["M"] = _rotation(c, seed)
        s.update(_pools(c, pool, seed + 3, s["M"]))
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The handle, the scratch and the output that a serving program keeps between calls."""
    from paper_2604_19157_amd import binding as saw

    c, s["saw"] = s["c"], saw
    if c["op"] != "prompt":
        k = saw.Cache(1, c["n_kv"], c["d"], c["h"], c["mask"], signs=s["signs"], dense=s["learned"])
        k.num_pages = s["k_codes"].shape[0]
        k.k_codes, k.k_meta, k.v_codes, k.v_meta = (s[n] for n in ("k_codes", "k_meta", "v_codes", "v_meta"))
        s["cache"] = k
    if c["op"] == "prompt":
        need = saw.prompt_workspace_bytes(s["q"], s["k"], c["B"], s["max_len"])
    elif c["op"] == "chunk":
        need = saw.paged_prompt_workspace_bytes(s["cache"], s["q"], c["B"], s["max_len"])
    elif c["op"] == "weights":
        need = saw.attn_weights_workspace_bytes(s["cache"], s["q"], c["B"], s["max_len"])
    else:
        return
    s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    if c["op"] != "weights":
        s["out"] = torch.empty_like(s["q"])


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    op = s["c"]["op"]
    if own:
        saw = s["saw"]
        if op == "prompt":
            return saw.prompt_attn(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], max_k_len=s["max_len"], causal=s["c"]["causal"], out=s["out"],
                                   workspace=s["ws"])
        if op == "chunk":
            return saw.paged_prompt_attn(s["cache"], s["q"], s["cu_q"], s["pt"], s["lens"], max_seq_len=s["max_len"], out=s["out"],
                                         workspace=s["ws"])
        if op == "weights":
            return saw.paged_attn_weights(s["cache"], s["q"], s["cu_q"], s["pt"], s["lens"], prev=s["prev"], scores=s["scores"],
                                          max_seq_len=s["max_len"], workspace=s["ws"])
        saw.evict_pages(s["cache"], s["scores"], s["pt"], s["lens"], s["dst"], s["c"]["budget"], recent=s["c"]["recent"],
                        max_seq_len=s["max_len"], new_lens=s["new_lens"], kept=s["kept"], scores_out=s["scores_out"])
    elif op == "evict":
        _evict(s)
    else:
        return {"prompt": _prompt, "chunk": _chunk, "weights": _weights}[op](s)
    return [s[n] for n in ("new_lens", "kept", "scores_out", "k_codes", "v_codes")] + [s[n][..., i] for n in ("k_meta", "v_meta") for i in (0, 1)]


def _padded_queries(s):
    """Queries as [B][n_kv][group x max_new][d] in 32 bits, their index among the packed ones, which of them there are, and how many
    tokens each may see."""
    c, d = s["c"], s["c"]["d"]
    group = c["n_q"] // c["n_kv"]
    start, n = s["cu_q"][:-1].long(), (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    i = torch.arange(s["max_new"], device="cuda")
    there = i < n[:, None]
    at = torch.where(there, start[:, None] + i, 0)
    q = s["q"][at].float().reshape(c["B"], s["max_new"], c["n_kv"], group, d).permute(0, 2, 3, 1, 4).reshape(c["B"], c["n_kv"], -1, d)
    sees = s["lens"].long()[:, None] - n[:, None] + i + 1
    return q, at, there, sees


def _softmax_terms(q, k, visible, group):
    """exp(logit - row maximum), zero where not visible, and their sums."""
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(1.0 / math.sqrt(q.shape[-1]))
    x = x.reshape(x.shape[0], x.shape[1], group, visible.shape[1], x.shape[-1])
    x.masked_fill_(~visible[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(torch.isinf(m), 0.0, m)).exp_()
    return p, p.sum(-1, keepdim=True)


def _attend(s, q, k, v, visible):
    c = s["c"]
    p, total = _softmax_terms(q, k, visible, c["n_q"] // c["n_kv"])
    o = torch.matmul(p.reshape(*q.shape[:3], -1), v)
    return o / torch.where(total == 0, 1.0, total).reshape(*q.shape[:3], 1)


def _packed(s, o, at, there):
    """[B][n_kv][group x max_new][d] back to the packed rows, rounded once."""
    c = s["c"]
    o = o.reshape(c["B"], c["n_kv"], -1, s["max_new"], c["d"]).permute(0, 3, 1, 2, 4).reshape(c["B"] * s["max_new"], c["n_q"], c["d"])
    # (rows that only pad the batch go to one row behind the last)
    rows = s["q"].shape[0]
    out = torch.zeros((rows + 1, c["n_q"], c["d"]), dtype=s["q"].dtype, device="cuda")
    out[torch.where(there, at, rows).reshape(-1)] = o.to(out.dtype)
    return out[:rows]


def _prompt(s):
    c = s["c"]
    q, at, there, sees = _padded_queries(s)
    j = torch.arange(s["max_len"], device="cuda")
    k_at = torch.where(j < s["lens"][:, None], s["cu_k"][:-1].long()[:, None] + j, 0)
    k, v = (s[n][k_at].float().permute(0, 2, 1, 3).contiguous() for n in "kv")
    limit = sees if c["causal"] else s["lens"].long()[:, None].expand_as(sees)
    visible = (j < torch.minimum(limit, s["lens"].long()[:, None])[..., None]) & there[..., None]
    return _packed(s, _attend(s, q, k, v, visible), at, there)


def _dequantised(s, name):
    """The sequences' cached vectors as they are stored, [B][n_kv][max_len][d]."""
    j = torch.arange(_pages(s["max_len"]), device="cuda")
    page = torch.where(j < (s["lens"][:, None] + PAGE - 1) // PAGE, s["pt"], 0).long()
    b, m = s[name + "_codes"][page], s[name + "_meta"][page]
    codes = torch.stack([b & 15, b >> 4], -1).flatten(-2).float()
    x = m[..., :1] * (codes - m[..., 1:])
    return x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], x.shape[2], -1, x.shape[-1])[:, :, :s["max_len"]].contiguous()


def _rotated(s, q):
    return torch.matmul(q, s["M"].float()) if s["c"]["mask"] & 1 else q


def _chunk(s):
    q, at, there, sees = _padded_queries(s)
    visible = (torch.arange(s["max_len"], device="cuda") < sees[..., None]) & there[..., None]
    o = _attend(s, _rotated(s, q), _dequantised(s, "k"), _dequantised(s, "v"), visible)
    if s["c"]["mask"] & 2:
        o = torch.matmul(o, s["M"].float().t().contiguous())
    return _packed(s, o, at, there)


def _weights(s):
    c = s["c"]
    q, _, there, sees = _padded_queries(s)
    j = torch.arange(s["max_len"], device="cuda")
    visible = (j < sees[..., None]) & there[..., None]
    p, total = _softmax_terms(_rotated(s, q), _dequantised(s, "k"), visible, c["n_q"] // c["n_kv"])
    w = (p / torch.where(total == 0, 1.0, total)).sum((2, 3))
    s["scores"].copy_(torch.where((j < s["lens"][:, None])[:, None], s["prev"] + w, s["scores"]))
    return s["scores"]


def _evict(s):
    c, n = s["c"], s["lens"].long()[:, None, None]
    budget, device = c["budget"], s["scores"].device
    j = torch.arange(s["max_len"], device=device)
    key = torch.where(j < n - c["recent"], s["scores"], torch.where(j < n, math.inf, -math.inf))
    order = key.sort(dim=-1, descending=True, stable=True)[1][..., :budget]
    order = torch.nn.functional.pad(order, (0, budget - order.shape[-1]), value=s["max_len"])
    i = torch.arange(budget, device=device)
    there = (i < n).expand(order.shape)
    at = torch.where(there, order, s["max_len"]).sort(-1)[0]
    s["kept"].copy_(torch.where(there, at, -1))
    at = torch.where(there, at, 0)
    s["scores_out"].copy_(torch.where(there, s["scores"].gather(-1, at), 0.0))
    s["new_lens"].copy_(s["lens"].clamp(max=budget))
    seq = torch.arange(c["B"], device=device)[:, None, None]
    head = torch.arange(c["n_kv"], device=device)[None, :, None]
    src, src_slot = s["pt"][seq, at // PAGE].long(), at % PAGE
    dst, dst_slot = s["dst"][seq, (i // PAGE).expand(at.shape)].long(), (i % PAGE).expand(at.shape)
    for pool in (s["k_codes"], s["v_codes"], s["k_meta"], s["v_meta"]):
        old = pool[dst, head, dst_slot]
        pool[dst, head, dst_slot] = torch.where(there[..., None], pool[src, head, src_slot], old)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it gives in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    c, d = case, case["d"]
    new = _spread(c["B"], c["lo"], c["hi"], 0)
    if c["op"] == "evict":
        kept = sum(min(n, c["budget"]) for n in new)
        return {"bytes": c["n_kv"] * (4 * sum(new) + kept * (2 * (d + 16) + 4) + 4 * 2 * c["budget"] * c["B"]), "flops": 0}
    # (queries and contexts are dealt out apart: the pairs of a mean sequence)
    ctx = sum(_spread(c["B"], c["ctx_lo"], c["ctx_hi"], 0)) / c["B"]
    causal = c.get("causal", True)
    pairs = sum(n * ctx + (n * (n + 1) / 2 if causal else n * n) for n in new)
    keys = sum(new) + ctx * c["B"]
    if c["op"] == "prompt":
        return {"bytes": 2 * d * (2 * sum(new) * c["n_q"] + 2 * keys * c["n_kv"]), "flops": 4 * d * c["n_q"] * pairs}
    if c["op"] == "chunk":
        return {"bytes": 2 * d * 2 * sum(new) * c["n_q"] + keys * c["n_kv"] * (d + 16), "flops": 4 * d * c["n_q"] * pairs}
    return {"bytes": 2 * d * sum(new) * c["n_q"] + keys * c["n_kv"] * (d // 2 + 8 + 8), "flops": 2 * d * c["n_q"] * pairs}


def exact(case, seed):
    """Sequence by sequence and head by head in 64 bits, in the space the values had before they were rotated."""
    c, s = case, prepare(case, seed)
    d, group = c["d"], c["n_q"] // c["n_kv"]
    lens = s["lens"].tolist()
    if c["op"] == "evict":
        scores, out = s["scores"].cpu().double().numpy(), np.zeros((c["B"], c["n_kv"], c["budget"]))
        for b in range(c["B"]):
            old = max(0, lens[b] - c["recent"])
            for h in range(c["n_kv"]):
                best = np.lexsort((np.arange(old), -scores[b, h, :old]))[:max(0, min(lens[b], c["budget"]) - (lens[b] - old))]
                keep = np.concatenate([np.sort(best), np.arange(old, lens[b])])
                out[b, h, :len(keep)] = scores[b, h, keep]
        return [None, None, torch.from_numpy(out), None, None, None, None, None, None]

    def stored(name, b, h, bit):
        page = s["pt"][b, torch.arange(lens[b], device="cuda") // PAGE].long()
        slot = torch.arange(lens[b], device="cuda") % PAGE
        x = s[name + "_codes"][page, h, slot]
        codes = torch.empty((lens[b], d), dtype=torch.float64, device="cuda")
        codes[:, 0::2], codes[:, 1::2] = (x % 16).double(), (x // 16).double()
        m = s[name + "_meta"][page, h, slot].double()
        x = m[:, :1] * (codes - m[:, 1:])
        return x @ s["M"].t() if c["mask"] & bit else x

    at = [0] + np.cumsum(s["new"]).tolist()
    rows = torch.zeros((at[-1], c["n_q"], d), dtype=torch.float64, device="cuda")
    totals = s["scores"].double().clone() if c["op"] == "weights" else None
    first = 0
    for b in range(c["B"]):
        n, L = s["new"][b], lens[b]
        see = torch.arange(n, device="cuda") + L - n if c.get("causal", True) else torch.full((n,), L - 1, device="cuda")
        hidden = torch.arange(L, device="cuda")[None, :] > see[:, None]
        for h in range(c["n_kv"]):
            if c["op"] == "prompt":
                k, v = s["k"][first:first + L, h].double(), s["v"][first:first + L, h].double()
            else:
                k = stored("k", b, h, 1)
                v = stored("v", b, h, 2) if c["op"] == "chunk" else None
            for j in range(h * group, (h + 1) * group):
                x = s["q"][at[b]:at[b + 1], j].double() @ k.t() / math.sqrt(d)
                w = torch.softmax(x.masked_fill_(hidden, -math.inf), -1)
                if v is not None:
                    rows[at[b]:at[b + 1], j] = w @ v
                else:
                    totals[b, h, :L] += w.sum(0)
            if totals is not None:
                totals[b, h, :L] += s["prev"][b, h, :L].double()
        first += L
    return rows if totals is None else totals
