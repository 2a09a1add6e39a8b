"""Shared by the GPU tests of packed queries: inputs, references in 64 bits and error bounds worked out per output.

Bounds.  With u the half step of the output's type (bf16 2^-8, fp16 2^-11), w the exact weights of a row, A = sum_j w_j |v_j| per channel and
e the most that a logit can be off, an output is off by at most
    u |o| + A (u_p + exp(2 e) - 1 + 2^-20 + n 2^-22)          (1 + a few u for products of these)
  u_p      rounding of a weight before the product with V (its type's half step; over the INT4 pages weight and value enter as fp16, 2^-10)
  2 e      in the exponent: a weight's logit and its sum's, off in opposite directions
  2^-20    the exponential and the division;  n 2^-22   sums of n terms in fp32, of weights and of the product (each at most n 2^-23)
and e = scale (sum_c |q_c k_c|) (d 2^-23 + u_q) + 2^-22 |logit|, u_q the rounding of query and key
before their product (over the INT4 pages fp16 each, 2^-10; two fp16 limbs of the query: 2^-21; 16-bit keys: 0).
"""
import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def rand(shape, seed, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def weights64(q, k, visible, scale):
    """(weights [n][L], largest logit error per unit: scale * sum |q||k| and |logit| maxima over visible keys [n])"""
    x = q @ k.T * scale
    mag = np.abs(q) @ np.abs(k).T * scale
    x = np.where(visible, x, -np.inf)
    m = x.max(1, keepdims=True, initial=-np.inf)
    p = np.exp(x - np.where(np.isfinite(m), m, 0))
    t = p.sum(1, keepdims=True)
    w = p / np.where(t == 0, 1, t)
    top = np.where(visible, mag, 0).max(1, initial=0)
    big = np.where(visible, np.abs(np.where(visible, x, 0)), 0).max(1, initial=0)
    return w, top, big


def visible(n, L, causal=True):
    if not causal:
        return np.ones((n, L), bool)
    return np.arange(L)[None, :] <= np.arange(n)[:, None] + L - n


def bound(o, A, top, big, n, d, u, u_p, u_q=0.0, more=0.0):
    """more: a further part of e"""
    e = top * (d * 2.0 ** -23 + u_q) + big * 2.0 ** -22 + more
    rel = u_p + np.expm1(2 * e) + 2.0 ** -20 + n * 2.0 ** -22
    return (u * np.abs(o) + A * rel[:, None]) * (1 + 4 * u) + 1e-30


def prompt_reference(q, k, v, cu_q, cu_k, causal, scale=None):
    """(out, bound) in 64 bits for tensors of one 16-bit type."""
    u = U[q.dtype]
    qd, kd, vd = (x.double().numpy() for x in (q, k, v))
    Hq, d = q.shape[1:]
    G = Hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, tol = np.zeros(qd.shape), np.zeros(qd.shape)
    for b in range(len(cu_q) - 1):
        qs, ks = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        n, L = qs.stop - qs.start, ks.stop - ks.start
        if n == 0 or L == 0:
            continue
        for j in range(Hq):
            w, top, big = weights64(qd[qs, j], kd[ks, j // G], visible(n, L, causal), scale)
            out[qs, j] = w @ vd[ks, j // G]
            tol[qs, j] = bound(out[qs, j], w @ np.abs(vd[ks, j // G]), top, big, L, d, u, u)
    return out, tol


def check(got, want, tol, what=""):
    err = np.abs(got.double().cpu().numpy() - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}, {err[bad].max():.3g} against {tol[bad][err[bad].argmax()]:.3g}"


def check_odd(got, want, tol, odd, cu_q, cu_k, causal, G, what=""):
    """A channel is NaN where its row sees a NaN or infinities of both signs, infinite where it sees one, and what the finite values give elsewhere.
    odd [T_k][Hkv][d]: the values in float64."""
    got = got.double().cpu().numpy()
    for b in range(len(cu_q) - 1):
        n, L = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        x = odd[cu_k[b]:cu_k[b + 1]]
        for i in range(n):
            seen = x[:max(L - n + i + 1, 0) if causal else L]
            nan, pos, neg = (f(seen).any(0).repeat(G, 0) for f in (np.isnan, np.isposinf, np.isneginf))
            o = got[cu_q[b] + i]
            assert np.isnan(o[nan | (pos & neg)]).all(), (what, b, i)
            assert np.isposinf(o[pos & ~neg & ~nan]).all() and np.isneginf(o[neg & ~pos & ~nan]).all(), (what, b, i)
            fine = ~(nan | pos | neg)
            assert (np.abs(o - want[cu_q[b] + i])[fine] <= tol[cu_q[b] + i][fine]).all(), (what, b, i)


def milliseconds(f):
    """The best of four calls."""
    best = []
    for _ in range(4):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        best.append(a.elapsed_time(b))
    return min(best)
