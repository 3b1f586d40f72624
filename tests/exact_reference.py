"""Exact attention and the paged cache in 64 bits, from the definitions, and the error a kernel may make."""
import math

import torch

F32, BF16 = torch.float32, torch.bfloat16


def attend(q, k, v, seen, scale):
    """One head: q [n,d], k, v [m,d], seen [n] = number of leading keys each query sees.  Returns (y, lse) in float64."""
    q, k, v = q.double(), k.double(), v.double()
    seen = torch.as_tensor(seen, device=q.device)[:, None]
    s = (scale * (q @ k.T)).masked_fill(torch.arange(k.shape[0], device=q.device) >= seen, -math.inf)
    if not k.shape[0]:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    l = torch.logsumexp(s, -1)
    w = torch.exp(s - torch.where(torch.isinf(l), torch.zeros_like(l), l)[:, None])
    return w @ v, l


def prompt(Q, K, V, cu_q, cu_k, causal, scale):
    G = Q.shape[1] // K.shape[1]
    Y = torch.zeros(Q.shape, dtype=torch.float64, device=Q.device)
    L = torch.zeros(Q.shape[:2], dtype=torch.float64, device=Q.device)
    for s in range(len(cu_q) - 1):
        a, b, c, e = cu_q[s], cu_q[s + 1], cu_k[s], cu_k[s + 1]
        nq, nk = b - a, e - c
        seen = [i + nk - nq + 1 for i in range(nq)] if causal else [nk] * nq
        for h in range(Q.shape[1]):
            Y[a:b, h], L[a:b, h] = attend(Q[a:b, h], K[c:e, h // G], V[c:e, h // G], seen, scale)
    return Y, L


def tolerance(d, keys, dtype, most_logit, most_v, tensor_cores, spread=1.0):
    """Largest error of an output element, before the output's own rounding, and of lse.

    u = 2^-24.  A logit is a sum of d products in float32: off by at most (d + 3) u times the sum of their magnitudes,
    here at most most_logit; the argument of exp2 and exp2 itself add 2^-21 |s| and 2^-21.  So every weight has a relative
    error e, and with the float32 sums over the keys ((keys + 8) u; tensor cores may drop bits below, so 4 u a key)
    a weighted mean of values up to most_v is off by 2 (e + sums) most_v.  Weights rounded to bfloat16 add half a step,
    2^-8, of a value each (`spread`: of the range of values that the product sees, in units of most_v)."""
    u = 2.0 ** -24
    e = (d + 3) * (4 if tensor_cores else 1) * u * most_logit + 2.0 ** -21 * (1 + most_logit)
    sums = (keys + 8) * (4 if tensor_cores else 1) * u
    y = 2 * (e + sums) * most_v
    if tensor_cores and dtype == BF16:
        y += spread * 2.0 ** -8 * most_v
    return y, e + sums + 2.0 ** -21 * most_logit


def check(Y, L, refY, refL, tol_y, tol_l):
    half = torch.finfo(Y.dtype).eps / 2
    assert torch.isfinite(Y.float()).all()
    bad = (Y.double() - refY).abs() - (tol_y + half * refY.abs())
    assert bad.max().item() <= 0, (bad.max().item(), tol_y)
    if L is not None:
        none = torch.isinf(refL)
        assert torch.equal(torch.isinf(L), none) and (L[none] < 0).all()
        off = (L.double() - refL)[~none].abs() - 2.0 ** -23 * refL[~none].abs()
        assert off.numel() == 0 or off.max().item() <= tol_l


def most_logit(Q, K, scale):
    """Bound of scale * sum |q_i k_i| over all pairs."""
    return abs(scale) * (Q.double().norm(dim=-1).max() * K.double().norm(dim=-1).max()).item()


# ---------------------------------------------------------------- cache
def rotate(x, pos, cos, sin, adjacent):
    """x [T,n,d] in its type, rotated in float64 (the products of the given float32 tables), rounded once to the type."""
    dims = 2 * cos.shape[1]
    out = x.double().clone()
    for k in range(dims // 2):
        i, j = (2 * k, 2 * k + 1) if adjacent else (k, k + dims // 2)
        c, s = cos[pos.long(), k].double()[:, None], sin[pos.long(), k].double()[:, None]
        out[..., i] = x[..., i].double() * c - x[..., j].double() * s
        out[..., j] = x[..., j].double() * c + x[..., i].double() * s
    return out.to(x.dtype)


def groups(x):
    """(codes, lo, step) of x [..., d] by the definition: codes [..., d] float64, lo and step [..., d/32] bfloat16."""
    g = x.double().unflatten(-1, (-1, 32))
    lo = g.amin(-1).to(BF16)
    step = ((g.amax(-1) - lo.double()) / 15).to(BF16)
    by = step.double()[..., None]
    c = torch.where(by > 0, (g - lo.double()[..., None]) / torch.where(by > 0, by, torch.ones_like(by)), torch.zeros_like(g))
    return c.round().clamp(0, 15).flatten(-2), lo, step


def value(codes, lo, step):
    return (lo.double()[..., None] + codes.unflatten(-1, (-1, 32)) * step.double()[..., None]).flatten(-2)


def unpack(buf, page, d):
    """Codes [..., page, d] (float64), lo and step [..., page, d/32] of a 4-bit cache's bytes [..., page * 5 d / 8]."""
    rows = buf[..., :page * d // 2].unflatten(-1, (page, d // 2)).long()
    codes = torch.empty(*rows.shape[:-1], d, dtype=torch.float64, device=buf.device)
    for i in range(d):
        g, t, e = i // 32, i % 32 // 8, i % 8
        codes[..., i] = ((rows[..., t * (d // 8) + 4 * g + e // 2] >> (4 * (e % 2))) & 15).double()
    par = buf[..., page * d // 2:].contiguous().view(BF16).unflatten(-1, (page, d // 32, 2))
    return codes, par[..., 0], par[..., 1]


def held(cache):
    """What the cache stands for: keys and values [pages, page, Hk, d] in float64."""
    c = cache.desc
    out = []
    for buf in (cache.keys, cache.values):
        x = value(*unpack(buf, c.page, c.d)) if c.bits == 4 else buf.double()
        out.append(x.transpose(1, 2))
    return out
