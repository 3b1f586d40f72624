"""Infinities that float32 operands of exact attention hold, against the definition and against the CUDA-core kernels.

A logit with an infinity is one (its sign that of the finite factor's times the infinity's), or NaN where the factor is zero:
a weight of zero, or a row of NaN.  The tensor-core kernels work with parts of the operands and have to give the same."""
import math

import pytest
import torch

from paper_2607_12789_b200 import binding
from tests import exact_reference as ref

pytestmark = pytest.mark.gpu
F32 = torch.float32
SIMT = binding.FLAG_SIMT


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


KINDS = ["exact", "inexact", "large"]


def _factors(kind, g, rows, H, d, dim):
    """Queries whose element `dim` is exact in the parts' format, is not, or is so large that its product with a stand-in for
    an infinity could overflow; signs in turn."""
    Q = _randn(g, rows, H, d)
    sign = 1.0 - 2.0 * ((torch.arange(rows, device="cuda")[:, None] + torch.arange(H, device="cuda")) % 2)
    if kind == "exact":
        Q = Q.to(torch.bfloat16).float()
        Q[:, :, dim] = sign * 0.5
    elif kind == "inexact":
        Q[:, :, dim] = sign * (0.3 + torch.rand(rows, H, device="cuda", generator=g))
    else:
        Q[:, :, dim] = sign * (1000.0 + 4.0e4 * torch.rand(rows, H, device="cuda", generator=g))
    return Q


def _expect(Q, K, V, seen, scale, d):
    """(rows that are finite by the definition, their outputs and sums in 64 bits, tolerances): one head."""
    s = scale * (Q.double() @ K.double().T)
    hidden = torch.arange(K.shape[0], device="cuda") >= torch.as_tensor(seen, device="cuda")[:, None]
    s = s.masked_fill(hidden, -math.inf)
    ok = ~(torch.isnan(s) | (s == math.inf)).any(-1)
    top = s.amax(-1, keepdim=True)
    w = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = w.sum(-1, keepdim=True)
    y = (w @ V.double()) / torch.where(total > 0, total, torch.ones_like(total))
    l = (torch.log(total) + top)[:, 0]
    # (a dimension in which every finite key is zero adds exact zeros to finite logits)
    finite = torch.where(torch.isfinite(K), K, torch.zeros_like(K))
    ty, tl = ref.tolerance(d, K.shape[0], F32, ref.most_logit(Q * finite.any(0), finite, scale), V.abs().max().item(), True)
    return ok, y, l, ty, tl


def _compare(Y, L, ok, y, l, ty, tl):
    assert torch.isnan(Y[~ok]).all()
    if ok.any():
        ref.check(Y[ok], L[ok], y[ok], l[ok], ty, tl)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("inf", [math.inf, -math.inf])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_one_infinite_element_of_a_key_of_a_prompt(d, kind, inf, causal):
    g = _gen(101 + d)
    n, H, Hk, dim = 150, 4, 2, 37
    Q, K, V = _factors(kind, g, n, H, d, dim), _randn(g, n, Hk, d), _randn(g, n, Hk, d)
    K[:, :, dim] = 0.0                                      # (finite keys: the large elements stay out of their logits)
    K[3, 0, dim] = K[90, 1, dim] = K[149, 0, dim] = inf
    Q[10, :, dim] = 0.0
    out = []
    for flags in (0, SIMT):
        att = binding.ExactAttention(H, Hk, d, dtype=F32, causal=causal, flags=flags)
        Y, L = att(Q, K, V, _ints([0, n]), lse=True)
        att.check()
        seen = [i + 1 if causal else n for i in range(n)]
        some = 0
        for h in range(H):
            want = _expect(Q[:, h], K[:, h // 2], V[:, h // 2], seen, att.heads.scale, d)
            some += int((want[0] & torch.tensor([x > 90 for x in seen], device="cuda")).sum())
            _compare(Y[:, h], L[:, h], *want)
        assert some > 20                                    # rows that see an infinite element and are finite
        out.append(torch.isnan(Y))
    assert torch.equal(*out)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("inf", [math.inf, -math.inf])
@pytest.mark.parametrize("heads,nq", [((4, 2), 1), ((12, 1), 1), ((4, 2), 3)])
def test_one_infinite_element_of_a_cached_key(d, kind, inf, heads, nq):
    g = _gen(103 + d)
    (H, Hk), page, lens, dim = heads, 16, [70, 9, 333], 21
    B = len(lens)
    per = [-(-n // page) for n in lens]
    pages = sum(per)
    c = binding.PagedCache.empty(pages, page, Hk, d, dtype=F32)
    table = torch.zeros(B, max(per), dtype=torch.int32, device="cuda")
    order, at = torch.randperm(pages, device="cuda", generator=g).to(torch.int32), 0
    Q = _factors(kind, g, B * nq, H, d, dim)
    rows = []
    for b, k in enumerate(per):
        table[b, :k] = order[at:at + k]
        at += k
        K, V = _randn(g, lens[b], Hk, d), _randn(g, lens[b], Hk, d)
        K[:, :, dim] = 0.0
        K[lens[b] // 2, :, dim] = K[lens[b] - 1, 0, dim] = inf
        t = torch.arange(lens[b], device="cuda")
        c.append(K, V, (table[b, t // page] * page + t % page).to(torch.int32))
        rows.append((K, V))
    out = []
    for flags in (0, SIMT):
        plan = c.plan(H, B, nq, flags=flags)
        Y, L = c.attend(Q, table, _ints(lens), lse=True, plan=plan)
        c.check(plan)
        some = 0
        for b, (K, V) in enumerate(rows):
            part, seen = slice(b * nq, (b + 1) * nq), [lens[b] - nq + 1 + i for i in range(nq)]
            for h in range(H):
                want = _expect(Q[part, h], K[:, h * Hk // H], V[:, h * Hk // H], seen, plan[0].scale, d)
                some += int(want[0].sum())
                _compare(Y[part, h], L[part, h], *want)
        assert some > 0
        out.append(torch.isnan(Y))
    assert torch.equal(*out)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inf", [math.inf, -math.inf])
def test_an_infinite_query_element(d, inf):
    """Every logit of such a row is an infinity: all of them negative, and no key has a weight; one positive, and it is NaN."""
    g = _gen(107 + d)
    n, H, dim = 60, 2, 5
    Q, K, V = _randn(g, n, H, d), _randn(g, n, H, d), _randn(g, n, H, d)
    K[:, 0, dim], K[:, 1, dim] = -0.5 * math.copysign(1, inf), -math.copysign(1, inf) * (0.3 + torch.rand(n, device="cuda", generator=g))
    Q[7, :, dim] = Q[40, :, dim] = inf
    K2 = K.clone()
    K2[20, :, dim] *= -1                                    # row 40 sees this one, row 7 does not (causal)
    c = binding.PagedCache.empty(4, 16, H, d, dtype=F32)
    for flags in (0, SIMT):
        att = binding.ExactAttention(H, H, d, dtype=F32, flags=flags)
        Y, L = att(Q, K, V, _ints([0, n]), lse=True)
        assert (Y[[7, 40]] == 0).all() and (L[[7, 40]] == -math.inf).all()
        Y2, L2 = att(Q, K2, V, _ints([0, n]), lse=True)
        assert (Y2[7] == 0).all() and torch.isnan(Y2[40]).all()
        rest = [i for i in range(n) if i not in (7, 40)]
        assert torch.isfinite(Y[rest]).all() and torch.isfinite(Y2[rest]).all()
        for k, ok in ((K, True), (K2, False)):
            c.append(k, V, torch.arange(n, dtype=torch.int32, device="cuda"))
            y, l = c.attend(Q[40:41], _ints([[0, 1, 2, 3]]), _ints([n]), lse=True, flags=flags)
            assert (y == 0).all() and (l == -math.inf).all() if ok else torch.isnan(y).all()


def _few(n, d, H, logits):
    """Queries whose logits over n keys are the given ones (a scale of 1/8), values of 1."""
    Q, K = torch.zeros(1, H, d, device="cuda"), torch.zeros(n, H, d, device="cuda")
    Q[:, :, 0], K[:, :, 0] = 1.0, 8 * torch.tensor(logits, device="cuda")[:, None]
    return Q, K, torch.ones(n, H, d, device="cuda")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inf", [math.inf, -math.inf])
@pytest.mark.parametrize("flags", [0, SIMT], ids=["tc", "simt"])
def test_several_infinite_values_of_large_weights(d, inf, flags):
    """Logits of 0 first, then logits that make weights of nearly 2^8 relative to those: values of the same infinity add up to it."""
    n, H = 128, 2
    Q, K, V = _few(n, d, H, [0.0] * 64 + [7.9 * math.log(2)] * 64)
    V[70:74, :, 5] = inf
    c = binding.PagedCache.empty(n // 16, 16, H, d, dtype=F32)
    c.append(K, V, torch.arange(n, dtype=torch.int32, device="cuda"))
    y = c.attend(Q, torch.arange(n // 16, dtype=torch.int32, device="cuda")[None], _ints([n]), scale=0.125, flags=flags)
    assert (y[0, :, 5] == inf).all()
    y[:, :, 5] = 1.0
    assert ((y - 1).abs() <= 1e-5).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inf", [math.inf, -math.inf])
@pytest.mark.parametrize("flags", [0, SIMT], ids=["tc", "simt"])
@pytest.mark.parametrize("powers", [range(-104, -96), range(-112, -104), range(-120, -112), range(-125, -120)])
def test_an_infinite_value_of_a_tiny_weight(d, inf, flags, powers):
    """A weight near the smallest of float32 (2^-126) is one all the same, powers of two among them: an infinity under it
    reaches the row."""
    n = 64
    H = len(powers)
    Q, K, V = torch.zeros(1, H, d, device="cuda"), torch.zeros(n, H, d, device="cuda"), torch.ones(n, H, d, device="cuda")
    Q[:, :, 0], K[40, :, 0] = 1.0, torch.tensor(powers, device="cuda").float()
    V[40, :, 5] = inf
    c = binding.PagedCache.empty(n // 16, 16, H, d, dtype=F32)
    c.append(K, V, torch.arange(n, dtype=torch.int32, device="cuda"))
    att = binding.ExactAttention(H, H, d, dtype=F32, scale=math.log(2), causal=False, flags=flags)
    for y in (att(Q, K, V, _ints([0, 1]), _ints([0, n])),
              c.attend(Q, torch.arange(n // 16, dtype=torch.int32, device="cuda")[None], _ints([n]), scale=math.log(2), flags=flags)):
        assert (y[0, :, 5] == inf).all()
        y[:, :, 5] = 1.0
        assert ((y - 1).abs() <= 1e-5).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inf", [math.inf, -math.inf])
@pytest.mark.parametrize("flags", [0, SIMT], ids=["tc", "simt"])
@pytest.mark.parametrize("n", [150, 2500])
def test_one_infinite_element_of_a_bfloat16_key(d, inf, flags, n):
    """Prompts (the longer one split along its keys) and a cache, the last 40 queries."""
    g = _gen(109 + d)
    nq, H, Hk, dim, BF16 = 40, 4, 2, 37, torch.bfloat16
    Q, K, V = _factors("exact", g, nq, H, d, dim), _randn(g, n, Hk, d), _randn(g, n, Hk, d)
    K[:, :, dim] = 0.0
    K[3, 0, dim] = K[n // 2, 1, dim] = K[n - 2, 0, dim] = inf
    Q, K, V = Q.to(BF16), K.to(BF16), V.to(BF16)
    att = binding.ExactAttention(H, Hk, d, flags=flags)
    c = binding.PagedCache.empty(-(-n // 16), 16, Hk, d)
    c.append(K, V, torch.arange(n, dtype=torch.int32, device="cuda"))
    table = torch.arange(-(-n // 16), dtype=torch.int32, device="cuda")[None]
    plan = c.plan(H, 1, nq, flags=flags)
    for Y, L in (att(Q, K, V, _ints([0, nq]), _ints([0, n]), lse=True), c.attend(Q, table, _ints([n]), lse=True, plan=plan)):
        some = 0
        for h in range(H):
            ok, y, l, _, _ = _expect(Q[:, h], K[:, h // 2], V[:, h // 2], [n - nq + 1 + i for i in range(nq)], att.heads.scale, d)
            finite = torch.where(torch.isfinite(K), K, torch.zeros_like(K))
            ty, tl = ref.tolerance(d, n, BF16, ref.most_logit(Q, finite, att.heads.scale), V.abs().max().item(), not flags)
            some += int(ok.sum())
            _compare(Y[:, h], L[:, h], ok, y, l, ty, tl)
        assert some > 40
    att.check()
    c.check(plan)
