"""Logits of float32 queries over a cache: sequences of one token, whose lse is the logit, against 64 bits."""
import math

import pytest
import torch

from paper_2607_12789_b200 import binding
from tests import exact_reference as ref

pytestmark = pytest.mark.gpu
F32 = torch.float32
U = 2.0 ** -24


def _logits(d, bits, heads):
    """(lse, the logits in 64 bits, scale * sum |q| |k|) of 200 sequences of one token."""
    g = torch.Generator(device="cuda")
    g.manual_seed(401 + d)
    (H, Hk), B, page = heads, 200, 16
    c = binding.PagedCache.empty(B, page, Hk, d, dtype=F32, bits=bits)
    K = torch.randn(B, Hk, d, device="cuda", generator=g)
    slots = page * torch.arange(B, dtype=torch.int32, device="cuda")
    c.append(K, K, slots)
    Q = torch.randn(B, H, d, device="cuda", generator=g)
    plan = c.plan(H, B)
    lens = torch.ones(B, dtype=torch.int32, device="cuda")
    _, L = c.attend(Q, torch.arange(B, dtype=torch.int32, device="cuda")[:, None].contiguous(), lens, lse=True, plan=plan)
    c.check(plan)
    k = ref.held(c)[0][:, 0].repeat_interleave(H // Hk, 1)
    s = plan[0].scale * Q.double() * k
    return L.double(), s.sum(-1), s.abs().sum(-1)


def _rms(x):
    return x.square().mean().sqrt().item()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(4, 2), (16, 1)])
def test_float32_queries_over_4_bits(d, heads):
    """A group of 32 dimensions is about 12 roundings of numbers of at most its share A / G of A = scale * sum |q| |k|: the sums of
    the high parts, their additions, the middle, the sum of the queries.  Independent ones of u / sqrt(3) each (rounded), twice
    that (cut off), in G groups: 2 sqrt(12 / 3) u A / G sqrt(G) = 4 u A / sqrt(G), and two of the result, u |s| each."""
    L, s, A = _logits(d, 4, heads)
    assert _rms(L - s) <= 4 * U * _rms(A) / math.sqrt(d / 32) + 2 * U * _rms(s)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(4, 2), (16, 1)])
def test_float32_rows(d, heads):
    """32 dimensions are a chain of 4 cut-off sums, u of a partial sum each on average, in one direction; the partial sums of
    random terms are at most sqrt(32 / d) of the result: 4 u of that, in d / 32 independent groups 4 u |s|.  The operands' parts
    leave out a product of two low parts, uniform up to 2^-11 of their operands: 2^-22 / 3 of a term, 1.3 u |s| over random terms,
    and the rounding of a low part to 2^-11 of it, uniform, twice: 2^-23 / 3, 0.7 u |s| each; 1.7 u |s| of the three.
    The additions in registers and the roundings of the result, u / sqrt(3) each, are below 2 u |s|: 8 u |s|."""
    L, s, _ = _logits(d, 32, heads)
    assert _rms(L - s) <= 8 * U * _rms(s)
