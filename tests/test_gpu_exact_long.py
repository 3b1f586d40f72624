"""Exact attention at the far ends of its envelope: very many keys of one task, very many sequences of one call,
very many query heads to a key head."""
import math

import pytest
import torch

from paper_2607_12789_b200 import binding
from tests import exact_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_a_task_longer_than_the_limit_of_a_wait(causal):
    """One query over 50 million keys, not split: its tiles take longer than 0.2 s, which some waits of the kernel last."""
    n, d = 3 * 2 ** 24 + 77, 64
    if torch.cuda.mem_get_info()[0] < 5 * n * d * 2 // 2:
        pytest.skip("needs 16 GB of free device memory")
    # Every logit is 0 and every weight 1; sums of 1 and of -1 in tiles of 128 are exact in float32 up to 2^31, the last 77
    # keys' may be cut off by 4 (the distance of numbers about 2^25) for each of 8 groups of 16 keys: 32 / 2^25 = 2^-20.
    K, V = torch.zeros(n, 1, d, dtype=BF16, device="cuda"), torch.ones(n, 1, d, dtype=BF16, device="cuda")
    V[2 ** 25:, 0, 1] = -1
    Q = torch.ones(1, 1, d, dtype=BF16, device="cuda")
    att = binding.ExactAttention(1, 1, d, causal=causal, split=False)
    Y, L = att(Q, K, V, _ints([0, 1]), _ints([0, n]), lse=True)
    att.check()
    half = 2.0 ** -8
    want = torch.ones(d, dtype=torch.float64, device="cuda")
    want[1] = (2 ** 25 - (n - 2 ** 25)) / n
    assert ((Y[0, 0].double() - want).abs() <= 2.0 ** -20 + half * want.abs()).all()
    assert abs(L.item() - math.log(n)) <= 2.0 ** -20 + 2.0 ** -23 * math.log(n)


@pytest.mark.parametrize("dtype,flags,d", [(BF16, 0, 64), (BF16, 0, 128), (F32, 0, 64), (BF16, binding.FLAG_SIMT, 64)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_thousands_of_sequences(dtype, flags, d, causal):
    """4000 packed sequences of 0 to 20 tokens, padded for the reference to the longest."""
    g = torch.Generator(device="cuda")
    g.manual_seed(307)
    S, most, H, Hk = 4000, 20, 4, 2
    lens = [(7 * i) % (most + 1) for i in range(S)]
    ends = [0]
    for n in lens:
        ends.append(ends[-1] + n)
    T = ends[-1]
    Q, K, V = (torch.randn(T, m, d, device="cuda", generator=g).to(dtype) for m in (H, Hk, Hk))
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, causal=causal, flags=flags)
    Y, L = att(Q, K, V, _ints(ends), lse=True)
    att.check()
    at, i = torch.tensor(ends[:-1], device="cuda")[:, None], torch.arange(most, device="cuda")
    there = i < torch.tensor(lens, device="cuda")[:, None]
    rows = torch.where(there, at + i, torch.zeros_like(at))
    pad = lambda x: x[rows].double().repeat_interleave(H // x.shape[1], 2)
    s = att.heads.scale * torch.einsum("sihd,sjhd->shij", pad(Q), pad(K))
    seen = there[:, None, None, :] & ((i <= i[:, None]) if causal else torch.ones(most, most, dtype=torch.bool, device="cuda"))
    s = s.masked_fill(~seen, -math.inf)
    y = torch.einsum("shij,sjhd->sihd", torch.softmax(s, -1).nan_to_num(0.0), pad(V))
    l = torch.logsumexp(s, -1).transpose(1, 2)
    ty, tl = ref.tolerance(d, most, dtype, ref.most_logit(Q, K, att.heads.scale), V.abs().max().item(), not flags)
    ref.check(Y, L, y[there], l[there], ty, tl)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64)])
@pytest.mark.parametrize("G", [43, 65, 100, 128])
@pytest.mark.parametrize("lq,lk", [([3, 0, 20], [3, 0, 20]), ([1, 7], [2100, 300])], ids=["short", "split"])
def test_many_query_heads_to_a_key_head(dtype, d, G, lq, lk):
    """Tiles of a few queries, some of whose rows stay empty; the same queries over a cache, in blocks of 16 rows."""
    g = torch.Generator(device="cuda")
    g.manual_seed(311)
    Hk, page = 2, 16
    H = G * Hk
    ends = lambda lens: [sum(lens[:i]) for i in range(len(lens) + 1)]
    cq, ck = ends(lq), ends(lk)
    Q, K, V = (torch.randn(n, m, d, device="cuda", generator=g).to(dtype) for n, m in ((sum(lq), H), (sum(lk), Hk), (sum(lk), Hk)))
    att = binding.ExactAttention(H, Hk, d, dtype=dtype)
    Y, L = att(Q, K, V, _ints(cq), _ints(ck), lse=True)
    att.check()
    rY, rL = ref.prompt(Q, K, V, cq, ck, True, att.heads.scale)
    ty, tl = ref.tolerance(d, max(lk), dtype, ref.most_logit(Q, K, att.heads.scale), V.abs().max().item(), True)
    ref.check(Y, L, rY, rL, ty, tl)
    b = max(range(len(lk)), key=lambda i: lk[i])            # the longest sequence, its queries the newest of its keys
    n, nq, pages = lk[b], lq[b], -(-lk[b] // page)
    c = binding.PagedCache.empty(pages, page, Hk, d, dtype=dtype)
    c.append(K[ck[b]:ck[b + 1]], V[ck[b]:ck[b + 1]], torch.arange(n, dtype=torch.int32, device="cuda"))
    plan = c.plan(H, 1, nq)
    rows = slice(cq[b], cq[b + 1])
    Y, L = c.attend(Q[rows], torch.arange(pages, dtype=torch.int32, device="cuda")[None], _ints([n]), lse=True, plan=plan)
    c.check(plan)
    ref.check(Y, L, rY[rows], rL[rows], ty, tl)
