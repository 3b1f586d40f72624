"""Exact attention on the GPU (avq_prompt_attend, avq_cache_*) against the definitions in 64 bits."""
import math

import pytest
import torch

from paper_2607_12789_b200 import binding
from tests import exact_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SIMT = binding.FLAG_SIMT


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=F32):
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _ends(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


# ---------------------------------------------------------------- packed prompts
HEADS = [(1, 1), (4, 2), (6, 2), (8, 1), (5, 5), (14, 2)]
LENS = {"one": [1], "two": [2], "mixed": [1, 0, 37, 128, 2, 0], "edges": [127, 129, 64, 63, 65], "long": [700], "tail": [3, 513]}


def _run_prompt(dtype, flags, H, Hk, d, lq, lk, causal, seed, scale=None):
    g = _gen(seed)
    Q, K, V = _randn(g, sum(lq), H, d, dtype=dtype), _randn(g, sum(lk), Hk, d, dtype=dtype), _randn(g, sum(lk), Hk, d, dtype=dtype)
    cq, ck = _ends(lq), _ends(lk)
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, scale=scale, causal=causal, flags=flags)
    Y, L = att(Q, K, V, _ints(cq), None if lq == lk else _ints(ck), lse=True)
    att.check()
    s = att.heads.scale
    rY, rL = ref.prompt(Q, K, V, cq, ck, causal, s)
    ty, tl = ref.tolerance(d, max(lk), dtype, ref.most_logit(Q, K, s), V.abs().max().item(), not flags)
    ref.check(Y, L, rY, rL, ty, tl)


@pytest.mark.parametrize("dtype,flags,d", [(F32, 0, 64), (F32, 0, 128), (F32, 0, 8), (F32, 0, 96), (F32, 0, 256), (BF16, SIMT, 64),
                                           (BF16, SIMT, 40), (BF16, SIMT, 200), (BF16, 0, 64), (BF16, 0, 128)])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_prompt_against_64_bits(dtype, flags, d, lens, causal):
    H, Hk = HEADS[(len(lens) + d // 8) % len(HEADS)]
    _run_prompt(dtype, flags, H, Hk, d, LENS[lens], LENS[lens], causal, d + len(lens))


@pytest.mark.parametrize("dtype,flags,d", [(F32, 0, 64), (BF16, SIMT, 128), (BF16, 0, 64), (BF16, 0, 128)])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lq,lk", [([5, 1, 30, 200], [300, 64, 30, 257]), ([40, 9, 3, 140], [7, 0, 2, 20])], ids=["longer", "shorter"])
def test_prompt_with_other_keys_than_queries(dtype, flags, d, heads, lq, lk):
    """A further piece of a prompt (more keys than queries), and causal queries ahead of the first key (rows of zeros)."""
    _run_prompt(dtype, flags, *heads, d, lq, lk, True, 3)
    _run_prompt(dtype, flags, *heads, d, lq, lk, False, 4)


@pytest.mark.parametrize("dtype,flags", [(F32, 0), (BF16, SIMT), (BF16, 0)])
def test_prompt_of_wide_logits(dtype, flags):
    """Logits up to several hundred: the running maximum moves by far more than float32's exponent could hold as weights."""
    g = _gen(11)
    n, d = 400, 64
    Q, K, V = 6 * _randn(g, n, 2, d), 6 * _randn(g, n, 2, d), _randn(g, n, 2, d)
    K *= torch.linspace(0.1, 1.5, n, device="cuda")[:, None, None]
    Q, K, V = Q.to(dtype), K.to(dtype), V.to(dtype)
    for causal in (True, False):
        att = binding.ExactAttention(2, 2, d, dtype=dtype, causal=causal, flags=flags)
        Y, L = att(Q, K, V, _ints([0, n]), lse=True)
        rY, rL = ref.prompt(Q, K, V, [0, n], [0, n], causal, att.heads.scale)
        ty, tl = ref.tolerance(d, n, dtype, ref.most_logit(Q, K, att.heads.scale), V.abs().max().item(), not flags)
        ref.check(Y, L, rY, rL, ty, tl)


def test_negative_and_zero_scale_on_the_cuda_cores():
    _run_prompt(F32, 0, 2, 1, 64, [50, 3], [50, 3], True, 5, scale=-0.2)
    _run_prompt(F32, 0, 2, 1, 64, [50, 3], [50, 3], True, 6, scale=0.0)


@pytest.mark.parametrize("dtype,flags,d", [(F32, 0, 64), (BF16, SIMT, 64), (BF16, 0, 64), (BF16, 0, 128)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_a_query_does_not_see_has_no_effect(dtype, flags, d, bad):
    """Infinities and NaN in later keys, in other sequences and between sequences leave a row as it is, bit for bit."""
    g = _gen(17)
    H, Hk, lens = 4, 2, [150, 70, 31]
    cu = [5, 155, 225, 256]                                 # rows 0..4 belong to nobody, and 256.. neither
    T = 270
    Q, K, V = (_randn(g, T, n, d, dtype=dtype) for n in (H, Hk, Hk))
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, causal=True, flags=flags)
    clean = att(Q, K, V, _ints(cu))
    for at, before in ((100, 95), (155 + 69, 69), (155, 0)):   # a key of the first or second sequence
        K2, V2 = K.clone(), V.clone()
        K2[at], V2[at] = bad, bad
        for x in (K2, V2):
            x[:5], x[256:] = bad, bad
        Y = torch.full((T, H, d), 7.0, dtype=dtype, device="cuda")
        att(Q, K2, V2, _ints(cu), Y=Y)
        s = 0 if at < 155 else 1
        start, end = cu[s], cu[s + 1]
        assert torch.equal(Y[start:start + before], clean[start:start + before])
        assert torch.isnan(Y[at:end].float()).any(-1).any(-1).all() or not math.isnan(bad)
        other = [i for i in range(5, 256) if not start <= i < end]
        assert torch.equal(Y[other], clean[other])
        assert (Y[:5] == 7).all() and (Y[256:] == 7).all()
    # a single infinite value among finite keys reaches the rows that see it, in its column alone
    V2 = V.clone()
    V2[100, 0, 3] = bad
    Y = att(Q, K, V2, _ints(cu))
    want = clean.clone()
    want[100:155, :2, 3] = bad
    ok = (Y == want) | (torch.isnan(Y.float()) & torch.isnan(want.float()))
    assert ok[5:256].all()


@pytest.mark.parametrize("dtype,flags", [(F32, 0), (BF16, 0)])
def test_prompt_rows_as_views_and_on_another_stream(dtype, flags):
    g = _gen(23)
    H, Hk, d, lens = 6, 2, 64, [90, 33]
    wide = _randn(g, 123, H + 2 * Hk + 1, d, dtype=dtype)
    Q, K, V = wide[:, :H], wide[:, H:H + Hk], wide[:, H + Hk:H + 2 * Hk]
    cu = _ints(_ends(lens))
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, flags=flags)
    want = att(Q.contiguous(), K.contiguous(), V.contiguous(), cu)
    big = torch.full((123, H + 2, d), 9.0, dtype=dtype, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        att(Q, K, V, cu, Y=big[:, 1:1 + H])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(big[:, 1:1 + H], want) and (big[:, 0] == 9).all() and (big[:, -1] == 9).all()


@pytest.mark.parametrize("dtype,flags,d", [(F32, 0, 64), (F32, 0, 128), (F32, 0, 40), (BF16, SIMT, 64), (BF16, 0, 64), (BF16, 0, 128)])
def test_no_keys_at_all_and_rows_aligned_to_16_bytes_only(dtype, flags, d):
    """Without any key every row is zero and every sum -inf; rows 16 bytes further apart than they are long give the same."""
    g = _gen(27)
    H, Hk, n = 4, 2, 37
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, flags=flags)
    Q = _randn(g, n, H, d, dtype=dtype)
    none = Q[:0, :Hk]
    Y, L = att(Q, none, none, _ints([0, 20, n]), _ints([0, 0, 0]), lse=True)
    att.check()
    assert (Y == 0).all() and torch.isinf(L).all() and (L < 0).all()
    more = 16 // Q.element_size()
    apart = lambda t: torch.zeros(n * (t.shape[1] * d + more), dtype=dtype, device="cuda").as_strided(
        t.shape, (t.shape[1] * d + more, d, 1)).copy_(t)
    K, V = _randn(g, n, Hk, d, dtype=dtype), _randn(g, n, Hk, d, dtype=dtype)
    want = att(Q, K, V, _ints([0, 20, n]))
    Y = apart(torch.zeros_like(Q))
    att(apart(Q), apart(K), apart(V), _ints([0, 20, n]), Y=Y)
    assert torch.equal(Y, want)


@pytest.mark.parametrize("dtype,flags", [(F32, 0), (BF16, SIMT), (BF16, 0)])
def test_unusable_bounds_are_left_out_and_reported(dtype, flags):
    g = _gen(29)
    Q = _randn(g, 200, 2, 64, dtype=dtype)
    att = binding.ExactAttention(2, 2, 64, dtype=dtype, flags=flags)
    good = att(Q, Q, Q, _ints([0, 60, 200]))
    att.check()
    for cu in ([0, 60, 250], [-3, 60, 200], [0, 60, 2 ** 31 - 1], [0, 60, 20]):
        Y = torch.full_like(Q, 5.0)
        att(Q, Q, Q, _ints(cu), Y=Y)
        with pytest.raises(binding.AvqError, match="AVQ_ERR_INDEX"):
            att.check()
        att.check()                                        # reported once
        if cu[0] == 0:
            assert torch.equal(Y[:60], good[:60]) and (Y[60:] == 5).all()
        else:
            assert (Y[:60] == 5).all() and torch.equal(Y[60:], good[60:])


@pytest.mark.parametrize("dtype,flags", [(F32, 0), (BF16, 0)])
def test_a_captured_prompt_follows_its_inputs(dtype, flags):
    g = _gen(31)
    T, H, Hk, d = 300, 4, 2, 128
    Q, K, V = (_randn(g, T, n, d, dtype=dtype) for n in (H, Hk, Hk))
    cu = _ints([0, 100, 300])
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, flags=flags)
    Y = torch.zeros_like(Q)
    att(Q, K, V, cu, Y=Y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att(Q, K, V, cu, Y=Y)
    for ends in ([0, 250, 300], [0, 1, 2], [0, 0, 300]):
        Q.copy_(_randn(g, T, H, d))
        cu.copy_(_ints(ends))
        Y.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.full_like(Y, 3.0)
        att(Q, K, V, cu, Y=want)
        assert torch.equal(Y, want)
    att.check()


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_prompt_of_many_sequences(dtype, d, causal):
    """Far more tiles than the GPU has processors: a CTA takes one after another, long and short, with and without keys."""
    lens = [(37 * i) % 300 for i in range(70)] + [0, 1, 513]
    keys = [n + (i % 3) * 40 if i % 7 else max(n - 60, 0) for i, n in enumerate(lens)]
    _run_prompt(dtype, 0, 8, 8, d, lens, lens, causal, 13)
    _run_prompt(dtype, 0, 24, 8, d, lens, keys, causal, 14)


SPLIT = {"piece": ([64], [5000]), "one": ([1], [2500]), "several": ([3, 0, 70, 1], [2100, 3000, 64, 0]), "ahead": ([200, 30], [150, 4000]),
         "long": ([256], [20000])}


@pytest.mark.parametrize("d,heads", [(64, (4, 1)), (128, (2, 2)), (128, (16, 2)), (64, (3, 1))])
@pytest.mark.parametrize("lens", list(SPLIT))
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_few_queries_over_many_keys(d, heads, lens, causal):
    """Calls that are split along the keys, against 64 bits, twice alike, and near what a call without room for parts gives."""
    (H, Hk), (lq, lk) = heads, SPLIT[lens]
    _run_prompt(BF16, 0, H, Hk, d, lq, lk, causal, 15)
    g = _gen(16)
    Q, K, V = (_randn(g, n, m, d, dtype=BF16) for n, m in ((sum(lq), H), (sum(lk), Hk), (sum(lk), Hk)))
    cu = _ints(_ends(lq)), _ints(_ends(lk))
    whole = binding.ExactAttention(H, Hk, d, causal=causal, split=False)
    parts = binding.ExactAttention(H, Hk, d, causal=causal)
    assert whole.workspace.numel() == 256 and parts.workspace.numel() > 2 ** 20
    parts.workspace[256:].fill_(255)
    a, b, c = whole(Q, K, V, *cu), parts(Q, K, V, *cu), parts(Q, K, V, *cu)
    assert torch.equal(b, c)
    # each is within half a bfloat16 step of a weight times the largest value of the exact rows, and half a step of its own
    assert ((a.float() - b.float()).abs() <= 2 * (2.0 ** -8 * V.abs().max().item() + 2.0 ** -8 * a.float().abs()) + 1e-3).all()


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_split_calls_keep_what_is_not_seen_out(bad):
    g = _gen(18)
    H, Hk, d, lq, lk = 4, 1, 128, [20, 40], [3000, 2500]
    Q, K, V = (_randn(g, n, m, d, dtype=BF16) for n, m in ((80, H), (5700, Hk), (5700, Hk)))
    att = binding.ExactAttention(H, Hk, d)
    cq, ck = _ints([5, 25, 65]), _ints([100, 3100, 5600])
    clean = att(Q, K, V, cq, ck)
    K2, V2 = K.clone(), V.clone()
    for x in (K2, V2):
        x[:100], x[5600:], x[3100 - 5] = bad, bad, bad       # the last five queries but one of the first sequence see that key
    Y = torch.full((80, H, d), 7.0, dtype=BF16, device="cuda")
    att(Q, K2, V2, cq, ck, Y=Y)
    assert torch.equal(Y[5:20], clean[5:20]) and torch.equal(Y[25:65], clean[25:65])
    assert torch.isnan(Y[20:25].float()).any(-1).any(-1).all() and (Y[:5] == 7).all() and (Y[65:] == 7).all()
    V2 = V.clone()
    V2[3100 - 5, 0, 9] = bad
    Y = att(Q, K, V2, cq, ck)
    want = clean.clone()
    want[20:25, :, 9] = bad
    assert ((Y == want) | (torch.isnan(Y.float()) & torch.isnan(want.float())))[5:65].all()
    att.check()


def test_split_calls_leave_unusable_bounds_out_and_follow_a_captured_graph():
    g = _gen(19)
    Q, K, V = (_randn(g, n, m, 64, dtype=BF16) for n, m in ((60, 4), (6000, 2), (6000, 2)))
    att = binding.ExactAttention(4, 2, 64)
    Y = torch.full_like(Q, 5.0)
    att(Q, K, V, _ints([0, 30, 60]), _ints([0, 2500, 6001]), Y=Y)
    with pytest.raises(binding.AvqError, match="AVQ_ERR_INDEX"):
        att.check()
    # (where a call is split depends on all its sequences, and with it the rounding: held to 64 bits, not to another call)
    rY, _ = ref.prompt(Q[:30], K[:2500], V[:2500], [0, 30], [0, 2500], True, att.heads.scale)
    ty, _ = ref.tolerance(64, 2500, BF16, ref.most_logit(Q, K, att.heads.scale), V.abs().max().item(), True)
    ref.check(Y[:30], None, rY, None, ty, 0)
    assert (Y[30:] == 5).all()
    cq, ck = _ints([0, 30, 60]), _ints([0, 2500, 6000])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att(Q, K, V, cq, ck, Y=Y)
    for a, b in (([0, 1, 60], [0, 6000, 6000]), ([0, 60, 60], [0, 5500, 5600]), ([10, 20, 50], [0, 64, 4000])):
        cq.copy_(_ints(a))
        ck.copy_(_ints(b))
        Y.fill_(3.0)
        graph.replay()
        want = torch.full_like(Q, 3.0)
        att(Q, K, V, cq, ck, Y=want)
        assert torch.equal(Y, want)
    att.check()


# ---------------------------------------------------------------- the cache
def _cache(pages, page, Hk, d, dtype, bits, g, fill=True):
    c = binding.PagedCache.empty(pages, page, Hk, d, dtype=dtype, bits=bits)
    if fill:
        n = pages * page
        spread = 1 + 3 * (torch.rand(Hk, d, device="cuda", generator=g) < 0.1)
        c.append((_randn(g, n, Hk, d) * spread).to(dtype), _randn(g, n, Hk, d, dtype=dtype), torch.arange(n, dtype=torch.int32, device="cuda"))
        c.check()
    return c


TYPES = [(F32, 32), (BF16, 16), (F32, 4), (BF16, 4)]
IDS = ["f32", "bf16", "f32_in_4", "bf16_in_4"]


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
@pytest.mark.parametrize("d,dims", [(64, 64), (128, 64), (128, 128), (96, 32), (256, 256), (32, 16), (64, 0), (160, 48)])
@pytest.mark.parametrize("adjacent", [False, True], ids=["halves", "adjacent"])
def test_append_stores_what_the_definition_says(dtype, bits, d, dims, adjacent):
    g = _gen(d + dims)
    T, H, Hk, page, pages, rows = 53, 6, 3, 16, 9, 500
    wide = _randn(g, T, H + 2 * Hk, d) * torch.exp(2 * _randn(g, T, 1, 1))
    wide[7] = 0.25                                          # groups of one value: step 0
    wide = wide.to(dtype)
    Q, K, V = wide[:, :H], wide[:, H:H + Hk], wide[:, H + Hk:]
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:T].to(torch.int32)
    slots[[3, 20]] = -1
    pos = torch.randint(0, rows, (T,), device="cuda", generator=g).to(torch.int32)
    angle = torch.arange(rows, device="cuda").double()[:, None] * 100.0 ** (-torch.arange(max(dims // 2, 1), device="cuda").double() / 8)
    rot = dict(pos=pos, cos=angle.cos().float(), sin=angle.sin().float(), adjacent=adjacent) if dims else {}
    c = _cache(pages, page, Hk, d, dtype, bits, g, fill=False)
    for buf in (c.keys, c.values):
        buf.fill_(17 if bits == 4 else 17.0)
    before = [x.clone() for x in ref.held(c)]
    Qr = torch.full((T, H, d), 5.0, dtype=dtype, device="cuda")
    c.append(K, V, slots, Q=Q, Q_out=Qr, **rot)
    c.check()
    live = slots >= 0
    turn = lambda x: ref.rotate(x, pos, rot["cos"], rot["sin"], adjacent) if dims else x
    # Rotated in float32 each of the two products and their sum is rounded: 2^-24 of |x1| + |x2|, twice; then to the type.
    half = torch.finfo(dtype).eps / 2
    near = lambda got, want, x: ((got.double() - want.double()).abs()
                                 <= 2 * half * want.double().abs() + 2.0 ** -22 * x.double().abs().amax(-1, keepdim=True)).all()
    assert near(Qr[live], turn(Q)[live], Q[live]) and (Qr[~live] == 5).all()
    p, r = (slots[live] // page).long(), (slots[live] % page).long()
    after = ref.held(c)
    for got, want, x in ((after[0], turn(K)[live], K[live]), (after[1], V[live], V[live])):
        stored = got[p, r]
        if bits != 4:
            assert near(stored, want, x) and (x is not V[live] or torch.equal(stored, want.double()))
            continue
        codes, lo, step = ref.groups(want)
        exp = ref.value(codes, lo, step)
        # a code, lo or step may fall to the other side of a rounding where float32 arithmetic differs in its last bit:
        # the value then differs by a step at most, and by how far lo and step move; all but a few agree exactly
        each = step.double().repeat_interleave(32, -1)
        assert ((stored - exp).abs() <= 1.01 * each + 2.0 ** -7 * (lo.double().abs().repeat_interleave(32, -1) + 15 * each)).all()
        assert (stored != exp).double().mean().item() <= 0.01
        err = (stored - want.double()).abs()                 # and it is the nearest of the 16: half a step, and lo's rounding
        assert (err <= 0.51 * each + 2.0 ** -8 * (lo.double().abs().repeat_interleave(32, -1) + 16 * each) + 2.0 ** -22 * x.double().abs().amax()).all()
    rest = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    rest[slots[live].long()] = False
    for x, y in zip(before, after):
        a, b = (t.reshape(pages * page, Hk, d)[rest] for t in (x, y))
        assert torch.equal(a, b)
    Kr, Vr = c.read(slots, K=torch.full_like(K.contiguous(), 3.0), V=torch.full_like(V.contiguous(), 3.0))
    for got, x in ((Kr, after[0]), (Vr, after[1])):
        assert torch.equal(got[live], x[p, r].float().to(dtype)) or bits == 4 and near(got[live], x[p, r], x[p, r])
        assert (got[~live] == 3).all()
    c.append(K, V, slots, Q=Q, Q_out=Q, **rot)               # in place
    assert torch.equal(Q[live], Qr[live])
    c.check()


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
def test_slots_and_positions_out_of_range_are_skipped_and_reported(dtype, bits):
    g = _gen(41)
    c = _cache(4, 16, 2, 64, dtype, bits, g)
    x = _randn(g, 3, 2, 64, dtype=dtype)
    cos = torch.ones(10, 32, device="cuda")
    before = c.keys.clone(), c.values.clone()
    for slots, pos in (([64, -2, 2 ** 31 - 1], [0, 0, 0]), ([1, 2, 3], [10, -1, 2 ** 31 - 1])):
        c.append(x, x, _ints(slots), pos=_ints(pos), cos=cos, sin=cos)
        with pytest.raises(binding.AvqError, match="AVQ_ERR_INDEX"):
            c.check()
        assert torch.equal(c.keys, before[0]) and torch.equal(c.values, before[1])
    K = torch.full((3, 2, 64), 2.0, dtype=dtype, device="cuda")
    c.read(_ints([64, 5, -9]), K=K, V=K.clone())
    with pytest.raises(binding.AvqError, match="AVQ_ERR_INDEX"):
        c.check()
    assert (K[0] == 2).all() and (K[2] == 2).all() and not (K[1] == 2).any()
    c.append(x, x, _ints([-1, -1, -1]), pos=_ints([99, -5, 0]), cos=cos, sin=cos)
    c.check()                                               # a padded token's position is not looked at


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nan_in_a_group_read_as_nan(dtype):
    c = _cache(2, 16, 1, 64, dtype, 4, _gen(43))
    x = torch.zeros(3, 1, 64, dtype=dtype, device="cuda")
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 63] = math.inf, -math.inf, math.nan
    c.append(x, x, _ints([0, 1, 2]))
    for t in c.read(_ints([0, 1, 2])):
        bad = torch.isnan(t[:, 0].float()).view(3, 2, 32)
        assert bad[0, 0].all() and not bad[0, 1].any() and bad[1, 1].all() and not bad[1, 0].any() and bad[2, 1].all()


def _cached(c, H, lens, nq, flags, g, spare=3, scale=None, table=None):
    """Runs attend over random tables and checks every row; the rows of pages that no sequence holds are made NaN before."""
    d, page, Hk, B = c.desc.d, c.desc.page, c.desc.Hk, len(lens)
    per = [-(-n // page) for n in lens]
    order = torch.randperm(c.desc.pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((B, max(per) + spare), -7, dtype=torch.int32, device="cuda")
    at = 0
    used = torch.zeros(c.desc.pages, page, dtype=torch.bool, device="cuda")
    for b, k in enumerate(per):
        table[b, :k] = order[at:at + k]
        for j in range(k):
            used[order[at + j].long(), :min(page, lens[b] - j * page)] = True
        at += k
    n = int((~used).sum())
    if n:                                                   # what no sequence holds is NaN
        rows = (~used).flatten().nonzero().flatten().to(torch.int32)
        x = torch.full((n, Hk, d), math.nan, dtype=c.dtype, device="cuda")
        c.append(x, x, rows)
    G = H // Hk
    Q = _randn(g, B * nq, H, d, dtype=c.dtype)
    plan = c.plan(H, B, nq, scale=scale, flags=flags)
    plan[1][256:].fill_(255)
    Y, L = c.attend(Q, table, _ints(lens), lse=True, plan=plan)
    c.check(plan)
    assert all(torch.equal(a, b) for a, b in zip((Y, L), c.attend(Q, table, _ints(lens), lse=True, plan=plan)))
    keys, values = ref.held(c)
    rY, rL = torch.zeros_like(Y, dtype=torch.float64), torch.zeros_like(L, dtype=torch.float64)
    most_k = most_v = 0.0
    for b, m in enumerate(lens):
        t = torch.arange(m, device="cuda")
        k, v = (x[table[b, t // page].long(), t % page] for x in (keys, values))
        if m:
            most_k, most_v = max(most_k, k.norm(dim=-1).max().item()), max(most_v, v.abs().max().item())
        for h in range(H):
            rY[b * nq:(b + 1) * nq, h], rL[b * nq:(b + 1) * nq, h] = ref.attend(
                Q[b * nq:(b + 1) * nq, h], k[:, h // G], v[:, h // G], [m - nq + 1 + i for i in range(nq)], plan[0].scale)
    most = abs(plan[0].scale) * Q.double().norm(dim=-1).max().item() * most_k
    # (in 4 bits a weight multiplies a code, 0 .. 15 steps above lo: the range of a group, at most 2 most_v)
    ty, tl = ref.tolerance(d, max(max(lens), 1), c.dtype, most, most_v, not flags, spread=2.0 if c.desc.bits == 4 else 1.0)
    ref.check(Y, L, rY, rL, ty, tl)
    return Q, table


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
@pytest.mark.parametrize("flags,d", [(SIMT, 64), (SIMT, 96), (SIMT, 256), (0, 64), (0, 128)])
@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (12, 4), (7, 1), (40, 2)])
@pytest.mark.parametrize("page,nq,lens", [(16, 1, [1, 0, 17, 300, 16]), (64, 1, [901]), (32, 3, [2, 40, 0, 3, 129]), (48, 1, [47, 48, 49, 500])])
def test_cached_attention_against_64_bits(dtype, bits, flags, d, heads, page, nq, lens):
    g = _gen(d + page)
    H, Hk = heads
    pages = sum(-(-n // page) for n in lens) + 2
    _cached(_cache(pages, page, Hk, d, dtype, bits, g), H, lens, nq, flags, g)


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
@pytest.mark.parametrize("flags", [SIMT, 0], ids=["simt", "tc"])
def test_cached_attention_over_long_and_many_sequences(dtype, bits, flags):
    g = _gen(53)
    _cached(_cache(300, 64, 1, 64, dtype, bits, g), 4, [18000], 1, flags, g)       # one long axis over all CTAs
    lens = [1 + (37 * i) % 200 for i in range(300)]                                # more sequences than CTAs
    _cached(_cache(sum(-(-n // 16) for n in lens), 16, 2, 64, dtype, bits, g), 2, lens, 1, flags, g, spare=0)
    _cached(_cache(140, 16, 2, 128, dtype, bits, g), 8, [2000, 5, 17, 160], 9, flags, g)   # 36 rows to a key head
    _cached(_cache(4, 16, 1, 64, dtype, bits, g), 3, [0, 0], 2, flags, g)          # nothing cached at all


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
@pytest.mark.parametrize("flags", [SIMT, 0], ids=["simt", "tc"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_a_later_token_has_no_effect_on_an_earlier_query(dtype, bits, flags, bad):
    g = _gen(59)
    nq, H, lens = 5, 6, [70, 33]
    c = _cache(8, 16, 2, 64, dtype, bits, g)
    Q, table = _cached(c, H, lens, nq, flags, g)
    plan = c.plan(H, 2, nq, flags=flags)
    clean = c.attend(Q, table, _ints(lens), plan=plan)
    x = torch.full((1, 2, 64), bad, dtype=dtype, device="cuda")
    token = lens[0] - 3                                     # the third of the five new ones
    c.append(x, x, table[0, token // 16:token // 16 + 1] * 16 + token % 16)
    Y = c.attend(Q, table, _ints(lens), plan=plan)
    assert torch.equal(Y[:2], clean[:2]) and torch.equal(Y[nq:], clean[nq:])
    assert torch.isnan(Y[2:nq].float()).all()


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
@pytest.mark.parametrize("flags", [SIMT, 0], ids=["simt", "tc"])
@pytest.mark.parametrize("d,nq,lens", [(64, 1, [1, 20, 0, 333]), (128, 3, [70, 3, 500]), (64, 1, [9000]), (128, 2, [6000, 40])])
def test_nan_in_queries_and_whole_units_of_tokens_stays_nan(dtype, bits, flags, d, nq, lens):
    """Rows whose logits are all NaN, in the whole sequence or in what one warp or CTA has of it, are NaN; others are as before."""
    g = _gen(67)
    H, Hk, B = 4, 2, len(lens)
    c = _cache(sum(-(-n // 16) for n in lens) + 2, 16, Hk, d, dtype, bits, g)
    Q, table = _cached(c, H, lens, nq, flags, g)
    plan = c.plan(H, B, nq, flags=flags)
    Y, L = c.attend(Q, table, _ints(lens), lse=True, plan=plan)
    for b, n in enumerate(lens):
        if not n:
            continue
        row, Q2 = b * nq + nq - 1, Q.clone()
        Q2[row, 1] = math.nan                                # one head of the sequence's newest query
        Y2, L2 = c.attend(Q2, table, _ints(lens), lse=True, plan=plan)
        assert torch.isnan(Y2[row, 1].float()).all() and torch.isnan(L2[row, 1])
        Y2[row, 1], L2[row, 1] = Y[row, 1], L[row, 1]
        assert torch.equal(Y2, Y) and torch.equal(L2, L)
    b = B - 1                                               # 16 tokens of NaN keys in front, which every query sees
    slots = table[b, 0] * 16 + torch.arange(16, dtype=torch.int32, device="cuda")
    x = torch.full((16, Hk, d), math.nan, dtype=dtype, device="cuda")
    c.append(x, torch.zeros_like(x), slots)
    Y2, L2 = c.attend(Q, table, _ints(lens), lse=True, plan=plan)
    assert torch.isnan(Y2[b * nq:].float()).all() and torch.isnan(L2[b * nq:]).all()
    assert torch.equal(Y2[:b * nq], Y[:b * nq]) and torch.equal(L2[:b * nq], L[:b * nq])
    c.check(plan)


@pytest.mark.parametrize("dtype,flags,d", [(F32, 0, 64), (F32, SIMT, 96), (BF16, SIMT, 64), (BF16, 0, 64), (BF16, 0, 128)])
@pytest.mark.parametrize("lq,lk", [([1, 40, 200], [1, 40, 200]), ([20, 3], [3000, 2500])])
def test_a_nan_query_gives_a_nan_row(dtype, flags, d, lq, lk):
    g = _gen(68)
    H, Hk, cq = 4, 2, _ends(lq)
    Q, K, V = (_randn(g, n, m, d, dtype=dtype) for n, m in ((sum(lq), H), (sum(lk), Hk), (sum(lk), Hk)))
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, flags=flags)
    Y, L = att(Q, K, V, _ints(cq), _ints(_ends(lk)), lse=True)
    for row in [cq[s + 1] - 1 for s in range(len(lq))]:
        Q2 = Q.clone()
        Q2[row, 2] = math.nan
        Y2, L2 = att(Q2, K, V, _ints(cq), _ints(_ends(lk)), lse=True)
        assert torch.isnan(Y2[row, 2].float()).all() and torch.isnan(L2[row, 2])
        Y2[row, 2], L2[row, 2] = Y[row, 2], L[row, 2]
        assert torch.equal(Y2, Y) and torch.equal(L2, L)
    att.check()


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
@pytest.mark.parametrize("flags", [SIMT, 0], ids=["simt", "tc"])
def test_unusable_pages_and_lengths_are_left_out_and_reported(dtype, bits, flags):
    g = _gen(61)
    c = _cache(12, 16, 1, 64, dtype, bits, g)
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    Q = _randn(g, 3, 2, 64, dtype=dtype)
    plan = c.plan(2, 3, flags=flags)
    call = lambda t, n: c.attend(Q, t, _ints(n), plan=plan)
    good = call(table, [64, 40, 64])
    c.check(plan)
    broken = table.clone()
    broken[1, 1] = 12
    broken[2, 3] = -1
    Y = call(broken, [64, 40, 48])
    with pytest.raises(binding.AvqError, match="AVQ_ERR_INDEX"):
        c.check(plan)
    assert torch.equal(Y[0], good[0]) and torch.isfinite(Y.float()).all()
    for n, like in (([65, 40, 2 ** 31 - 1], [64, 40, 64]), ([64, -5, 64], [64, 0, 64])):
        Y = call(table, n)
        with pytest.raises(binding.AvqError, match="AVQ_ERR_INDEX"):
            c.check(plan)
        assert torch.equal(Y, call(table, like))
        c.check(plan)


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
def test_offsets_beyond_32_bits(dtype, bits):
    """A cache whose buffers are longer than 2^32 bytes, with the sequence at its end (and one at its beginning)."""
    Hk, d, page = 8, 128, 64
    per = Hk * page * (80 if bits == 4 else d * bits // 8)
    pages = 2 ** 32 // per + 40
    if torch.cuda.mem_get_info()[0] < 3 * pages * per:
        pytest.skip("needs 14 GB of free device memory")
    g = _gen(67)
    c = binding.PagedCache.empty(pages, page, Hk, d, dtype=dtype, bits=bits)
    n, T = 10, 600
    for first in (0, pages - n):
        ids = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
        slots = (ids[:, None] * page + torch.arange(page, dtype=torch.int32, device="cuda")).flatten()[:T].contiguous()
        K, V = _randn(g, T, Hk, d, dtype=dtype), _randn(g, T, Hk, d, dtype=dtype)
        c.append(K, V, slots)
        small = binding.PagedCache.empty(n, page, Hk, d, dtype=dtype, bits=bits)
        small.append(K, V, torch.arange(T, dtype=torch.int32, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(c.read(slots), small.read(torch.arange(T, dtype=torch.int32, device="cuda"))))
        Q = _randn(g, 1, 16, d, dtype=dtype)
        for flags in (0, SIMT):
            assert torch.equal(c.attend(Q, ids[None], _ints([T]), flags=flags),
                               small.attend(Q, torch.arange(n, dtype=torch.int32, device="cuda")[None], _ints([T]), flags=flags))
    c.check()


@pytest.mark.parametrize("dtype,bits", TYPES, ids=IDS)
def test_a_captured_step_follows_its_lengths(dtype, bits):
    """append and attend of one generation step, captured once and replayed for growing lengths."""
    g = _gen(71)
    B, H, Hk, d, page = 3, 8, 2, 64, 16
    c = _cache(60, page, Hk, d, dtype, bits, g)
    table = torch.randperm(60, device="cuda", generator=g).to(torch.int32).view(B, 20)
    lens, slots, pos = _ints([30, 1, 100]), _ints([0] * B), _ints([0] * B)
    angle = torch.arange(400, device="cuda").float()[:, None] * 0.1 ** torch.arange(32, device="cuda").float()
    K, V, Q = (_randn(g, B, n, d, dtype=dtype) for n in (Hk, Hk, H))
    plan = c.plan(H, B)
    Y, Qr = torch.zeros_like(Q), torch.zeros_like(Q)

    def step():
        c.append(K, V, slots, pos=pos, cos=angle.cos(), sin=angle.sin(), Q=Q, Q_out=Qr)
        c.attend(Qr, table, lens, Y=Y, plan=plan)

    def place():
        pos.copy_(lens - 1)
        slots.copy_(table.gather(1, (pos // page).long()[:, None])[:, 0] * page + pos % page)

    place()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        lens += _ints([1, 60, 7])
        place()
        for x in (K, V, Q):
            x.copy_(_randn(g, *x.shape))
        graph.replay()
        got = Y.clone()
        step()
        assert torch.equal(got, Y)
    c.check()
    c.check(plan)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,flags,d", [(F32, 0, 64), (BF16, SIMT, 64), (BF16, 0, 64), (BF16, 0, 128)])
def test_pieces_of_prompts_and_steps_equal_the_whole(dtype, flags, d):
    """Two sequences served piece by piece - rotated and appended, read back and attended to as packed prompts, then token by
    token over the pages - against the attention of the whole rotated sequences, with an ordinary cache."""
    g = _gen(73)
    H, Hk, page, lens = 4, 2, 16, [137, 77]
    B = len(lens)
    Q, K, V = ([_randn(g, n, m, d, dtype=dtype) for n in lens] for m in (H, Hk, Hk))
    angle = torch.arange(200, device="cuda").double()[:, None] * 50.0 ** (-torch.arange(d // 2, device="cuda").double() / (d // 2))
    cos, sin = angle.cos().float(), angle.sin().float()
    c = _cache(20, page, Hk, d, dtype, None, g, fill=False)
    table = torch.randperm(20, device="cuda", generator=g).to(torch.int32).view(B, 10)
    att = binding.ExactAttention(H, Hk, d, dtype=dtype, flags=flags)
    plan = c.plan(H, B, flags=flags)
    out = [[], []]
    turned = [[], []]
    slot = lambda b, p: (table[b, p // page] * page + p % page).to(torch.int32)
    have = [0, 0]
    for piece in ([60, 10], [70, 60]):
        now = [h + n for h, n in zip(have, piece)]
        at = [torch.arange(h, n, device="cuda") for h, n in zip(have, now)]
        cat = lambda x: torch.cat([x[b][at[b]] for b in range(B)])
        pos = torch.cat(at).to(torch.int32)
        q = c.append(cat(K), cat(V), torch.cat([slot(b, at[b]) for b in range(B)]), pos=pos, cos=cos, sin=sin, Q=cat(Q))
        all_slots = torch.cat([slot(b, torch.arange(now[b], device="cuda")) for b in range(B)])
        y = att(q, *c.read(all_slots), _ints(_ends(piece)), _ints(_ends(now)))
        for b in range(B):
            out[b].append(y[_ends(piece)[b]:_ends(piece)[b + 1]])
            turned[b].append(q[_ends(piece)[b]:_ends(piece)[b + 1]])
        have = now
    for t in range(7):
        pos = _ints(have)
        q = c.append(torch.stack([K[b][have[b]] for b in range(B)]), torch.stack([V[b][have[b]] for b in range(B)]),
                     torch.stack([slot(b, pos[b].long()) for b in range(B)]), pos=pos, cos=cos, sin=sin,
                     Q=torch.stack([Q[b][have[b]] for b in range(B)]))
        have = [h + 1 for h in have]
        y = c.attend(q, table, _ints(have), plan=plan)
        for b in range(B):
            out[b].append(y[b:b + 1])
            turned[b].append(q[b:b + 1])
    c.check()
    c.check(plan)
    att.check()
    for b in range(B):
        assert have[b] == lens[b]
        every = torch.arange(lens[b], device="cuda")
        k = c.read(slot(b, every))[0]
        q = torch.cat(turned[b])
        for got, x in ((k, K[b]), (q, Q[b])):
            want = ref.rotate(x, every, cos, sin, False)
            half = torch.finfo(dtype).eps / 2
            assert ((got.double() - want.double()).abs() <= 2 * half * want.double().abs() + 2.0 ** -22 * x.double().abs().amax()).all()
        rY, _ = ref.prompt(q, k, V[b], [0, lens[b]], [0, lens[b]], True, att.heads.scale)
        ty, _ = ref.tolerance(d, lens[b], dtype, ref.most_logit(q, k, att.heads.scale), V[b].abs().max().item(), not flags)
        ref.check(torch.cat(out[b]), None, rY, None, ty, 0)
