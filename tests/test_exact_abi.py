"""Exact attention and the paged cache: what is refused on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2607_12789_b200 import binding, build
from tests import exact_reference as ref

OK, ODD = 0x1000, 0x1008


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _heads(**kw):
    base = dict(H=4, Hk=2, d=64, dtype=binding.AVQ_BF16, scale=0.125, flags=0)
    base.update(kw)
    return binding.AvqHeads(*base.values())


def _cache(**kw):
    base = dict(keys=OK, values=OK, pages=10, page=16, Hk=2, d=64, dtype=binding.AVQ_BF16, bits=16)
    base.update(kw)
    return binding.AvqCache(*base.values())


def _prompt(lib, h, Q=OK, qs=256, K=OK, ks=128, V=OK, vs=128, cq=OK, ck=OK, S=1, Tq=5, Tk=9, Y=OK, ys=256, L=0, ws=OK, n=256):
    return lib.avq_prompt_attend(h, Q, qs, K, ks, V, vs, cq, ck, S, Tq, Tk, Y, ys, L, ws, n, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(H=0), 2), (dict(Hk=0), 2), (dict(H=5), 2), (dict(d=0), 2), (dict(dtype=3), 2), (dict(scale=float("inf")), 2),
    (dict(flags=1), 2), (dict(flags=16), 2), (dict(d=60, flags=2), 3), (dict(d=264, flags=2), 3), (dict(H=70000, Hk=1, flags=2), 3),
    (dict(d=96), 3), (dict(scale=0.0), 3), (dict(scale=-1.0), 3), (dict(H=258, Hk=2), 3),
])
def test_unusable_heads_are_refused(lib, kw, want):
    h = _heads(**kw)
    assert lib.avq_prompt_workspace_bytes(h) == 0
    assert _prompt(lib, h, qs=1 << 20, ys=1 << 20) == want


def test_room_for_parts(lib):
    """Two parts for each of 148 CTAs: 256 rows of d values, a maximum and a sum; none where no kernel splits."""
    assert lib.avq_prompt_workspace_bytes(_heads()) == 256
    assert lib.avq_prompt_split_bytes(_heads()) == 256 + 4 * 2 * 148 * 256 * 66
    assert lib.avq_prompt_split_bytes(_heads(d=128)) == 256 + 4 * 2 * 148 * 256 * 130
    assert lib.avq_prompt_split_bytes(_heads(dtype=0)) == lib.avq_prompt_split_bytes(_heads(flags=2)) == 256
    assert lib.avq_prompt_split_bytes(_heads(d=96)) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(S=-1), 2), (dict(Tq=-1), 2), (dict(Tk=-1), 2), (dict(ck=0), 2), (dict(qs=248), 2), (dict(ks=120), 2), (dict(ys=0), 2),
    (dict(Q=0), 1), (dict(K=0), 1), (dict(V=0), 1), (dict(Y=0), 1), (dict(cq=0), 1), (dict(Q=ODD), 4), (dict(V=ODD), 4),
    (dict(qs=260), 4), (dict(vs=1 << 31), 3), (dict(S=(1 << 20) + 1), 3), (dict(ws=0), 5), (dict(n=255), 5), (dict(ws=0x1080), 4),
])
def test_unusable_prompts_are_refused(lib, kw, want):
    assert _prompt(lib, _heads(), **kw) == want


def test_calls_without_work_do_nothing(lib):
    assert _prompt(lib, _heads(), S=0) == 0 and _prompt(lib, _heads(), Tq=0, Q=0, Y=0) == 0
    assert lib.avq_cache_append(_cache(), 0, 128, 0, 128, 0, 0, None, 0, 0, 0, 0, 0, 0, 0) == 0
    assert lib.avq_cache_read(_cache(), 0, 0, 0, 0, 0, 0, 0, 0) == 0
    assert lib.avq_cache_attend(_heads(), _cache(), 0, 0, 0, 0, 0, 0, 1, 0, 0, 0, 0, 0, 0) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(pages=0), 2), (dict(page=0), 2), (dict(Hk=-1), 2), (dict(d=0), 2), (dict(dtype=9), 2), (dict(bits=8), 2), (dict(bits=32), 2),
    (dict(page=24), 3), (dict(page=2048), 3), (dict(d=60), 3), (dict(d=72, bits=4), 3), (dict(pages=1 << 27), 3), (dict(d=512), 3),
])
def test_unusable_caches_are_refused(lib, kw, want):
    c = _cache(**kw)
    assert lib.avq_cache_bytes(c) == 0
    assert lib.avq_cache_read(c, OK, 1, OK, 1 << 20, OK, 1 << 20, 0, 0) == want
    assert lib.avq_cache_append(c, OK, 1 << 20, OK, 1 << 20, OK, 1, None, 0, 0, 0, 0, 0, 0, 0) == want


def test_bytes(lib):
    assert lib.avq_cache_bytes(_cache()) == 10 * 2 * 16 * 64 * 2
    assert lib.avq_cache_bytes(_cache(bits=4)) == 10 * 2 * 16 * 40
    assert lib.avq_cache_bytes(_cache(pages=1 << 26, bits=4)) == (1 << 26) * 2 * 16 * 40


def test_unusable_rows_are_refused(lib):
    put = lambda c=None, K=OK, ks=128, V=OK, vs=128, sl=OK, T=3, rot=None, Q=0, qs=0, H=0, Qo=0, qo=0, hd=0: \
        lib.avq_cache_append(c or _cache(), K, ks, V, vs, sl, T, rot, Q, qs, H, Qo, qo, hd, 0)
    rot = lambda **kw: binding.AvqRotation(*dict(dict(cos=OK, sin=OK, pos=OK, rows=8, dims=32, adjacent=0), **kw).values())
    assert put(K=0) == 1 and put(V=0) == 1 and put(sl=0) == 1 and put(_cache(values=0)) == 1 and put(_cache(keys=ODD)) == 4
    assert put(ks=120) == 2 and put(vs=132) == 4 and put(V=ODD) == 4 and put(T=-1) == 2 and put(hd=0x1010) == 4
    assert put(rot=rot(dims=40)) == 2 and put(rot=rot(dims=80)) == 2 and put(rot=rot(cos=ODD)) == 4
    assert put(rot=rot(pos=0)) == 1 and put(rot=rot(sin=0)) == 1 and put(rot=rot(rows=-1)) == 2
    assert put(Q=OK, qs=256, H=0, Qo=OK, qo=256) == 2 and put(Q=OK, qs=256, H=4, Qo=0, qo=256) == 1
    assert put(Q=OK, qs=200, H=4, Qo=OK, qo=256) == 2
    get = lambda c=None, sl=OK, T=3, K=OK, ks=128, V=OK, vs=128: lib.avq_cache_read(c or _cache(), sl, T, K, ks, V, vs, 0, 0)
    assert get(sl=0) == 1 and get(K=0) == 1 and get(vs=120) == 2 and get(V=ODD) == 4 and get(T=-1) == 2


def test_numbers_of_rows_that_pass_32_bits_in_sums_are_refused(lib):
    many = 1 << 30
    one = _heads(H=1, Hk=1)
    assert _prompt(lib, one, Tq=many) == 3 and _prompt(lib, one, Tk=many) == 3 and _prompt(lib, one, ck=0, Tq=2 ** 31 - 1, Tk=2 ** 31 - 1) == 3
    c = _cache(Hk=1)
    for T in (many, 2 ** 31 - 1):
        assert lib.avq_cache_append(c, OK, 64, OK, 64, OK, T, None, 0, 0, 0, 0, 0, 0, 0) == 3
        assert lib.avq_cache_read(c, OK, T, OK, 64, OK, 64, 0, 0) == 3
    n = lib.avq_cache_attend_workspace_bytes(one, 1, 1)
    assert lib.avq_cache_attend(one, c, OK, 64, OK, many // 16, OK, 1, 1, OK, 64, 0, OK, n, 0) == 3


def test_unusable_cached_calls_are_refused(lib):
    n = lib.avq_cache_attend_workspace_bytes(_heads(), 3, 1)
    assert n > 256
    call = lambda h=None, c=None, Q=OK, qs=256, tb=OK, tp=4, ln=OK, B=3, nq=1, Y=OK, ys=256, ws=OK, nb=n: \
        lib.avq_cache_attend(h or _heads(), c or _cache(), Q, qs, tb, tp, ln, B, nq, Y, ys, 0, ws, nb, 0)
    assert call(_heads(flags=binding.FLAG_CAUSAL)) == 2 and call(_heads(d=96), _cache(d=96), 384) == 3
    assert call(_heads(scale=-1.0)) == 3 and call(_heads(H=4, Hk=4)) == 2 and call(_heads(dtype=0)) == 2
    assert call(B=-1) == 2 and call(nq=0) == 2 and call(tp=-1) == 2 and call(tp=1 << 28) == 3
    assert call(Q=0) == 1 and call(tb=0) == 1 and call(ln=0) == 1 and call(Y=0) == 1 and call(qs=240) == 2 and call(Y=ODD) == 4
    assert call(ws=0) == 5 and call(nb=n - 1) == 5 and call(ws=0x1010) == 4 and call(c=_cache(keys=0)) == 1


def test_the_binding_refuses_what_it_cannot_pass_on():
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        binding.ExactAttention(4, 2, 64, dtype=torch.float16, device="cpu")
    with pytest.raises(binding.AvqError, match="UNSUPPORTED"):
        binding.ExactAttention(4, 2, 96, device="cpu")
    a = binding.ExactAttention(4, 2, 64, device="cpu")
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be"):
        a(q, q, q, cu)
    k = q[:, :2]
    with pytest.raises(ValueError, match="CUDA device"):
        a(q, k, k, cu)
    with pytest.raises(ValueError, match="int32"):
        a(q, k, k, cu.long())
    with pytest.raises(TypeError):
        a(q.float(), k, k, cu)
    with pytest.raises(ValueError, match="dense"):
        a(q.transpose(0, 1).contiguous().transpose(0, 1), k, k, cu)
    with pytest.raises(ValueError, match="cu_k"):
        a(q, k[:3], k[:3], cu)
    with pytest.raises(ValueError):
        binding.PagedCache(torch.zeros(3, 2, 16, 64), torch.zeros(3, 2, 16, 64), 16, 64)
    c = binding.PagedCache.empty(3, 16, 2, 64, bits=4, device="cpu")
    with pytest.raises(ValueError, match="positions"):
        c.append(k, k, torch.zeros(5, dtype=torch.int32), cos=torch.zeros(4, 32))
    with pytest.raises(ValueError, match="CUDA device"):
        c.read(torch.zeros(5, dtype=torch.int32))
    with pytest.raises(ValueError, match="same number of rows"):
        c.attend(q, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def test_the_reference_against_written_out_numbers():
    """Two keys, one query: weights by math.exp; codes of 0..31 in one group: lo 0, step 31/15 in bfloat16."""
    import math
    q, k, v = torch.tensor([[1.0, 2.0]]), torch.tensor([[3.0, 0.0], [0.0, 1.0]]), torch.tensor([[1.0, 0.0], [0.0, 4.0]])
    y, l = ref.attend(q, k, v, [2], 0.5)
    a, b = math.exp(1.5), math.exp(1.0)
    assert abs(y[0, 0].item() - a / (a + b)) < 1e-14 and abs(y[0, 1].item() - 4 * b / (a + b)) < 1e-14
    assert abs(l.item() - math.log(a + b)) < 1e-14
    y, l = ref.attend(q, k, v, [0], 0.5)
    assert y.abs().max() == 0 and l.item() == -math.inf
    c, lo, step = ref.groups(torch.arange(32.0))
    assert lo.item() == 0 and abs(step.item() - 2.0625) < 1e-12 and c[31].item() == 15 and c[1].item() == 0 and c[2].item() == 1
    c, lo, step = ref.groups(torch.full((32,), 3.0))
    assert step.item() == 0 and c.max() == 0 and (ref.value(c, lo, step) == 3).all()
    buf = torch.zeros(16 * 40, dtype=torch.uint8)
    buf[2 * 32 + 1 * 8 + 4 * 1 + 1] = 0x9 | 0x3 << 4         # row 2, t = 1, group 1: dimensions 32 + 8 + 2 and + 3
    codes, _, _ = ref.unpack(buf, 16, 64)
    assert codes[2, 42] == 9 and codes[2, 43] == 3 and codes.sum() == 12
