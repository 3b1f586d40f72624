"""Exact operators of one plan on several streams, in several graphs and by several threads at once: each call gives what it
gives alone, bit for bit."""
import threading

import pytest
import torch

from paper_2607_12789_b200 import binding

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _split_prompt(n):
    """n problems of few queries over many keys, which are split along the keys, for one plan."""
    g = torch.Generator(device="cuda")
    g.manual_seed(211)
    H, Hk, d, lq, lk = 4, 2, 128, 70, 12000
    att = binding.ExactAttention(H, Hk, d)
    rand = lambda T, heads: torch.randn(T, heads, d, device="cuda", generator=g).to(BF16)
    x = [(rand(lq, H), rand(lk, Hk), rand(lk, Hk)) for _ in range(n)]
    cu = _ints([0, lq]), _ints([0, lk])
    return att, lambda i, Y: att(*x[i], *cu, Y=Y), (lq, H, d)


def _cached(n):
    """n queries over one long cached sequence, which is shared out among all CTAs, for one plan."""
    g = torch.Generator(device="cuda")
    g.manual_seed(223)
    H, Hk, d, page, pages = 8, 2, 128, 64, 300
    c = binding.PagedCache.empty(pages, page, Hk, d)
    rand = lambda T, heads: torch.randn(T, heads, d, device="cuda", generator=g).to(BF16)
    T = pages * page
    c.append(rand(T, Hk), rand(T, Hk), torch.arange(T, dtype=torch.int32, device="cuda"))
    table, lens, q, plan = _ints([list(range(pages))]), _ints([T - 5]), [rand(1, H) for _ in range(n)], c.plan(H, 1)
    return plan, lambda i, Y: c.attend(q[i], table, lens, Y=Y, plan=plan), (1, H, d)


CASES = {"prompt": _split_prompt, "cached": _cached}
N, ROUNDS = 2, 25


def _setup(case):
    plan, call, shape = CASES[case](N)
    want = [torch.zeros(shape, dtype=BF16, device="cuda") for _ in range(N)]
    for i in range(N):
        call(i, want[i])
    torch.cuda.synchronize()
    out = [[torch.zeros(shape, dtype=BF16, device="cuda") for _ in range(ROUNDS)] for _ in range(N)]
    torch.cuda.synchronize()
    return plan, call, want, out


def _check(want, out):
    torch.cuda.synchronize()
    assert not torch.equal(want[0], want[1])
    for i in range(N):
        assert all(torch.equal(y, want[i]) for y in out[i])


@pytest.mark.parametrize("case", list(CASES))
def test_one_plan_on_two_streams(case):
    plan, call, want, out = _setup(case)
    streams = [torch.cuda.Stream() for _ in range(N)]
    for k in range(ROUNDS):
        for i in range(N):
            with torch.cuda.stream(streams[i]):
                call(i, out[i][k])
    _check(want, out)


@pytest.mark.parametrize("case", list(CASES))
def test_one_plan_in_two_graphs_replayed_at_once(case):
    plan, call, want, out = _setup(case)
    graphs, streams = [], [torch.cuda.Stream() for _ in range(N)]
    for i in range(N):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for k in range(ROUNDS):
                call(i, out[i][k])
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(N):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    _check(want, out)


@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("same", [True, False], ids=["one_stream", "two_streams"])
def test_one_plan_by_two_threads(case, same):
    plan, call, want, out = _setup(case)
    errors = []

    def work(i, stream):
        try:
            with torch.cuda.stream(stream):
                for k in range(ROUNDS):
                    call(i, out[i][k])
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    streams = [torch.cuda.current_stream() if same else torch.cuda.Stream() for _ in range(N)]
    threads = [threading.Thread(target=work, args=(i, streams[i])) for i in range(N)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    _check(want, out)


@pytest.mark.parametrize("flags", [0, binding.FLAG_SIMT], ids=["tc", "simt"])
def test_bad_pages_and_lengths_of_calls_without_a_plan_are_reported(flags):
    g = torch.Generator(device="cuda")
    g.manual_seed(227)
    c = binding.PagedCache.empty(4, 16, 2, 64)
    q = torch.randn(2, 4, 64, device="cuda", generator=g).to(BF16)
    table = _ints([[0, 1], [2, 3]])
    good = c.attend(q, table, _ints([20, 32]), flags=flags)
    c.check()
    assert torch.equal(good, c.attend(q, table, _ints([20, 32]), flags=flags, plan=c.plan(4, 2, flags=flags)))
    for t, n in ((_ints([[0, 4], [2, 3]]), [20, 32]), (_ints([[0, 1], [2, -1]]), [20, 32]), (table, [33, 32]), (table, [20, -1])):
        c.attend(q, t, _ints(n), flags=flags)
        c.attend(q, table, _ints([20, 32]), flags=flags)    # (a good call behind it takes nothing back)
        with pytest.raises(binding.AvqError, match="AVQ_ERR_INDEX"):
            c.check()
        c.check()                                           # reported once
