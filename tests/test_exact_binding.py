"""The binding of the exact operators: what it refuses before anything is launched (no GPU needed)."""
import pytest
import torch

from paper_2607_12789_b200 import binding, build

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


def _cached(B=2):
    c = binding.PagedCache.empty(6, 16, 2, 64, device="cpu")
    return c, torch.zeros(B, 4, 64, dtype=BF16), torch.zeros(B, 3, dtype=torch.int32), torch.full((B,), 5, dtype=torch.int32)


def test_a_plan_with_another_scale_or_other_flags_is_refused():
    c, Q, table, lens = _cached()
    plan = c.plan(4, 2, scale=0.3, flags=binding.FLAG_SIMT)
    for kw, what in ((dict(scale=0.125), "scale"), (dict(scale=0.0), "scale"), (dict(flags=16), "flags"),
                     (dict(scale=0.3, flags=binding.FLAG_CAUSAL), "flags")):
        with pytest.raises(ValueError, match=what):
            c.attend(Q, table, lens, plan=plan, **kw)
    for kw in ({}, dict(scale=0.3), dict(flags=binding.FLAG_SIMT), dict(scale=0.3, flags=binding.FLAG_SIMT)):
        with pytest.raises(ValueError, match="CUDA device"):   # (these agree; the tensors are the CPU's)
            c.attend(Q, table, lens, plan=plan, **kw)


def test_keys_and_values_on_different_devices_are_refused():
    keys = torch.zeros(3, 2, 16, 64, dtype=BF16)
    with pytest.raises(ValueError, match="device"):
        binding.PagedCache(keys, keys.to("meta"), 16, 64)


def test_a_check_away_from_the_workspace_s_device_is_refused(monkeypatch):
    """The header is read behind the work of the current device's stream: work on another device would not be waited for."""
    called = []
    monkeypatch.setattr(binding, "_lib", type("L", (), {"avq_check": staticmethod(lambda *a: called.append(a) or 0)}))
    monkeypatch.setattr(binding, "_raw_stream", lambda: 0)
    att, c = object.__new__(binding.ExactAttention), object.__new__(binding.PagedCache)
    att.workspace = c.header = torch.empty(256, dtype=torch.uint8)
    for check in (att.check, c.check, lambda: c.check((None, att.workspace, 1, 1))):
        with pytest.raises(ValueError, match="CUDA device"):
            check()
    assert not called



def test_a_plan_s_room_is_one_stream_s_alone(monkeypatch):
    """The first eager call's stream has the plan's own room; other streams and captures get room of the allocator's each time."""
    capturing = [True]
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: capturing[0], raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: None)
    for room, size in ((binding.ExactAttention(4, 2, 64, device="cpu").room, 4 * 2 * 148 * 256 * 66),
                       (_cached()[0].plan(4, 2).room, binding.lib().avq_cache_attend_workspace_bytes(_cached()[0].plan(4, 2)[0], 2, 1) - 256)):
        own = room.workspace.data_ptr() + 256
        capturing[0] = True
        at, kept = room.scratch(7)                          # a capture does not make its stream the plan's
        assert at == kept.data_ptr() != own and kept.numel() == room.bytes == size
        capturing[0] = False
        assert room.scratch(5) == (own, None) and room.scratch(5) == (own, None)
        a, b = room.scratch(6), room.scratch(7)
        assert len({own, a[0], b[0]}) == 3 and a[1].numel() == b[1].numel() == size
        capturing[0] = True
        assert room.scratch(5)[0] != own
    assert binding.ExactAttention(4, 2, 64, device="cpu", split=False).room.bytes == 0


def test_the_header_s_constant_and_the_binding_s_agree():
    import os
    import re
    hdr = open(os.path.join(os.path.dirname(binding.__file__), "..", "include", "avq_attn.h")).read()
    assert int(re.search(r"#define AVQ_PROMPT_SPLIT_KEYS (\d+)", hdr).group(1)) == binding.PROMPT_SPLIT_KEYS


def test_header_and_scratch_apart_are_refused_where_unusable(lib):
    OK, h = 0x1000, binding.AvqHeads(4, 2, 64, binding.AVQ_BF16, 0.125, 0)
    prompt = lambda header=OK, scratch=OK, n=1 << 30: lib.avq_prompt_attend_scratch(
        h, OK, 256, OK, 128, OK, 128, OK, OK, 1, 5, 9, 0, 256, 0, header, scratch, n, 0)
    assert prompt() == 1                                    # (no Y: rows are looked at first)
    prompt = lambda header=OK, scratch=OK, n=1 << 30: lib.avq_prompt_attend_scratch(
        h, OK, 256, OK, 128, OK, 128, OK, OK, 1, 5, 1 << 30, OK, 256, 0, header, scratch, n, 0)
    assert prompt(header=0) == 5 and prompt(header=0x1080) == 4 and prompt(scratch=0x1010) == 4
    assert prompt() == 3 and prompt(scratch=0, n=0) == 3    # (so many keys are refused: nothing is launched)
    c = binding.AvqCache(OK, OK, 10, 16, 2, 64, binding.AVQ_BF16, 16)
    n = lib.avq_cache_attend_workspace_bytes(h, 3, 1) - 256
    call = lambda header=OK, scratch=OK, n=n, Y=OK: lib.avq_cache_attend_scratch(
        h, c, OK, 256, OK, 4, OK, 3, 1, Y, 256, 0, header, scratch, n, 0)
    assert call(header=0) == 5 and call(scratch=0) == 5 and call(n=n - 1) == 5 and call(header=0x1010) == 4
    assert call(scratch=0x1010) == 4 and call(Y=0) == 1


def test_plans_can_be_copied():
    import copy
    import pickle
    a = binding.ExactAttention(6, 2, 128, scale=0.3, causal=False, flags=binding.FLAG_SIMT, device="cpu", split=False)
    b = binding.ExactAttention(6, 2, 64, device="cpu")
    for x in (a, b):
        for y in (copy.deepcopy(x), pickle.loads(pickle.dumps(x))):
            assert [getattr(y.heads, f) for f, _ in binding.AvqHeads._fields_] == [getattr(x.heads, f) for f, _ in binding.AvqHeads._fields_]
            assert y.dtype is x.dtype and y.room.bytes == x.room.bytes and y.room.header == y.workspace.data_ptr() != x.room.header
    p = _cached()[0].plan(4, 2, flags=binding.FLAG_SIMT)
    q = copy.deepcopy(p)
    assert q[2:] == p[2:] and q[0].flags == p[0].flags and q.room.header == q[1].data_ptr() != p.room.header and q[1].numel() == p[1].numel()
