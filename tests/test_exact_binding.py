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

