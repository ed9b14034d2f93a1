"""CPU tests of what the training layer refuses before it launches anything. Tensors are on the CPU; the library's plans
and positions are its own, its launches are replaced by a note of their names."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import RotaryPrefill
from paper_2608_06146_gb300.inputs import PageSpec

HQ, HKV, D, BF16 = 4, 2, 128, torch.bfloat16
PAGES = [PageSpec(20, 4, [0, 2], [7, 3])]


@pytest.fixture
def launched(monkeypatch):
    pbuild.build()
    real, names = pa.load_library(), []

    class Lib:
        def __getattr__(self, name):
            if name in ("padoc_qk_rotary", "padoc_qk_rotary_bwd", "padoc_ancestor_prefill_attn", "padoc_ancestor_prefill_bwd"):
                return lambda *a: names.append(name) or 0
            return getattr(real, name)
    # (the workspace's size asks for the number of SMs)
    monkeypatch.setattr(pa, "padoc_qk_rotary_bwd_workspace_size", lambda rotary, rows: 4096)
    monkeypatch.setattr(pa, "_dev", lambda t, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(pa, "_current_device", lambda: -1)
    monkeypatch.setattr(pa, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(pa, "load_library", lambda *a: Lib())
    return names


def layer(norm=True):
    w = [torch.ones(D, dtype=BF16) for _ in range(2)] if norm else (None, None)
    rot = pa.Rotary(np.ones(D // 2), head_dim=D, q_weight=w[0], k_weight=w[1], device="cpu")
    return RotaryPrefill(PAGES, rot, HQ, HKV, BF16, "cpu", training=True)


def tensors(T):
    z = lambda h, dt=BF16: torch.zeros((T, h, D), dtype=dt)
    return dict(q=z(HQ), k=z(HKV), v=z(HKV), out=z(HQ), dout=z(HQ), lse=torch.zeros((T, HQ)), scale=0.1, dq=z(HQ), dk=z(HKV),
                dv=z(HKV), dq_weight=torch.zeros(D), dk_weight=torch.zeros(D))


def off(t):
    """The same tensor 8 bytes past a 16-byte boundary."""
    flat = torch.zeros(t.numel() + 16, dtype=t.dtype)
    at = (16 - flat.data_ptr() % 16) % 16 // 2 + 4
    return flat[at:at + t.numel()].view(t.shape)


BWD = ["padoc_ancestor_prefill_bwd", "padoc_qk_rotary_bwd"]


def test_backward_of_a_layer_runs_both_steps(launched):
    for norm in (True, False):
        lay = layer(norm)
        launched.clear()
        lay.run_bwd(**tensors(lay.T))
        assert launched == BWD
    launched.clear()
    t = tensors(lay.T)
    del t["dq_weight"], t["dk_weight"]                   # not needed without a norm
    lay.run_bwd(**t)
    assert launched == BWD


@pytest.mark.parametrize("name, bad", [
    ("dq_weight", lambda t: None), ("dk_weight", lambda t: None), ("dq_weight", lambda t: t.to(BF16)),
    ("dk_weight", lambda t: t[:64]), ("q", lambda t: t[:-1]), ("q", lambda t: t[:, :2]), ("k", lambda t: t.float()),
    ("q", lambda t: None), ("q", off), ("k", off), ("dq", off), ("dk", off), ("dq", lambda t: t[:, :2].contiguous()),
    ("dq", lambda t: t.float()), ("dk", lambda t: t[:-1]), ("k", lambda t: torch.zeros((t.shape[0], HKV * D + 4), dtype=BF16)[:, :HKV * D].view(-1, HKV, D)),
])
def test_backward_of_a_layer_is_refused_before_it_writes(launched, name, bad):
    lay = layer()
    t = tensors(lay.T)
    t[name] = bad(t[name])
    launched.clear()
    with pytest.raises((ValueError, TypeError)):
        lay.run_bwd(**t)
    assert launched == []


def test_backward_of_a_layer_on_another_device_is_refused_before_it_writes(launched, monkeypatch):
    lay = layer()
    launched.clear()
    monkeypatch.setattr(pa, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="device"):
        lay.run_bwd(**tensors(lay.T))
    assert launched == []


SHORT = [(name, bad) for name in ("v", "out", "lse", "dout", "dv") for bad in ("rows", "heads", "dtype")]


@pytest.mark.parametrize("name, bad", SHORT)
def test_tensors_that_are_not_the_layers_are_refused(launched, name, bad):
    # (the attention calls take addresses: a tensor with fewer rows or heads would be read or written past its end)
    lay = layer()
    t = tensors(lay.T)
    t[name] = {"rows": lambda x: x[:-1], "heads": lambda x: x[:, :1].contiguous(),
               "dtype": lambda x: x.half()}[bad](t[name])
    launched.clear()
    with pytest.raises(ValueError):
        lay.run_bwd(**t)
    if name in ("v", "out", "lse"):
        with pytest.raises(ValueError):
            lay.run(**{n: t[n] for n in ("q", "k", "v", "scale", "out", "lse")})
    assert launched == []
    good = tensors(lay.T)
    lay.run(**{n: good[n] for n in ("q", "k", "v", "scale", "out", "lse")})
    assert launched == ["padoc_qk_rotary", "padoc_ancestor_prefill_attn"]


@pytest.mark.parametrize("name", ["q_dst", "out", "lse"])
def test_step_outputs_that_are_too_small_are_refused(launched, monkeypatch, name):
    monkeypatch.setattr(pa.load_library().__class__, "padoc_mpd_launch_step_rotary", lambda *a: launched.append("step") or 0,
                        raising=False)
    rot = pa.Rotary(np.ones(D // 2), head_dim=D, device="cpu")
    z = lambda h, n=5, dt=BF16: torch.zeros((n, h, D), dtype=dt)
    step, pos, ints = pa.padoc_mpd_step(), torch.zeros((5, 1), dtype=torch.int32), torch.zeros(64, dtype=torch.int32)
    step.num_streams = 4

    def call(**kw):
        t = dict(q_dst=z(HQ), out=z(HQ, 4), lse=torch.zeros((4, HQ)))
        t.update(kw)
        pa.padoc_mpd_launch_step_rotary(step, None, ints, pa.padoc_kv_pool(), rot, z(HKV), z(HKV), z(HQ), pos, t["q_dst"], 0.1,
                                        t["out"], t["lse"], ints)
    call()
    bad = [torch.zeros((3, HQ)), torch.zeros((4, HQ - 1)), torch.zeros((4, HQ)).half()] if name == "lse" else \
        [z(HQ, 3), z(HQ - 1), z(HQ, dt=torch.float32), torch.zeros((5, HQ, D // 2), dtype=BF16)]
    for b in bad:
        with pytest.raises(ValueError):
            call(**{name: b})
    assert launched == ["step"]
