"""CPU tests of the addresses that the rotary calls hand to the library: those of the tensors as they are at the call,
although the same objects may have been given other memory since. The library is replaced by one that notes what it
gets; tensors are on the CPU."""
import ctypes
import struct
import types

import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa

BF16, F32 = torch.bfloat16, torch.float32
D = 64


class Noted:
    """A library whose calls succeed; `seen` holds what the last one got."""

    def __init__(self):
        self.seen = {}

    def __getattr__(self, name):
        return lambda *args: self._call(name, args)

    def _call(self, name, args):
        for a in args:
            c = getattr(a, "_obj", a)
            if isinstance(c, pa.padoc_rotary):
                self.seen.update(qw=c.q_weight, kw=c.k_weight)
            if isinstance(c, pa.padoc_mpd_run_args):
                self.seen.update(k=c.k_src, v=c.v_src, q=c.q_src, out=c.out, lse=c.lse, rows=c.src_total)
        if name == "padoc_mpd_runner_set_rotary":
            self.seen["pos"] = args[2]
        return 0


@pytest.fixture
def lib(monkeypatch):
    pbuild.build()
    real, noted = pa.load_library(), Noted()
    noted.padoc_build_rotary_table = real.padoc_build_rotary_table
    monkeypatch.setattr(pa, "load_library", lambda *a: noted)
    monkeypatch.setattr(pa, "_dev", lambda t, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(pa, "_current_device", lambda: -1)
    monkeypatch.setattr(pa, "_stream_ptr", lambda stream: None)
    return noted


def spec(dtype=BF16, norm=True):
    w = [torch.nn.Parameter(torch.ones(D, dtype=dtype)) for _ in range(2)] if norm else (None, None)
    return pa.Rotary(np.ones(D // 2), head_dim=D, q_weight=w[0], k_weight=w[1], device="cpu")


def calls(rot, dt=BF16):
    """Every call that takes a spec, with rows of a dtype."""
    z = lambda h, n=4: torch.zeros((n, h, D), dtype=dt)
    q, k, pos, ints = z(2), z(1), torch.zeros((4, 1), dtype=torch.int32), torch.arange(4, dtype=torch.int32)
    pool, w = torch.zeros((2, 1, 16, D), dtype=dt), torch.zeros(D)
    e4m3 = types.SimpleNamespace(k_codes=pool, c=pa.padoc_kv_pool_e4m3())
    step = pa.padoc_mpd_step()
    return [lambda: pa.padoc_qk_rotary(rot, q, k, pos, z(2), z(1)),
            lambda: pa.padoc_qk_rotary_bwd_workspace_size(rot, 4),
            lambda: pa.padoc_qk_rotary_bwd(rot, z(2), z(1), pos, z(2), z(1), q, k, w, w.clone(), torch.zeros(256, dtype=torch.uint8)),
            lambda: pa.padoc_append_rotary_inputs(rot, pool, pool.clone(), k, k, pos, ints),
            lambda: pa.padoc_append_rotary_inputs_e4m3(rot, e4m3, k, k, pos, ints),
            lambda: pa.padoc_mpd_launch_step_rotary(step, None, ints, pa.padoc_kv_pool(), rot, k, k, q, pos, z(2), 1.0, z(2),
                                                    w, ints)]


@pytest.mark.parametrize("i", range(6))
def test_norm_weights_that_were_given_other_memory(lib, i):
    rot = spec()
    call = calls(rot)[i]
    call()
    assert lib.seen["qw"] == rot.q_weight.data_ptr() and lib.seen["kw"] == rot.k_weight.data_ptr()
    held = rot.q_weight.data, rot.k_weight.data   # (the old memory is not given out again)
    rot.k_weight.data = torch.ones(D, dtype=BF16)
    call()
    assert lib.seen["kw"] == rot.k_weight.data_ptr() != held[1].data_ptr() and lib.seen["qw"] == held[0].data_ptr()
    with torch.no_grad():
        rot.q_weight.set_(torch.ones(D, dtype=BF16))
    call()
    assert lib.seen["qw"] == rot.q_weight.data_ptr() != held[0].data_ptr()
    rot.q_weight = torch.ones(D, dtype=BF16)      # another object in its place
    call()
    assert lib.seen["qw"] == rot.q_weight.data_ptr()


def test_norm_weights_of_another_dtype_or_shape(lib):
    rot = spec(F32)
    for w in (rot.q_weight, rot.k_weight):
        w.data = w.data.to(BF16)                  # as module.to(bfloat16) does
    calls(rot)[0]()                               # rows of bf16
    assert rot.dtype is BF16 and lib.seen["qw"] == rot.q_weight.data_ptr()
    rot.q_weight.data = rot.q_weight.data.float()
    with pytest.raises(ValueError):               # of two dtypes
        calls(rot)[0]()
    for bad in (torch.ones(D // 2, dtype=BF16), torch.ones(2 * D, dtype=BF16)[::2], torch.ones(D, dtype=torch.float16)):
        rot = spec()
        call = calls(rot)[0]
        rot.q_weight.data = bad
        with pytest.raises((ValueError, TypeError)):
            call()
    rot = spec()
    rot.k_weight.data = rot.k_weight.data[:D // 2]       # the same address
    with pytest.raises(ValueError):
        calls(rot)[0]()


def test_spec_without_weights_stays_without(lib):
    rot = spec(norm=False)
    for call in calls(rot)[:2]:
        call()
    assert lib.seen["qw"] is None and lib.seen["kw"] is None


def runner():
    cfg = pa.padoc_decode_config()
    cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim = 2, 1, D
    pool = pa.padoc_kv_pool()
    pool.dtype = pa.PADOC_DTYPE_BF16
    return pa.MpdRunner(types.SimpleNamespace(_h=None), cfg, pool)


def test_runner_reads_weights_and_positions_at_every_step(lib):
    r, rot = runner(), spec()
    src = [torch.zeros((4, h, D), dtype=BF16) for h in (1, 1, 2)]
    row, pos = np.zeros(4, np.int32), torch.zeros((4, 1), dtype=torch.int32)
    o = types.SimpleNamespace(shape=(4, 2, D), dtype=BF16, is_cuda=True, is_contiguous=lambda: True, data_ptr=lambda: 64, detach=lambda: None)
    l = types.SimpleNamespace(shape=(4, 2), dtype=F32, is_cuda=True, is_contiguous=lambda: True, data_ptr=lambda: 128, detach=lambda: None)
    step = lambda: r.step(*src, row, 1.0, o, l)
    r.set_rotary(rot, pos)
    step()
    held = rot.q_weight.data, pos.data
    rot.q_weight.data = torch.ones(D, dtype=BF16)
    step()
    assert lib.seen["qw"] == rot.q_weight.data_ptr() != held[0].data_ptr()
    pos.set_(torch.zeros((4, 1), dtype=torch.int32))
    step()
    assert lib.seen["pos"] == pos.data_ptr()
    rot.k_weight.data = rot.k_weight.data.float()
    with pytest.raises(ValueError):
        step()
    assert r.rotates(rot, pos) and not r.rotates(rot, pos.clone())
    rot.k_weight.data = rot.k_weight.data.to(BF16)
    step()
    r.set_rotary(None)
    step()
    assert not r.rotates(rot, pos)


def test_runner_reads_sources_and_outputs_where_they_are(lib, monkeypatch):
    r = runner()
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))   # (as if on the GPU)
    new = lambda h, n=4: torch.zeros((n, h, D), dtype=BF16)
    k, v, q, row = new(1), new(1), new(2), np.zeros(4, np.int32)
    out, lse = new(2), torch.zeros((4, 2))
    step = lambda: r.step(k, v, q, row, 1.0, out, lse)
    step()
    held = [t.clone().set_(t) for t in (k, v, q, out, lse)]   # (their memory is not given out again)
    for name, t, h in (("k", k, 1), ("v", v, 1), ("q", q, 2), ("out", out, 2)):
        before = t.data_ptr()
        t.set_(new(h))
        step()
        assert lib.seen[name] == t.data_ptr() != before
    lse.set_(torch.zeros((4, 2)))
    step()
    assert lib.seen["lse"] == lse.data_ptr() != held[4].data_ptr()
    for t, h in ((k, 1), (v, 1), (q, 2)):
        t.set_(new(h, 3))                                     # fewer rows
    step()
    assert lib.seen["rows"] == 3
    for t, bad in ((k, new(2)), (q, new(2).float()), (out, new(3)), (lse, torch.zeros((4, 3)))):
        good = t.clone().set_(t)
        t.data = bad
        for _ in range(2):
            with pytest.raises((ValueError, TypeError)):
                step()
        t.data = good
        step()
    # memory that the runner has seen is not given out again while it may take it for the same tensor's
    seen = k.data_ptr()
    k.data = new(1, 3)
    assert all(new(1, n).data_ptr() != seen for n in range(1, 4) for _ in range(8))
    step()
    assert lib.seen["k"] == k.data_ptr()


def test_runner_with_rotary_on_another_device_is_refused(lib, monkeypatch):
    r, rot = runner(), spec()
    row, pos = np.zeros(4, np.int32), torch.zeros((4, 1), dtype=torch.int32)
    k, v, q = (torch.zeros((4, h, D), dtype=BF16) for h in (1, 1, 2))
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))   # (as if on the GPU)
    out, lse = torch.zeros((4, 2, D), dtype=BF16), torch.zeros((4, 2))
    r.set_rotary(rot, pos)
    r.step(k, v, q, row, 1.0, out, lse)
    lib.seen.clear()
    monkeypatch.setattr(pa, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="device"):
        r.step(k, v, q, row, 1.0, out, lse)
    with pytest.raises(ValueError, match="device"):
        r.set_rotary(rot, pos)
    assert not lib.seen


def test_loop_over_a_pool_on_another_device_than_its_rotary(lib, monkeypatch):
    from paper_2608_06146_gb300 import engine
    rot = spec(norm=False)
    monkeypatch.setattr(torch.cuda, "Event", lambda: None)
    with pytest.raises(ValueError, match="device"):
        engine.MaskedParallelLoop(2, 2, 1, D, BF16, "meta", rotary=rot)
    engine.MaskedParallelLoop(2, 2, 1, D, BF16, "cpu", rotary=rot)
