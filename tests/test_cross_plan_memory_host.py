"""CPU test of a CrossPlan's memory: it stays the plan's for every stream that a call of it went to."""
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import engine
from paper_2608_06146_gb300 import padoc_attn as pa


@pytest.mark.parametrize("training", [False, True])
def test_memory_is_kept_for_the_streams_of_the_calls(monkeypatch, training):
    # (a plan that is dropped while another stream than its own runs its call would leave that call to read whatever
    # is allocated there next)
    pbuild.build()
    pa.load_library()
    kept, calls, current = [], [], [7]
    monkeypatch.setattr(pa, "_stream_ptr", lambda s: current[0] if s is None else getattr(s, "cuda_stream", s))
    monkeypatch.setattr(pa, "padoc_cross_attn", lambda *a: calls.append(pa._stream_ptr(a[-1])))
    monkeypatch.setattr(pa, "padoc_cross_attn_bwd", lambda *a: calls.append(pa._stream_ptr(a[-1])))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw, device=None: raw)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: 0)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((t.data_ptr(), s)))
    plan = engine.CrossPlan([(0, 3, 0, 900)], 16, 2, 128, torch.bfloat16, "cpu", training=training)
    own = [t.data_ptr() for t in (plan.plan_dev, plan.workspace, plan.bwd_workspace) if t is not None]
    assert len(own) == 2 + training

    class Side:
        cuda_stream = 9
    used = []
    for stream in (None, 8, Side(), 0, None, 8, 1):
        plan.run(None, None, None, 0.1, None, None, stream)
        used.append(pa._stream_ptr(stream))
        if training:
            plan.run_bwd(None, None, None, None, None, None, 0.1, None, None, None, stream)
            used.append(used[-1])
    current[0] = 11                               # the current stream has changed
    plan.run(None, None, None, 0.1, None, None)
    assert calls == used + [11]
    assert {(p, s) for p in own for s in (7, 8, 9, 0, 11)} == set(kept)   # (1 is the default stream, too)
    assert len(kept) == len(own) * 6
