"""CPU tests of the decoding loop's own memory and of what a refused call leaves behind. The loop is made over CPU
tensors; streams, events and launches are replaced by ones that note their use, the scheduler is the library's."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import engine
from paper_2608_06146_gb300 import padoc_attn as pa

HQ, HKV, D, BF16 = 16, 2, 128, torch.bfloat16


class Stream:
    cuda_stream = 0

    def __init__(self, name):
        self.name = name


class Event:
    def synchronize(self):
        pass

    def record(self, stream):
        pass


class Cuda:
    """What the loop does: the stream of each allocation, what is kept for which stream, the launches."""

    def __init__(self):
        self.current, self.made, self.kept, self.launches = Stream("main"), [], [], []
        self.side = Stream("side")


@pytest.fixture
def cuda(monkeypatch):
    pbuild.build()
    real, c = pa.load_library(), Cuda()
    empty = torch.empty

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.before, c.current = c.current, self.stream

        def __exit__(self, *e):
            c.current = self.before

    def noted(*a, **kw):
        t = empty(*a, **kw)
        if "device" in kw:
            c.made.append((t.data_ptr(), c.current.name))
        return t

    class Lib:
        def __getattr__(self, name):
            if name.startswith(("padoc_mpd_launch", "padoc_copy", "padoc_append")):
                return lambda *a: c.launches.append(name) or 0
            return getattr(real, name)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: c.current)
    monkeypatch.setattr(torch, "empty", noted)
    monkeypatch.setattr(torch.Tensor, "pin_memory", lambda t: t)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: c.kept.append((t.data_ptr(), s.name)))
    monkeypatch.setattr(pa, "_dev", lambda t, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(pa, "_current_device", lambda: -1)
    monkeypatch.setattr(pa, "load_library", lambda *a: Lib())
    return c


def make(num_blocks, prefix=20, forks=2):
    loop = engine.MaskedParallelLoop(num_blocks, HQ, HKV, D, BF16, "cpu")
    loop.mpd = pa.Mpd(num_blocks)
    rows = [torch.zeros((max(prefix, 1), h, D), dtype=BF16) for h in (HQ, HKV, HKV)]
    loop.add_page(prefix, forks, False, rows[1], rows[2], np.zeros(prefix, np.int32))
    return loop, rows


def where(c, t):
    return [s for p, s in c.made if p == t.data_ptr()][-1]


def test_room_that_an_upload_needs_is_made_on_its_stream(cuda):
    loop, _ = make(4000, prefix=1600)       # 100 blocks
    old = loop._ints
    loop._upload([np.arange(5000, dtype=np.int32)], cuda.side)
    assert loop._ints is not old and where(cuda, loop._ints) == "side"
    assert (old.data_ptr(), "side") in cuda.kept
    np.testing.assert_array_equal(loop._ints[:5000].numpy(), np.arange(5000))


def test_room_that_a_step_needs_is_made_on_its_stream(cuda):
    loop, rows = make(4000, prefix=1600, forks=100)
    old = loop._ints, loop.q_step, loop.workspace
    ids, out, lse = loop.step(rows[1], rows[2], rows[0], lambda i: np.zeros(len(i), np.int32), 0.1, stream=cuda.side)
    assert len(ids) == 101 and "padoc_mpd_launch_step" in cuda.launches
    new = loop._ints, loop.q_step, loop.workspace
    assert all(a is not b for a, b in zip(old, new))
    assert all(where(cuda, t) == "side" for t in new + (out, lse))
    assert all((t.data_ptr(), "side") in cuda.kept for t in old)
    assert new[1].shape[0] >= 101 and new[1].shape[1:] == (HQ, D)
    cuda.kept.clear()
    loop.end_step(num_streams=len(ids))
    loop.step(rows[1], rows[2], rows[0], lambda i: np.zeros(len(i), np.int32), 0.1, out, lse, stream=cuda.side)
    assert not cuda.kept and loop._ints is new[0] and loop.q_step is new[1] and loop.workspace is new[2]
