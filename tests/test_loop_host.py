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
            if name.startswith(("padoc_mpd_launch", "padoc_mpd_runner", "padoc_copy", "padoc_append")):
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
    monkeypatch.setattr(pa, "_stream_ptr", lambda stream: None)
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


def used(num_blocks=64):
    """A loop whose pool has free blocks below live ones, and whose branches have a row each; the copies it asks for."""
    loop, rows = make(num_blocks, prefix=40)
    pid, _ = loop.add_page(40, 3, False, rows[1], rows[2], np.zeros(40, np.int32))
    ids, _, _ = loop.step(rows[1], rows[2], rows[0], lambda i: np.zeros(len(i), np.int32), 0.1)
    loop.end_step(num_streams=len(ids))
    loop.drop_page(0)
    return loop, [int(i) for i in ids if int(i) > 2], rows


def pairs(loop, monkeypatch):
    """The (source, destination) lists of the copies from now on."""
    got = []
    monkeypatch.setattr(loop, "_copy_blocks", lambda src, dst, stream, pool=None: got.append((list(src), list(dst))))
    return got


def refusal(what, monkeypatch):
    """Something that makes a copy fail, until the context ends."""
    m = monkeypatch.context()
    p = m.__enter__()
    if what == "device":
        p.setattr(pa, "_current_device", lambda: 1)
    else:                       # no pinned memory for longer lists
        def none(t):
            raise MemoryError
        p.setattr(torch.Tensor, "pin_memory", none)
    return m


@pytest.mark.parametrize("what", ["device", "memory"])
@pytest.mark.parametrize("act", ["fork", "compact", "resize"])
def test_a_move_that_cannot_be_made_leaves_the_scheduler_as_it_was(cuda, monkeypatch, act, what):
    twin, live, _ = used()
    loop, same, _ = used()
    assert live == same
    branch = live[1]
    call = {"fork": lambda lp: lp.fork_stream(branch, 2), "compact": lambda lp: lp.compact(),
            "resize": lambda lp: lp.resize(30)}[act]
    before = loop.status()
    if what == "memory":
        loop._stage = [None, None]
    m = refusal(what, monkeypatch)
    with pytest.raises((ValueError, MemoryError)):
        call(loop)
    m.__exit__(None, None, None)
    assert loop.status() == before and loop.k_pool.shape[0] == 64
    want, got = pairs(twin, monkeypatch), pairs(loop, monkeypatch)
    a, b = call(twin), call(loop)
    assert np.array_equal(a, b) and got == want and len(want[0][0]) > 0


def test_a_page_whose_rows_cannot_be_sent_is_not_admitted(cuda, monkeypatch):
    loop, _, rows = used()
    before = loop.status()
    loop._stage = [None, None]
    m = refusal("memory", monkeypatch)
    with pytest.raises(MemoryError):
        loop.add_page(40, 1, False, rows[1], rows[2], np.zeros(40, np.int32))
    m.__exit__(None, None, None)
    assert loop.status() == before
    with pytest.raises((TypeError, ValueError)):
        loop.add_page(2, 1, False, rows[1], rows[2], [0, None])
    assert loop.status() == before
    with pytest.raises(pa.PadocError) as e:          # a page that does not fit
        loop.add_page(10 ** 6, 1, False, rows[1], rows[2], np.zeros(1, np.int32))
    assert e.value.status == 6 and loop.status() == before
    loop.add_page(40, 1, False, rows[1], rows[2], np.zeros(40, np.int32))
    loop.add_page(0, 1, False, rows[1], rows[2], None)
    assert loop.status()[0] == before[0] + 2


def test_moves_of_an_empty_pool(cuda):
    loop, _, _ = used()
    loop.drop_page(1)
    assert loop.compact() == 0
    loop.resize(0)
    assert loop.status() == (0, 0, 0) and loop.compact() == 0
    loop.resize(12)
    assert loop.status() == (0, 0, 12) and loop.k_pool.shape[0] == 12


def test_a_step_of_a_loop_without_streams_needs_no_positions(cuda, monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))   # (as if on the GPU)
    loop, _, rows = used()
    loop.drop_page(1)
    loop.rotary = pa.Rotary(np.ones(D // 2), head_dim=D, device="cpu")
    out, lse = torch.zeros((4, HQ, D), dtype=BF16), torch.zeros((4, HQ))
    assert loop.step(rows[1], rows[2], rows[0], lambda i: i, 0.1)[0].size == 0
    loop.end_step(num_streams=0)
    n, ids = loop.run_step(rows[1], rows[2], rows[0], np.zeros(8, np.int32), 0.1, out, lse)
    assert n == 0 and len(ids) == 0
    loop.add_page(0, 1, False, rows[1], rows[2], None)
    with pytest.raises(ValueError, match="pos"):
        loop.run_step(rows[1], rows[2], rows[0], np.zeros(8, np.int32), 0.1, out, lse)
