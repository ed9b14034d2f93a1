"""CPU tests of the decoding loop's cross attention: what a call copies and what it leaves of the step's own counts. The
loop runs over CPU tensors with the streams, events and launches of test_loop_host; the cross attention call is noted."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import padoc_attn as pa

from .test_loop_host import BF16, D, HKV, HQ, cuda, make   # noqa: F401 (cuda: a fixture)


@pytest.fixture
def calls(cuda, monkeypatch):                              # noqa: F811
    noted = []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(pa, "padoc_cross_attn", lambda info, plan, *a: noted.append((int(info.plan_ints), plan.data_ptr())))
    return noted


def _step(loop):
    rows = [torch.zeros((64, h, D), dtype=BF16) for h in (HKV, HKV, HQ)]
    ids, _, _ = loop.step(*rows, lambda i: i % 64, 0.1, torch.zeros((64, HQ, D), dtype=BF16), torch.zeros((64, HQ)))
    return ids


def _cross(loop, ids):
    q, k = torch.zeros((len(ids), HQ, D), dtype=BF16), torch.zeros((1000, HKV, D), dtype=BF16)
    return loop.cross_step(ids, q, k, k, 0.1)


def test_the_steps_bytes_are_not_those_of_the_plan(calls):
    loop = make(200)[0]
    for i in range(3):
        loop.set_states(i, 100 * i, 90)
    ids = _step(loop)
    step = loop.h2d_bytes
    assert step > 0
    _cross(loop, ids)
    (words, _), = calls
    assert loop.h2d_bytes == step and loop.cross_h2d_bytes == 4 * (-(-words // 32) * 32)
    _cross(loop, ids)                                      # the plan is kept
    assert loop.h2d_bytes == step and loop.cross_h2d_bytes == 0
    loop.end_step(np.zeros(len(ids), np.int32), np.zeros(len(ids), np.uint8))
    loop.set_states(0, 5, 6)
    ids = _step(loop)
    step = loop.h2d_bytes
    _cross(loop, ids)
    assert loop.h2d_bytes == step and loop.cross_h2d_bytes == 4 * (-(-calls[-1][0] // 32) * 32)


def test_a_captured_call_is_refused(calls, cuda, monkeypatch):   # noqa: F811
    # a replay would run the captured grid over whatever plan the loop's later calls have left in its place
    loop = make(200)[0]
    loop.set_states(0, 0, 90)
    ids = _step(loop)
    _cross(loop, ids)
    kept = loop._cross_plan
    for asked in (cuda.current, cuda.side):
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "is_current_stream_capturing", lambda: cuda.current is asked)
            with pytest.raises(ValueError, match="CrossPlan"):
                loop.cross_step(ids, torch.zeros((len(ids), HQ, D), dtype=BF16), *[torch.zeros((1000, HKV, D), dtype=BF16)] * 2, 0.1,
                                stream=asked)
    assert len(calls) == 1 and loop._cross_plan is kept
    _cross(loop, ids)
    assert len(calls) == 2


def _layouts(cuda):                                        # noqa: F811
    """A loop of three pages with a layout stream each, over states of their own."""
    loop, rows = make(200, forks=0)
    loop.set_states(0, 10, 20)
    for i in (1, 2):
        loop.add_page(20, 0, False, rows[1], rows[2], np.zeros(20, np.int32), states=(100 * i, 30 + i))
    return loop


def test_branches_of_every_layout_stream_at_once(calls, cuda):   # noqa: F811
    # one number of forks for all streams, as the scheduler takes it
    loop = _layouts(cuda)
    ids = _step(loop)
    new = loop.end_step(2, num_streams=len(ids))
    assert [loop.states_of(i) for i in new] == [loop.states_of(p) for p in ids for _ in range(2)]
    assert loop.states_of(new[-1]) == (200, 32)


@pytest.mark.parametrize("status", [2, 4])
def test_branches_of_a_step_that_could_not_be_launched(calls, cuda, status):   # noqa: F811
    # past the planning such a step has begun and is the caller's to end: its branches see what its streams see
    loop = _layouts(cuda)
    ids = _step(loop)
    loop.end_step(num_streams=len(ids))
    loop.drop_page(0)

    class Runner:
        _ids = np.zeros(64, np.int32)

        def step(self, *a):
            begun, _ = loop.mpd.begin_step()
            self._ids[:len(begun)] = begun
            raise pa.PadocError("padoc_mpd_runner_step", status)
    loop._runner = Runner()
    with pytest.raises(pa.PadocError):
        loop.run_step(None, None, None, None, 0.1, None, None)
    new = loop.end_step([1, 2])
    assert [loop.states_of(i) for i in new] == [(100, 31), (200, 32), (200, 32)]


def test_a_refused_step_leaves_the_begun_ones_order(calls, cuda):   # noqa: F811
    loop = _layouts(cuda)
    ids = _step(loop)

    class Runner:
        _ids = np.full(64, 2, np.int32)

        def step(self, *a):
            raise pa.PadocError("padoc_mpd_runner_step", 1)   # a step is begun already
    loop._runner = Runner()
    with pytest.raises(pa.PadocError):
        loop.run_step(None, None, None, None, 0.1, None, None)
    new = loop.end_step([0, 1, 0])
    assert [loop.states_of(i) for i in new] == [loop.states_of(ids[1])]
