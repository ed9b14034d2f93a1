"""The decoding loop's cache moves on a stream of their own, while the stream that was current allocates: the block ids
that the copies read stay theirs."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import engine
from paper_2608_06146_gb300 import padoc_attn as pa

pytestmark = pytest.mark.gpu
HQ, HKV, D, BF16, DEV = 16, 2, 128, torch.bfloat16, "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def make(rotary=None):
    order = np.random.default_rng(3).permutation(3000)
    loop = engine.MaskedParallelLoop(3000, HQ, HKV, D, BF16, DEV, block_order=order, rotary=rotary)
    g = torch.Generator(DEV).manual_seed(9)
    q, k, v = (torch.randn(400, h, D, device=DEV, generator=g).to(BF16) for h in (HQ, HKV, HKV))
    for p in range(60):   # 25 blocks each, at uploads that fit the first array of ids
        loop.add_page(400, 1, False, k, v, np.random.default_rng(p).permutation(400))
    return loop, (q, k, v)


def test_moves_on_a_side_stream():
    want, src = make()
    live = want.compact()
    want.resize(1700)
    torch.cuda.synchronize()
    loop, _ = make()
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    side.wait_stream(main)
    words = loop._ints.numel()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)   # some 10 ms: the copies are still to come when the ids' array is replaced
    assert loop.compact(side) == live == 1500
    other = [torch.full((n,), 2999, dtype=torch.int32, device=DEV) for n in (words, 2 * words, 4 * words) for _ in range(4)]
    loop.resize(1700, side)
    other += [torch.full((n,), 2999, dtype=torch.int32, device=DEV) for n in (words, 2 * words, 4 * words) for _ in range(4)]
    assert loop._ints.numel() > words and other
    main.wait_stream(side)
    row = np.arange(128, dtype=np.int32)
    got = []
    for lp in (want, loop):
        ids, out, lse = lp.step(src[1], src[2], src[0], lambda i: row[i], 0.1)
        got.append((ids, out, lse))
    pa.padoc_check_device_errors()
    assert torch.equal(want.k_pool[:live], loop.k_pool[:live]) and torch.equal(want.v_pool[:live], loop.v_pool[:live])
    assert np.array_equal(got[0][0], got[1][0]) and len(got[0][0]) == 120
    assert torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][2], got[1][2])


def test_steps_on_a_side_stream_that_need_more_room():
    results = []
    for stream in (None, torch.cuda.Stream()):
        loop, src = make()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        row, kept = np.arange(128, dtype=np.int32), []
        for s in range(3):
            ids, out, lse = loop.step(src[1], src[2], src[0], lambda i: row[i] + s, 0.1, stream=stream)
            loop.end_step(num_streams=len(ids))
            kept.append((out, lse))
            torch.full((1 << 16,), 7, dtype=torch.int32, device=DEV)
        torch.cuda.synchronize()
        results.append(kept)
    pa.padoc_check_device_errors()
    for a, b in zip(*results):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_moves_refused_on_another_device_leave_the_loop_as_it_was(monkeypatch):
    results = []
    for refused in (False, True):
        loop, src = make()
        row = np.arange(512, dtype=np.int32) % 400
        step = lambda: loop.step(src[1], src[2], src[0], lambda i: row[i], 0.1)
        ids, _, _ = step()
        loop.end_step(num_streams=len(ids))
        loop.drop_page(3)
        branch = int(loop.step(src[1], src[2], src[0], lambda i: row[i], 0.1)[0][0])
        loop.end_step(num_streams=118)
        if refused:
            before = loop.status()
            with monkeypatch.context() as m:
                m.setattr(pa, "_current_device", lambda: 1)   # (as if another GPU were current)
                for call in (lambda: loop.fork_stream(branch, 2), loop.compact, lambda: loop.resize(2000)):
                    with pytest.raises(ValueError, match="device"):
                        call()
            assert loop.status() == before and loop.k_pool.shape[0] == 3000
        new = loop.fork_stream(branch, 2)
        loop.compact()
        loop.resize(1800)
        ids, out, lse = step()
        results.append((new, ids, out, lse))
    pa.padoc_check_device_errors()
    a, b = results
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1]) and len(a[1]) == 120
    assert torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])
