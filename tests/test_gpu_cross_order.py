"""Cross attention behind the kernels before it in the stream, and in a capture: a plan that the kernel before writes, a
loop's step that is captured."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import CrossPlan, MaskedParallelLoop

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def inputs(segments, hq, hkv, d, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows, keys = max(s[0] + s[1] for s in segments), max(s[2] + s[3] for s in segments)
    new = lambda n, h: torch.randn((n, h, d), generator=g, device=DEV).to(dtype)   # noqa: E731
    return new(rows, hq), new(keys, hkv), new(keys, hkv), new(rows, hq)


@pytest.mark.parametrize("segments,hq,hkv,d,dtype", [
    ([(0, 24, 0, 9001)], 16, 2, 128, BF16),                  # lists of items, joined parts
    ([(0, 3, 0, 30_000)], 4, 4, 64, BF16),                   # few rows, joined parts
    ([(0, 40, 0, 700), (40, 5, 0, 0)], 4, 1, 64, F32),       # fp32, joined parts, rows without keys
    ([(0, 700, 0, 300), (700, 40, 300, 1000)], 16, 16, 64, BF16)])
def test_a_plan_that_the_kernel_before_writes(segments, hq, hkv, d, dtype):
    # the block copy lets the next kernel start before it has written anything, the plan's words last
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV, training=True)
    q, k, v, dout = inputs(segments, hq, hkv, d, dtype)
    want, wl = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    plan.run(q, k, v, 0.1, want, wl)
    plan.run_bwd(q, k, v, want, dout, wl, 0.1, *grads)
    block = 2 * 16 * 128                                     # words
    words, blocks = int(plan.info.plan_ints), 20_000
    own = -(-words // block)
    src, dst = (torch.zeros((blocks, 2, 16, 128), device=DEV) for _ in range(2))
    src.view(torch.int32).view(-1)[(blocks - own) * block:][:words] = plan.plan_dev[:words]
    there = dst.view(torch.int32).view(-1)[(blocks - own) * block:][:words]
    spare = [torch.zeros((blocks, 2, 16, 128), device=DEV) for _ in range(2)]
    to, of = pa.KvPools([(spare[0], dst)]), pa.KvPools([(spare[1], src)])
    order = torch.arange(blocks, dtype=torch.int32, device=DEV)
    for _ in range(3):
        out, lse = torch.full_like(q, 77.0), torch.full_like(wl, 77.0)
        got = [torch.full_like(t, 77.0) for t in grads]
        there.zero_()
        torch.cuda.synchronize()
        pa.padoc_copy_kv_blocks(to, order, order, of)
        pa.padoc_cross_attn(plan.info, there, q, k, v, 0.1, out, lse, plan.workspace)
        torch.cuda.synchronize()
        there.zero_()
        torch.cuda.synchronize()
        pa.padoc_copy_kv_blocks(to, order, order, of)
        pa.padoc_cross_attn_bwd(plan.info, there, q, k, v, out, dout, lse, 0.1, *got, plan.bwd_workspace)
        pa.padoc_check_device_errors()
        assert np.array_equal(there.cpu().numpy(), plan.plan_dev[:words].cpu().numpy())
        assert torch.equal(out, want) and torch.equal(lse, wl)
        assert all(torch.equal(a, b) for a, b in zip(got, grads))


def test_a_loops_captured_step_is_refused_and_a_plan_of_its_streams_captured():
    loop = MaskedParallelLoop(100, 16, 2, 128, BF16, DEV)
    q, k, v, _ = inputs([(0, 8, 0, 900)], 16, 2, 128, BF16)
    loop.add_page(4, 2, False, k, v, np.arange(4), states=(100, 700))
    ids, o, _ = loop.step(k, v, q, lambda i: i % 8, 0.1)
    loop.end_step(num_streams=len(ids))
    want, wl = loop.cross_step(ids, o, k, v, 0.1)
    plan = CrossPlan([(0, len(ids), 100, 700)], 16, 2, 128, BF16, DEV)
    out, lse = torch.zeros_like(want), torch.zeros_like(wl)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.run(o, k, v, 0.1, out, lse)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(ValueError, match="CrossPlan"):
            loop.cross_step(ids, o, k, v, 0.1, out, lse)
        plan.run(o, k, v, 0.1, out, lse)
    out.zero_()
    loop.set_states(int(ids[0]), 0, 5)
    loop.cross_step(ids, o, k, v, 0.1)            # another plan in the loop's memory
    graph.replay()
    torch.cuda.synchronize()
    pa.padoc_check_device_errors()
    assert torch.equal(out, want) and torch.equal(lse, wl)


@pytest.mark.parametrize("current", [False, True])
def test_a_plan_dropped_while_another_stream_runs_its_calls(current):
    segments, hq, hkv, d = [(0, 24, 0, 9001), (24, 300, 100, 500)], 16, 2, 128
    q, k, v, dout = inputs(segments, hq, hkv, d, BF16)
    plan = CrossPlan(segments, hq, hkv, d, BF16, DEV, training=True)
    want = [torch.empty_like(t) for t in (q, q, k, v)] + [torch.empty(q.shape[:2], device=DEV)]
    got = [torch.zeros_like(t) for t in want]
    plan.run(q, k, v, 0.1, want[0], want[4])
    plan.run_bwd(q, k, v, want[0], dout, want[4], 0.1, *want[1:4])
    sizes = [t.nbytes for t in (plan.plan_dev, plan.workspace, plan.bwd_workspace)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    del plan
    plan = CrossPlan(segments, hq, hkv, d, BF16, DEV, training=True)
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        stream = None if current else side
        plan.run(q, k, v, 0.1, got[0], got[4], stream=stream)
        plan.run_bwd(q, k, v, got[0], dout, got[4], 0.1, *got[1:4], stream=stream)
    del plan
    for _ in range(4):      # what is allocated now lies elsewhere
        for n in sizes:
            torch.empty(n, dtype=torch.uint8, device=DEV).fill_(255)
    torch.cuda.synchronize()
    pa.padoc_check_device_errors()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
