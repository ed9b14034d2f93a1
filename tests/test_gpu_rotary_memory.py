"""The rotary calls on the GPU when the same tensor objects are given other memory between calls: results are those of
the memory that the objects have at the call."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import MaskedParallelLoop

pytestmark = pytest.mark.gpu
DEV, BF16, HQ, HKV, D = "cuda:0", torch.bfloat16, 16, 2, 128
INV = 5e6 ** (-np.arange(D // 2) / (D // 2))


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def rand(seed, *shape, dtype=BF16):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


def rotary(w):
    return pa.Rotary(INV, head_dim=D, q_weight=w[0], k_weight=w[1], device=DEV)


def test_norm_weights_given_other_memory():
    n, pool_shape = 40, (8, HKV, 16, D)
    q, k, v = rand(1, n, HQ, D), rand(2, n, HKV, D), rand(3, n, HKV, D)
    dq_out, dk_out = rand(4, n, HQ, D), rand(5, n, HKV, D)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)[:, None].contiguous()
    slots = torch.arange(n, dtype=torch.int32, device=DEV)

    def results(rot):
        new = lambda h: torch.empty((n, h, D), dtype=BF16, device=DEV)
        qo, ko, dq, dk, qd, q8 = new(HQ), new(HKV), new(HQ), new(HKV), new(HQ), new(HQ)
        dqw, dkw = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
        ws = torch.empty(pa.padoc_qk_rotary_bwd_workspace_size(rot, n), dtype=torch.uint8, device=DEV)
        pool = [torch.zeros(pool_shape, dtype=BF16, device=DEV) for _ in range(2)]
        p8 = pa.E4M3Pool(8, HKV, D, DEV)
        pa.padoc_qk_rotary(rot, q, k, pos, qo, ko)
        pa.padoc_qk_rotary_bwd(rot, dq_out, dk_out, pos, dq, dk, q, k, dqw, dkw, ws)
        pa.padoc_append_rotary_inputs(rot, *pool, k, v, pos, slots, q, qd)
        pa.padoc_append_rotary_inputs_e4m3(rot, p8, k, v, pos, slots, q, q8)
        pa.padoc_check_device_errors()
        return [qo, ko, dq, dk, dqw, dkw, qd, q8, *pool, p8.k_codes, p8.k_scales]
    w = [torch.nn.Parameter(1 + 0.3 * rand(6 + i, D)) for i in range(2)]
    rot = rotary(w)
    first = results(rot)
    held = [p.data for p in w]
    for i, p in enumerate(w):
        p.data = 1 + 0.3 * rand(8 + i, D)
    got, want = results(rot), results(rotary([p.data.clone() for p in w]))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not torch.equal(got[0], first[0]) and not torch.equal(got[1], first[1]) and held


@pytest.mark.parametrize("mode", ["step", "runner"])
def test_a_loop_whose_norm_weights_are_given_other_memory(mode):
    q, k, v = rand(11, 4, HQ, D), rand(12, 4, HKV, D), rand(13, 4, HKV, D)
    pos = torch.arange(4, dtype=torch.int32, device=DEV)[:, None].contiguous()
    w = [torch.nn.Parameter(1 + 0.3 * rand(14 + i, D)) for i in range(2)]
    rot = rotary(w)
    lp = MaskedParallelLoop(8, HQ, HKV, D, BF16, DEV, rotary=rot)
    lp.add_page(0, 0, False, k, v, np.zeros(0, np.int32))
    out, lse = torch.empty((4, HQ, D), dtype=BF16, device=DEV), torch.empty((4, HQ), device=DEV)
    row, want, held = np.zeros(4, np.int32), [], []
    for i in range(3):
        row[:] = i
        if mode == "step":
            lp.step(k, v, q, lambda ids: row[ids], 0.1, pos_src=pos)
        else:
            lp.run_step(k, v, q, row, 0.1, out, lse, pos_src=pos)
        lp.end_step(num_streams=1)
        ko, qo = torch.empty_like(k), torch.empty_like(q)
        pa.padoc_qk_rotary(rotary([p.data.clone() for p in w]), q, k, pos, qo, ko)
        want.append(ko[i])
        held.append([p.data for p in w])
        for j, p in enumerate(w):
            p.data = 1 + 0.3 * rand(20 + 2 * i + j, D)
    pa.padoc_check_device_errors()
    assert torch.equal(lp.k_pool[0, :, :3].transpose(0, 1), torch.stack(want))
