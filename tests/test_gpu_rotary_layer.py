"""The training layer's refusals on the GPU: a refused call has written nothing."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import RotaryPrefill
from paper_2608_06146_gb300.inputs import PageSpec

pytestmark = pytest.mark.gpu
DEV, BF16, HQ, HKV, D = "cuda:0", torch.bfloat16, 16, 2, 128
PAGES = [PageSpec(60, 12, [0, 5, 12, 5], [17, 3, 30, 1])]


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def test_backward_without_the_weights_gradients_writes_nothing():
    w = [torch.ones(D, dtype=BF16, device=DEV) for _ in range(2)]
    layer = RotaryPrefill(PAGES, pa.Rotary(np.ones(D // 2), head_dim=D, q_weight=w[0], k_weight=w[1], device=DEV), HQ, HKV,
                          BF16, DEV, training=True)
    new = lambda h, x: torch.full((layer.T, h, D), x, dtype=BF16, device=DEV)
    q, k, v, out, dout = new(HQ, 0.5), new(HKV, 0.25), new(HKV, 1.0), new(HQ, 0.0), new(HQ, 1.0)
    lse = torch.zeros((layer.T, HQ), device=DEV)
    layer.run(q, k, v, 0.1, out, lse)
    dq, dk, dv = new(HQ, 7.0), new(HKV, 7.0), new(HKV, 7.0)
    for dw in (None, torch.zeros(D, dtype=BF16, device=DEV)):
        with pytest.raises(ValueError):
            layer.run_bwd(q, k, v, out, dout, lse, 0.1, dq, dk, dv, dw, dw)
    pa.padoc_check_device_errors()
    assert all(bool((t == 7.0).all()) for t in (dq, dk, dv))
    dqw, dkw = torch.zeros(D, device=DEV), torch.zeros(D, device=DEV)
    layer.run_bwd(q, k, v, out, dout, lse, 0.1, dq, dk, dv, dqw, dkw)
    pa.padoc_check_device_errors()
    assert not bool((dv == 7.0).any()) and torch.isfinite(dq).all() and torch.isfinite(dqw).all()
