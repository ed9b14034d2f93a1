"""The rotary kernels' angles at half a turn.

Tolerance: a sine and a cosine 0.9e-6 off at most, so u c - v s is off by 1.1e-6 (|u| + |v|) with its roundings, and by
one rounding to the stored type."""
import numpy as np
import pytest
import torch

from oracle import rotary as orot
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def f64(t):
    return t.detach().cpu().double().numpy()


def check(got, want, size, rel):
    eps = torch.finfo(got.dtype).eps / 2
    tol = eps * np.abs(want) + (1 + eps) * rel * size + 1e-37
    bad = ~(np.abs(f64(got) - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off"


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_angles_at_half_a_turn(dtype, adjacent):
    # table entries whose product with position 1 has the upper word t at and around INT32_MAX and INT32_MIN (from
    # INT32_MAX - 63 on t rounds up to 2^31, half a turn), at the quarter turns and around zero
    top = [2 ** 31 - 1 - j for j in (0, 1, 31, 32, 33, 62, 63, 64, 65, 127, 128, 255)]
    t = top + [-2 ** 31 + j for j in (0, 1, 63, 64, 65, 128)] + [2 ** 30 + j for j in (-1, 0, 1)] + \
        [-2 ** 30 + j for j in (-1, 0, 1)] + [0, 1, -1] + [2 ** 29, -2 ** 29, 2 ** 31 - 2 ** 10, 12345, -98765]
    entry = np.array([(x << 32 | 0xFFFFFFFC) if i % 2 else x << 32 for i, x in enumerate(t)], np.int64)   # (the axis: 0)
    n, hq, hkv = len(t), 3, 1
    assert n == 32
    d = 2 * n
    rot = pa.Rotary(np.zeros(n), head_dim=d, adjacent=adjacent, device=DEV)
    rot.table.copy_(torch.from_numpy(entry))
    pos = torch.tensor([[1], [-1], [0], [1]], dtype=torch.int32, device=DEV)
    g = torch.Generator(DEV).manual_seed(3)
    q, k = (torch.randn(4, h, d, device=DEV, generator=g).to(dtype) for h in (hq, hkv))
    q[3, 0] = 1.0                                          # (u cos t - v sin t of equal members: cancels near 1/8 turn)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    pa.padoc_qk_rotary(rot, q, k, pos, qo, ko)
    pa.padoc_check_device_errors()
    # the product's fraction of a turn, exact to 2^-53
    turns = entry.astype(np.float64) * 2.0 ** -64
    angle = f64(pos) * turns[None] * (2 * np.pi)
    for got, x in ((qo, q), (ko, k)):
        check(got, *orot.forward(f64(x), None, 0.0, angle, adjacent), 1.1e-6)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    pa.padoc_qk_rotary_bwd(rot, q, k, pos, dq, dk)
    for got, x in ((dq, q), (dk, k)):
        check(got, *orot.turn_back(f64(x), angle, adjacent), 1.1e-6)
