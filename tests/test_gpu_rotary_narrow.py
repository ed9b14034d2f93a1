"""The append of bf16 heads whose dims, or rotated dims, are an odd multiple of 8: their vectors are of 8 bytes.

Tolerance: 3e-6 (|u| + |v|) for a pair (a sine and a cosine 0.9e-6 off; the norm's scale: half of 1.25e-6 for a sum of 256
squares, two units of the last place for the root, and the roundings, on both members), and one rounding to bf16."""
import numpy as np
import pytest
import torch

from oracle import rotary as orot
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa

pytestmark = pytest.mark.gpu
DEV, BF16, BS = "cuda:0", torch.bfloat16, 16


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


# (rows, hq, hkv, d, rot, adjacent, norm): bf16 heads or rotated parts in odd multiples of 8
NARROW = [(1, 16, 2, 72, 72, False, True), (77, 3, 1, 72, 24, True, True), (640, 16, 2, 72, 72, False, False),
          (61, 4, 2, 128, 40, False, True), (33, 5, 5, 64, 24, True, False), (9, 4, 1, 256, 248, False, True),
          (17, 1, 1, 8, 8, False, True), (2100, 7, 1, 72, 56, True, True), (300, 2, 2, 136, 136, False, True)]


@pytest.mark.parametrize("rows,hq,hkv,d,rot,adjacent,norm", NARROW)
def test_append_of_heads_in_8_byte_vectors(rows, hq, hkv, d, rot, adjacent, norm):
    rng = np.random.default_rng(rows + d)
    g = torch.Generator(DEV).manual_seed(rows)
    w = [(1 + 0.3 * torch.randn(d, device=DEV, generator=g)).to(BF16) for _ in range(2)] if norm else (None, None)
    inv = 5e6 ** (-np.arange(rot // 2) / (rot // 2))
    axis = rng.integers(0, 3, rot // 2)
    spec = pa.Rotary(inv, axis, 3, d, adjacent=adjacent, q_weight=w[0], k_weight=w[1], device=DEV)
    pos = torch.from_numpy(rng.integers(-50, 3000, (rows, 3)).astype(np.int32)).to(DEV)
    x = torch.randn(rows, hq + 2 * hkv, d, device=DEV, generator=g).to(BF16)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    n, nb = max(1, rows - 3), rows // BS + 5
    src = torch.from_numpy(rng.permutation(rows)[:n].astype(np.int32)).to(DEV)
    slots = torch.from_numpy(rng.permutation(nb * BS)[:n].astype(np.int32)).to(DEV)
    pools = [torch.full((nb, hkv, BS, d), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
    qd = torch.full((n + 2, hq, d), 5.0, dtype=BF16, device=DEV)
    pa.padoc_append_rotary_inputs(spec, *pools, k, v, pos, slots, q, qd, src)
    pa.padoc_check_device_errors()
    at, block, row = src.long(), slots.long() // BS, slots.long() % BS
    angle = orot.angles(pos[at].cpu().numpy(), inv, axis)
    w64 = [None if t is None else f64(t) for t in w]
    check(qd[:n], *orot.forward(f64(q[at]), w64[0], 1e-6, angle, adjacent), 3e-6)
    check(pools[0][block, :, row], *orot.forward(f64(k[at]), w64[1], 1e-6, angle, adjacent), 3e-6)
    assert torch.equal(pools[1][block, :, row], v[at]) and bool((qd[n:] == 5.0).all())
    # rows of no slot are as they were, and the packed call gives the same bits
    rest = torch.ones((nb, BS), dtype=torch.bool, device=DEV)
    rest[block, row] = False
    for p in pools:
        assert bool((p.transpose(1, 2)[rest] == 3.0).all())
    qo, ko = (torch.empty((rows, h, d), dtype=BF16, device=DEV) for h in (hq, hkv))
    pa.padoc_qk_rotary(spec, q, k, pos, qo, ko)
    assert torch.equal(qd[:n], qo[at]) and torch.equal(pools[0][block, :, row], ko[at])
    # without queries and without a row list
    for p in pools:
        p.fill_(3.0)
    pa.padoc_append_rotary_inputs(spec, *pools, k, v, pos, slots, count=n)
    pa.padoc_check_device_errors()
    assert torch.equal(pools[0][block, :, row], ko[:n]) and torch.equal(pools[1][block, :, row], v[:n])
    for p in pools:
        assert bool((p.transpose(1, 2)[rest] == 3.0).all())
