"""GPU parity of the head norms and rotary positions: the packed forward and backward, the append into the
paged pool and into the FP8 pool, against the 64-bit definition (oracle/rotary.py).

Tolerances, derived (worst cases, relative, in units of 1e-6; 2^-24 = 0.06). The angle's fraction of a turn is cut
at 2^-32 and rounded to 24 bits: 0.2 rad; the hardware's sine and cosine are 2^-20.5 = 0.67 off at most: in all 0.9 on
each of c and s, and u c - v s is 1.1 (|u| + |v|) off with its roundings. The norm's scale: a sum of 256 squares in at
most 21 additions (1.25, halved by the root), the root's 2 units of the last place and the roundings: 0.95, on both u
and v. So FWD = 3 x amplitude x (|u| + |v|), and one rounding to the stored type, eps / 2 of the value. Backward: g has
1.1; r g x w 2.4; the mean of w g h: 1.25 for its sum, 1.3 for its terms' w g, 0.95 for r; times r r x: 5.9. BWD = 6 x
the sum of the magnitudes that the formula adds. The weights' gradient sums (rows x heads) products r g x, each 2.2
off, in chains of fewer than 500 fp32 additions: DW = 2.2 + 512 x 0.06 of the sum of the magnitudes.
"""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import rotary as orot
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import ChunkPrefillPlan, DecodePlan, MaskedParallelLoop, RotaryPrefill
from paper_2608_06146_gb300.inputs import LoopTokenSource, PageSpec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BS = 16
FWD, BWD, DW = 3e-6, 6e-6, 2.2e-6 + 512 * 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def up(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def f64(t):
    return t.detach().cpu().double().numpy()


class Spec:
    """A rotary spec on both sides."""

    def __init__(self, seed, d, rot, axes, adjacent, norm, dtype, amplitude=1.0, eps=1e-6, base=5e6):
        g = np.random.default_rng(seed)
        n = rot // 2
        self.inv = base ** (-np.arange(n) / n)
        self.axis = g.integers(0, axes, n)
        self.adjacent, self.amplitude, self.eps, self.d, self.axes = adjacent, amplitude, eps, d, axes
        self.qw = self.kw = None
        if norm:
            self.qw, self.kw = (up(1 + 0.3 * g.standard_normal(d)).to(dtype) for _ in range(2))
        self.dev = pa.Rotary(self.inv, self.axis, axes, d, adjacent=adjacent, q_weight=self.qw, k_weight=self.kw, eps=eps,
                             amplitude=amplitude, device=DEV)

    def w64(self, w):
        return None if w is None else f64(w)

    def angle(self, pos):
        return orot.angles(pos.cpu().numpy(), self.inv, self.axis)

    def forward(self, x, w, pos):
        return orot.forward(f64(x), self.w64(w), self.eps, self.angle(pos), self.adjacent, self.amplitude)

    def backward(self, dz, x, w, pos):
        return orot.backward(f64(dz), None if x is None else f64(x), self.w64(w), self.eps, self.angle(pos), self.adjacent,
                             self.amplitude)


def check(got, want, size, rel, name):
    """|got - want| within the stored type's rounding and rel x size."""
    got_, eps = f64(got), torch.finfo(got.dtype).eps / 2
    tol = eps * np.abs(want) + (1 + eps) * rel * size + 1e-37
    bad = ~(np.abs(got_ - want) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got_ - want) / tol):.2f} x the bound"


def positions(rng, rows, axes, far=0):
    return up((far + rng.integers(-50, 3000, (rows, axes))).astype(np.int32))


def qkv(rng, rows, hq, hkv, d, dtype, scale=1.0):
    x = up(scale * rng.standard_normal((rows, hq + 2 * hkv, d))).to(dtype)
    return x, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


# (dtype, rows, hq, hkv, d, rot, axes, adjacent, norm, far)
SHAPES = [
    (BF16, 1, 16, 2, 128, 128, 3, False, True, 0),
    (BF16, 77, 16, 2, 128, 128, 3, False, True, 10 ** 6),
    (BF16, 500, 16, 2, 128, 128, 1, True, False, 0),
    (BF16, 33, 7, 1, 128, 64, 2, False, True, 0),
    (BF16, 19, 5, 3, 64, 64, 2, True, True, 0),
    (BF16, 40, 6, 6, 80, 32, 3, False, True, 0),
    (BF16, 21, 3, 1, 72, 72, 2, False, True, 0),
    (BF16, 21, 3, 1, 72, 24, 2, True, True, 0),
    (BF16, 9, 4, 1, 256, 256, 4, False, True, 0),
    (BF16, 9, 4, 1, 256, 248, 4, False, False, 0),
    (BF16, 5, 1, 1, 8, 8, 1, False, True, 0),
    (BF16, 1000, 33, 1, 96, 96, 1, False, False, 0),
    (F32, 1, 4, 1, 64, 64, 1, False, False, 0),
    (F32, 368, 4, 1, 64, 64, 3, False, True, 10 ** 6),
    (F32, 50, 16, 2, 128, 128, 3, True, True, 0),
    (F32, 23, 2, 2, 256, 128, 2, False, True, 0),
    (F32, 23, 3, 1, 40, 24, 2, True, False, 0),
    (F32, 2500, 1, 1, 8, 8, 1, False, True, 0),
    (BF16, 10001, 16, 2, 128, 128, 3, False, True, 0),
    (BF16, 9990, 7, 1, 128, 64, 2, True, True, 0),
    (F32, 70001, 1, 1, 64, 64, 2, False, True, 0),
]
ids = lambda s: f"{'bf16' if s[0] is BF16 else 'f32'}-{s[1]}x{s[2]}+{s[3]}x{s[4]}-r{s[5]}-a{s[6]}{'-adj' if s[7] else ''}{'-norm' if s[8] else ''}"


@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_forward_and_backward(shape):
    dtype, rows, hq, hkv, d, rot, axes, adjacent, norm, far = shape
    rng = np.random.default_rng(rows + d)
    sp = Spec(rows, d, rot, axes, adjacent, norm, dtype, amplitude=1.0 if rows % 2 else 1.2)
    pos = positions(rng, rows, axes, far)
    _, q, k, _ = qkv(rng, rows, hq, hkv, d, dtype)
    new = lambda h: torch.full((rows, h, d), float("nan"), dtype=dtype, device=DEV)
    qo, ko = new(hq), new(hkv)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko)
    pa.padoc_check_device_errors()
    for got, x, w, name in ((qo, q, sp.qw, "q"), (ko, k, sp.kw, "k")):
        check(got, *sp.forward(x, w, pos), FWD, name)
    # backward: the upstream gradients in a buffer of their own, the results in slices of one
    _, dqo, dko, _ = qkv(rng, rows, hq, hkv, d, dtype)
    dqkv = torch.full((rows, hq + 2 * hkv, d), 7.0, dtype=dtype, device=DEV)
    dq, dk = dqkv[:, :hq], dqkv[:, hq:hq + hkv]
    dqw, dkw = (torch.full((d,), float("nan"), device=DEV) for _ in range(2))
    ws = torch.empty(max(pa.padoc_qk_rotary_bwd_workspace_size(sp.dev, rows), 256), dtype=torch.uint8, device=DEV)
    args = (q, k, dqw, dkw, ws) if norm else ()
    pa.padoc_qk_rotary_bwd(sp.dev, dqo, dko, pos, dq, dk, *args)
    pa.padoc_check_device_errors()
    for got, dz, x, w, gw, name in ((dq, dqo, q, sp.qw, dqw, "dq"), (dk, dko, k, sp.kw, dkw, "dk")):
        dx, size, dw, terms = sp.backward(dz, x, w, pos)
        check(got, dx, size, BWD if norm else FWD, name)
        if norm:
            check(gw, dw, terms, DW, name + "_weight")
    assert bool((dqkv[:, hq + hkv:] == 7).all()), "the rows' other heads are left as they were"
    # a second call gives the same bits, also in place
    first = (dq.clone(), dk.clone(), dqw.clone(), dkw.clone())
    dq2, dk2 = dqo.contiguous(), dko.contiguous()
    pa.padoc_qk_rotary_bwd(sp.dev, dq2, dk2, pos, dq2, dk2, *args)
    assert torch.equal(dq2, first[0]) and torch.equal(dk2, first[1])
    if norm:
        assert torch.equal(dqw, first[2]) and torch.equal(dkw, first[3])
    q2, k2 = q.clone().contiguous(), k.clone().contiguous()
    pa.padoc_qk_rotary(sp.dev, q2, k2, pos, q2, k2)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    pa.padoc_check_device_errors()


def test_gradients_against_differences_of_the_forward():
    # fp32 forward: differences with step 2^-6 of values of size 1: truncation 2^-12 x a third derivative of
    # the norm (a few units), rounding 2^-24 x sum of 512 terms / 2^-6: together below 1e-2 of the gradients' size
    rng = np.random.default_rng(3)
    sp = Spec(3, 64, 64, 2, False, True, F32)
    rows, pos = 4, positions(rng, 4, 2)
    _, q, k, _ = qkv(rng, rows, 2, 1, 64, F32)
    _, gq, gk, _ = qkv(rng, rows, 2, 1, 64, F32)
    q, k, gq, gk = (x.contiguous() for x in (q, k, gq, gk))

    def loss(q, k):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko)
        return float((qo.double() * gq.double()).sum() + (ko.double() * gk.double()).sum())
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    dqw, dkw = torch.empty(64, device=DEV), torch.empty(64, device=DEV)
    ws = torch.empty(pa.padoc_qk_rotary_bwd_workspace_size(sp.dev, rows), dtype=torch.uint8, device=DEV)
    pa.padoc_qk_rotary_bwd(sp.dev, gq, gk, pos, dq, dk, q, k, dqw, dkw, ws)
    h = 2.0 ** -6
    for t, g, other in ((q, dq, k), (k, dk, q)):
        for at in [(0, 0, 0), (1, 0, 31), (2, 0, 32), (3, 0, 63)]:
            e = torch.zeros_like(t)
            e[at] = h
            two = [(loss(t + s * e, other) if t is q else loss(other, t + s * e)) for s in (1, -1)]
            assert abs((two[0] - two[1]) / (2 * h) - float(g[at])) < 1e-2
    for w, g in ((sp.qw, dqw), (sp.kw, dkw)):
        for j in (0, 17, 63):
            two = []
            for s in (1, -1):
                w[j] += s * h
                two.append(loss(q, k))
                w[j] -= s * h
            assert abs((two[0] - two[1]) / (2 * h) - float(g[j])) < 1e-2 * max(1, abs(float(g[j])))


def test_backward_of_short_heads_between_long_ones():
    # heads of several sizes share a kernel, whose shared memory differs: the limit set for one serves the others
    for d in (200, 40, 200, 248, 24, 248):
        sp = Spec(d, d, 8, 1, False, True, BF16)
        rng = np.random.default_rng(d)
        pos = positions(rng, 3, 1)
        _, q, k, _ = qkv(rng, 3, 2, 1, d, BF16)
        _, dqo, dko, _ = qkv(rng, 3, 2, 1, d, BF16)
        dq, dk = (torch.empty((3, h, d), dtype=BF16, device=DEV) for h in (2, 1))
        dqw, dkw = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        ws = torch.empty(pa.padoc_qk_rotary_bwd_workspace_size(sp.dev, 3), dtype=torch.uint8, device=DEV)
        pa.padoc_qk_rotary_bwd(sp.dev, dqo, dko, pos, dq, dk, q, k, dqw, dkw, ws)
        dx, size, dw, terms = sp.backward(dqo, q, sp.qw, pos)
        check(dq, dx, size, BWD, "dq")
        check(dqw, dw, terms, DW, "dq_weight")


def test_no_rows():
    sp = Spec(0, 128, 128, 3, False, True, BF16)
    e = lambda h: torch.empty((0, h, 128), dtype=BF16, device=DEV)
    pos = torch.empty((0, 3), dtype=torch.int32, device=DEV)
    pa.padoc_qk_rotary(sp.dev, e(16), e(2), pos, e(16), e(2))
    dqw, dkw = (torch.full((128,), float("nan"), device=DEV) for _ in range(2))
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    pa.padoc_qk_rotary_bwd(sp.dev, e(16), e(2), pos, e(16), e(2), e(16), e(2), dqw, dkw, ws)
    pa.padoc_check_device_errors()
    assert bool((dqw == 0).all()) and bool((dkw == 0).all())


def test_zero_and_infinite_heads():
    # a head of zeros norms to zero (eps above 0), its gradient is w g / sqrt(eps); an infinity gives NaN in its own head only
    sp = Spec(1, 128, 128, 1, False, True, BF16, eps=2.0 ** -12)
    rows, pos = 4, torch.arange(4, dtype=torch.int32, device=DEV)[:, None].contiguous()
    q = torch.randn((rows, 2, 128), device=DEV).to(BF16)
    q[0, 0] = 0
    q[1, 0, 5] = float("inf")
    k = q[:, :1].contiguous()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko)
    assert bool((qo[0, 0] == 0).all())
    assert bool(torch.isnan(qo[1, 0]).any()) and bool(torch.isfinite(qo[1, 1]).all())
    assert bool(torch.isfinite(qo[2:]).all()) and bool(torch.isfinite(qo[0]).all())
    g = torch.randn_like(q)
    gk = g[:, :1].contiguous()
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    dqw, dkw = torch.empty(128, device=DEV), torch.empty(128, device=DEV)
    ws = torch.empty(pa.padoc_qk_rotary_bwd_workspace_size(sp.dev, rows), dtype=torch.uint8, device=DEV)
    pa.padoc_qk_rotary_bwd(sp.dev, g, gk, pos, dq, dk, q, k, dqw, dkw, ws)
    dx, size, _, _ = orot.backward(f64(g)[:1, :1], f64(q)[:1, :1], f64(sp.qw), sp.eps, sp.angle(pos)[:1])
    check(dq[:1, :1], dx, size, BWD, "a zero head's gradient")
    pa.padoc_check_device_errors()


def test_positions_past_24_bits():
    # the angle is reduced in integers: positions of 2^30 turn as exactly as their table's entries (fp64
    # frequencies: 2 x 2^-53 x 0.16 x 2^30 turns = 2.4e-7 rad at frequency 1, and as much from the checker's own product)
    sp = Spec(2, 64, 64, 2, False, False, F32)
    rng = np.random.default_rng(5)
    pos = up(rng.integers(-2 ** 31, 2 ** 31, (300, 2)).astype(np.int32))
    _, q, k, _ = qkv(rng, 300, 2, 1, 64, F32)
    qo, ko = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko)
    want, size = sp.forward(q, None, pos)
    check(qo, want, size, FWD + 1e-6, "q")


def test_a_table_of_more_axes_reads_the_last_one():
    # three axes in the table, one in the rows: every pair takes that one, nothing past a row is read
    sp = Spec(7, 64, 64, 3, False, False, BF16)
    rng = np.random.default_rng(7)
    pos = positions(rng, 5, 1)
    _, q, k, _ = qkv(rng, 5, 2, 1, 64, BF16)
    sp.dev.c.num_axes = sp.dev.num_axes = 1
    qo, ko = torch.empty((5, 2, 64), dtype=BF16, device=DEV), torch.empty((5, 1, 64), dtype=BF16, device=DEV)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko)
    sp.axis = 0 * sp.axis
    check(qo, *sp.forward(q, None, pos), FWD, "q")
    check(ko, *sp.forward(k, None, pos), FWD, "k")


@pytest.mark.parametrize("what", ["dtype", "pos", "heads", "strides", "cpu", "weights", "slots", "expand", "align", "device"])
def test_python_refusals(what):
    sp = Spec(1, 64, 64, 1, False, True, BF16)
    q, k = torch.zeros((4, 2, 64), dtype=BF16, device=DEV), torch.zeros((4, 1, 64), dtype=BF16, device=DEV)
    pos = torch.zeros((4, 1), dtype=torch.int32, device=DEV)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    run = lambda q=q, k=k, pos=pos, qo=qo, ko=ko: pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko)
    run()
    if what == "dtype":
        for bad in (dict(q=q.float(), k=k.float()), dict(q=q.half(), k=k.half()), dict(qo=qo.float()), dict(k=k.float())):
            with pytest.raises((TypeError, ValueError)):
                run(**bad)
    elif what == "pos":
        for bad in (pos.long(), pos[:3], torch.zeros((4, 2), dtype=torch.int32, device=DEV), pos[:, 0], pos.cpu(), None):
            with pytest.raises(ValueError):
                run(pos=bad)
    elif what == "heads":
        for bad in (dict(qo=qo[:, :1]), dict(ko=qo), dict(q=q[..., :32]), dict(q=q.reshape(4, 128))):
            with pytest.raises(ValueError):
                run(**bad)
    elif what == "strides":
        wide = torch.zeros((4, 2, 128), dtype=BF16, device=DEV)
        for bad in (wide[..., :64], wide[..., ::2]):
            with pytest.raises(ValueError):
                run(q=bad)
    elif what == "cpu":
        with pytest.raises(ValueError):
            run(q=q.cpu())
    elif what == "weights":
        with pytest.raises(ValueError):
            pa.padoc_qk_rotary_bwd(sp.dev, q, k, pos, qo, ko)
        w = torch.empty(64, dtype=BF16, device=DEV)
        ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
        with pytest.raises(ValueError):
            pa.padoc_qk_rotary_bwd(sp.dev, q, k, pos, qo, ko, q, k, w, w, ws)
        with pytest.raises(pa.PadocError) as e:
            pa.padoc_qk_rotary_bwd(sp.dev, q, k, pos, qo, ko, q, k, w.float(), w.float(), ws[:256])
        assert e.value.status == 3
    elif what == "slots":
        pool = torch.zeros((2, 1, BS, 64), dtype=BF16, device=DEV)
        slots = torch.arange(4, dtype=torch.int32, device=DEV)
        for bad in (dict(slots=slots.long()), dict(slots=slots, count=5), dict(slots=slots, src_rows=slots[:2]),
                    dict(slots=slots, q_src=q), dict(slots=slots, q_src=q, q_dst=qo[:2]),
                    dict(slots=torch.arange(5, dtype=torch.int32, device=DEV))):
            with pytest.raises(ValueError):
                pa.padoc_append_rotary_inputs(sp.dev, pool, pool, k, k, pos, **bad)
        with pytest.raises(ValueError):
            pa.padoc_append_rotary_inputs(sp.dev, pool, pool[:1], k, k, pos, slots)
    elif what == "device":
        sp.dev._device = 1                           # (as if it were on a second GPU)
        with pytest.raises(ValueError, match="device"):
            run()
        pools = pa.KvPools([(torch.zeros((2, 1, BS, 64), device=DEV),) * 2])
        pools._device = 1
        i = torch.zeros(1, dtype=torch.int32, device=DEV)
        with pytest.raises(ValueError, match="device"):
            pa.padoc_copy_kv_blocks(pools, i, i)
    elif what == "expand":
        with pytest.raises(pa.PadocError) as e:      # rows that lie on one another
            run(q=q[:1].expand(4, 2, 64))
        assert e.value.status == 1
    else:
        flat = torch.zeros(4 * 128 + 4, dtype=BF16, device=DEV)[4:].view(4, 2, 64)
        with pytest.raises(pa.PadocError) as e:      # 8 bytes off a 16-byte boundary
            run(q=flat)
        assert e.value.status == 1


def test_on_a_side_stream_and_in_a_graph():
    sp = Spec(6, 128, 128, 3, False, True, BF16)
    rng = np.random.default_rng(6)
    rows, pos = 200, positions(rng, 200, 3)
    x, q, k, _ = qkv(rng, rows, 16, 2, 128, BF16)
    e = lambda h: torch.empty((rows, h, 128), dtype=BF16, device=DEV)
    qo, ko, dq, dk = e(16), e(2), e(16), e(2)
    dqw, dkw = torch.empty(128, device=DEV), torch.empty(128, device=DEV)
    ws = torch.empty(pa.padoc_qk_rotary_bwd_workspace_size(sp.dev, rows), dtype=torch.uint8, device=DEV)

    def both(stream=None):
        pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko, stream)
        pa.padoc_qk_rotary_bwd(sp.dev, qo, ko, pos, dq, dk, q, k, dqw, dkw, ws, stream)
    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in (qo, ko, dq, dk, dqw, dkw)]
    side = torch.cuda.Stream()
    for t in (qo, ko, dq, dk, dqw, dkw):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((qo, ko, dq, dk, dqw, dkw), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    x.copy_(torch.randn_like(x))
    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in (qo, ko, dq, dk, dqw, dkw)]
    for t in (qo, ko, dq, dk, dqw, dkw):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((qo, ko, dq, dk, dqw, dkw), want))


# ------------------------------------------------------------------------------------------------
# Append
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("shape", [s for s in SHAPES if s[4] in (64, 80, 128)], ids=ids)
def test_append_equals_rotation_then_append(shape):
    dtype, rows, hq, hkv, d, rot, axes, adjacent, norm, far = shape
    rng = np.random.default_rng(rows)
    sp = Spec(rows, d, rot, axes, adjacent, norm, dtype)
    pos = positions(rng, rows, axes, far)
    _, q, k, v = qkv(rng, rows, hq, hkv, d, dtype)
    nb = rows // BS + 9
    src = rng.permutation(rows)[:max(1, rows - 3)].astype(np.int32)
    slots = up(rng.permutation(nb * BS)[:len(src)].astype(np.int32))
    pools = [torch.full((nb, hkv, BS, d), 3.0, dtype=dtype, device=DEV) for _ in range(4)]
    qd, qr = (torch.full((len(src) + 2, hq, d), 5.0, dtype=dtype, device=DEV) for _ in range(2))
    pa.padoc_append_rotary_inputs(sp.dev, pools[0], pools[1], k, v, pos, slots, q, qd, up(src))
    qo, ko = torch.empty((rows, hq, d), dtype=dtype, device=DEV), torch.empty((rows, hkv, d), dtype=dtype, device=DEV)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qo, ko)
    pa.padoc_append_inputs(pools[2], pools[3], ko, v.contiguous(), slots, qo, qr, up(src))
    pa.padoc_check_device_errors()
    assert torch.equal(qd, qr) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    # without queries and without a row list
    n = len(src)
    for p in pools:
        p.fill_(3.0)
    pa.padoc_append_rotary_inputs(sp.dev, pools[0], pools[1], k, v, pos, slots, count=n)
    pa.padoc_append_inputs(pools[2], pools[3], ko, v.contiguous(), slots, count=n)
    pa.padoc_check_device_errors()
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])


def test_append_past_32_bits():
    # a pool whose byte offsets pass 2^32, and sources whose rows lie far apart
    rng = np.random.default_rng(8)
    sp = Spec(8, 128, 128, 1, False, True, BF16)
    nb = (9 << 30) // (2 * BS * 128 * 2) // 2
    k_pool, v_pool = (torch.zeros((nb, 2, BS, 128), dtype=BF16, device=DEV) for _ in range(2))
    rows, stride = 5, 1 << 28
    buf = torch.zeros(rows * stride, dtype=BF16, device=DEV)
    view = lambda off, h: torch.as_strided(buf, (rows, h, 128), (stride, 128, 1), off)
    q, k, v = view(0, 16), view(16 * 128, 2), view(18 * 128, 2)
    for t in (q, k, v):
        t.copy_(torch.randn(t.shape, device=DEV))
    pos = positions(rng, rows, 1)
    slots = up(np.array([nb * BS - 1, 0, nb * BS - 17, 5, (nb // 2) * BS + 3], np.int32))
    qd = torch.empty((rows, 16, 128), dtype=BF16, device=DEV)
    pa.padoc_append_rotary_inputs(sp.dev, k_pool, v_pool, k, v, pos, slots, q, qd)
    pa.padoc_check_device_errors()
    sl = slots.cpu().numpy()
    check(qd, *sp.forward(q, sp.qw, pos), FWD, "q")
    got_k = torch.stack([k_pool[int(s) // BS, :, int(s) % BS] for s in sl])
    got_v = torch.stack([v_pool[int(s) // BS, :, int(s) % BS] for s in sl])
    check(got_k, *sp.forward(k, sp.kw, pos), FWD, "k")
    assert torch.equal(got_v, v)
    assert int((k_pool != 0).any(-1).sum()) == rows * 2


def _bad_slots_case(e4m3):
    sp = Spec(9, 128, 128, 1, False, False, BF16)
    rng = np.random.default_rng(9)
    _, q, k, v = qkv(rng, 6, 16, 2, 128, BF16)
    pos = positions(rng, 6, 1)
    nb = 4
    return sp, q, k, v, pos, nb


@pytest.mark.parametrize("bad", ["slot_high", "slot_low", "row_high", "row_low"])
@pytest.mark.parametrize("e4m3", [False, True])
def test_append_bad_ids_are_reported_and_skipped(bad, e4m3):
    sp, q, k, v, pos, nb = _bad_slots_case(e4m3)
    slots, src = np.array([3, 20, 40], np.int32), np.array([1, 4, 0], np.int32)
    (slots if bad.startswith("slot") else src)[1] = {"slot_high": nb * BS, "slot_low": -1, "row_high": 6, "row_low": -7}[bad]
    qd = torch.full((3, 16, 128), 5.0, dtype=BF16, device=DEV)
    if e4m3:
        pool = pa.E4M3Pool(nb, 2, 128, DEV)
        pool.k_scales.fill_(1e-9)   # (a former owner's scale)
        pa.padoc_append_rotary_inputs_e4m3(sp.dev, pool, k, v, pos, up(slots), q, qd, up(src))
        written = lambda b, r: bool((pool.k_codes[b, :, r] != 0).any())
    else:
        kp, vp = (torch.zeros((nb, 2, BS, 128), dtype=BF16, device=DEV) for _ in range(2))
        pa.padoc_append_rotary_inputs(sp.dev, kp, vp, k, v, pos, up(slots), q, qd, up(src))
        written = lambda b, r: bool((kp[b, :, r] != 0).any())
    with pytest.raises(pa.PadocError) as e:
        pa.padoc_check_device_errors()
    assert e.value.device_code == 1 and e.value.device_detail == int((slots if bad.startswith("slot") else src)[1])
    assert written(0, 3) and written(2, 8) and not written(1, 4)
    assert bool((qd[1] == 5).all()) and bool((qd[0] != 5).any()) and bool((qd[2] != 5).any())
    pa.padoc_check_device_errors()


# ------------------------------------------------------------------------------------------------
# Append into the FP8 pool
# ------------------------------------------------------------------------------------------------

def e4m3_model(codes, scales, slots, x):
    """The append's rule for rows x [count][Hkv][d] in fp32: (codes, scales), exact for exact inputs."""
    codes, scales = codes.copy(), scales.copy()
    i = 0
    while i < len(slots):
        n = 1
        while i + n < len(slots) and slots[i + n] == slots[i] + n and slots[i + n] % BS:
            n += 1
        b, r0 = slots[i] // BS, slots[i] % BS
        for g in range(scales.shape[1]):
            old = np.float32(0) if r0 == 0 else scales[b, g]
            new = max(old, np.abs(x[i:i + n, g]).max() / np.float32(448))
            if new > old > 0:
                codes[b, g, :r0] = oracle.e4m3_encode(oracle.e4m3_decode(codes[b, g, :r0]).astype(np.float32) * old / new)
            codes[b, g, r0:r0 + n] = oracle.e4m3_encode(x[i:i + n, g] / new) if new > 0 else 0
            scales[b, g] = new
        i += n
    return codes, scales


def stale_pool(rng, nb, hkv):
    pool = pa.E4M3Pool(nb, hkv, 128, DEV)
    for c in (pool.k_codes, pool.v_codes):
        c.copy_(up(rng.integers(0, 0x7E, tuple(c.shape)).astype(np.uint8)))
    for s in (pool.k_scales, pool.v_scales):
        s.copy_(up(rng.uniform(0.001, 0.02, tuple(s.shape)).astype(np.float32)))
    return pool


def runs(rng, kind, nb):
    """Slots of a call: one input a block, whole prefixes of odd length, chunks that start inside a block."""
    blocks = rng.permutation(nb)
    if kind == "step":
        return np.array([b * BS + rng.integers(0, BS) for b in blocks[:nb - 2]], np.int32)
    if kind == "prefix":
        return np.array([blocks[t // BS] * BS + t % BS for t in range(BS * (nb - 2) - 5)], np.int32)
    out, b = [], 0
    while b < nb - 4:
        first, n = int(rng.integers(0, BS)), int(rng.integers(1, 40))
        out += [blocks[b + (first + j) // BS] * BS + (first + j) % BS for j in range(n)]
        b += (first + n - 1) // BS + 1
    return np.array(out, np.int32)


@pytest.mark.parametrize("nb", [23, 260])     # (from some 1200 inputs on a warp looks through several)
@pytest.mark.parametrize("kind", ["step", "prefix", "chunks"])
@pytest.mark.parametrize("hq,hkv,rot,axes,adjacent,norm", [(16, 2, 128, 3, False, True), (8, 1, 64, 1, False, False),
                                                             (10, 5, 128, 2, True, True), (16, 2, 24, 3, True, False)])
def test_append_e4m3(kind, hq, hkv, rot, axes, adjacent, norm, nb):
    rng = np.random.default_rng(hq + rot)
    sp = Spec(rot, 128, rot, axes, adjacent, norm, BF16)
    slots = runs(rng, kind, nb)
    n = len(slots)
    rows = n + 4
    x, q, k, v = qkv(rng, rows, hq, hkv, 128, BF16, 3.0)
    x[:3] = 0                                   # rows of zeros
    pos = positions(rng, rows, axes)
    src = rng.permutation(rows)[:n].astype(np.int32)
    if kind == "step":
        src[:2] = [0, 1]
        slots[0] = slots[0] // BS * BS          # a block that starts with a row of zeros
    pool = stale_pool(rng, nb, hkv)
    before = [t.cpu().numpy() for t in (pool.k_codes, pool.k_scales, pool.v_codes, pool.v_scales)]
    qd = torch.empty((n, hq, 128), dtype=BF16, device=DEV)
    pa.padoc_append_rotary_inputs_e4m3(sp.dev, pool, k, v, pos, up(slots), q, qd, up(src))
    pa.padoc_check_device_errors()
    kc, ks, vc, vs = (t.cpu().numpy() for t in (pool.k_codes, pool.k_scales, pool.v_codes, pool.v_scales))
    at = torch.from_numpy(src.astype(np.int64)).to(DEV)
    check(qd, *sp.forward(q[at], sp.qw, pos[at]), FWD, "q")
    # V is not rotated: the rule bit for bit
    want_c, want_s = e4m3_model(before[2], before[3], slots, f64(v[at]).astype(np.float32))
    np.testing.assert_array_equal(vs, want_s)
    np.testing.assert_array_equal(vc, want_c)
    # K: the scale within the values' bound; with the GPU's scale, earlier rows bit for bit, new rows' codes
    # within half a step of the format (2^-4 of the value, 2^-10 of the scale where codes are subnormal)
    want, size = sp.forward(k[at], sp.kw, pos[at])
    touched = {}
    for i, s in enumerate(slots.tolist()):
        touched.setdefault(s // BS, []).append((s % BS, i))
    for b in range(nb):
        rows_in = [r for r, _ in touched.get(b, [])]
        r0 = min(rows_in, default=BS)
        for g in range(hkv):
            if b in touched:
                old = np.float32(0) if r0 == 0 else before[1][b, g]
                z = np.abs(np.stack([want[i, g] for _, i in touched[b]]))
                e = np.stack([size[i, g] for _, i in touched[b]]).max() * FWD
                assert abs(ks[b, g] - max(old, z.max() / 448)) <= (e / 448) + ks[b, g] * 2.0 ** -23
                if ks[b, g] == old or old == 0:
                    keep = before[0][b, g, :r0]
                else:
                    keep = oracle.e4m3_encode(oracle.e4m3_decode(before[0][b, g, :r0]).astype(np.float32) * old / ks[b, g])
                np.testing.assert_array_equal(kc[b, g, :r0], keep)
                for r, i in touched[b]:
                    got = oracle.e4m3_decode(kc[b, g, r]).astype(np.float64) * ks[b, g]
                    tol = np.maximum(2.0 ** -4 * np.abs(want[i, g]), 2.0 ** -10 * ks[b, g]) * (1 + 1e-5) + 2 * FWD * size[i, g]
                    assert (np.abs(got - want[i, g]) <= tol).all()
            rest = [r for r in range(r0, BS) if r not in rows_in]
            np.testing.assert_array_equal(kc[b, g, rest], before[0][b, g, rest])


@pytest.mark.parametrize("special", [False, True])
def test_append_e4m3_without_angles_equals_the_plain_append(special):
    # all positions 0, no norm: K goes in as it is, so single rows give the plain append's bits. special: infinities, NaN and
    # subnormals in V
    rng = np.random.default_rng(14)
    sp = Spec(14, 128, 128, 3, False, False, BF16)
    nb = 40
    slots = runs(rng, "step", nb)
    x, q, k, v = qkv(rng, len(slots), 16, 2, 128, BF16, 2.0)
    if special:
        v[3, 0, 7], v[4, 1, 100], v[5, 0, 0] = float("inf"), float("nan"), -float("inf")
        v[6] = float("nan")
        v[7, 1, 3:9] = 1e-40
    pos = torch.zeros((len(slots), 3), dtype=torch.int32, device=DEV)
    a = stale_pool(rng, nb, 2)
    b = pa.E4M3Pool.over(*(t.clone() for t in (a.k_codes, a.v_codes, a.k_scales, a.v_scales)))
    qa, qb = (torch.empty((len(slots), 16, 128), dtype=BF16, device=DEV) for _ in range(2))
    pa.padoc_append_rotary_inputs_e4m3(sp.dev, a, k, v, pos, up(slots), q, qa)
    pa.padoc_append_inputs_e4m3(b, k.contiguous(), v.contiguous(), up(slots), q.contiguous(), qb)
    pa.padoc_check_device_errors()
    for x, y in ((a.k_codes, b.k_codes), (a.v_codes, b.v_codes), (a.k_scales, b.k_scales), (a.v_scales, b.v_scales), (qa, qb)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("e4m3", [False, True])
def test_append_captured_replayed_and_on_two_streams(e4m3):
    # a captured append reads the buffers' contents at each replay; two streams append to pools of their own at once
    sp = Spec(31, 128, 128, 3, False, True, BF16)
    rng = np.random.default_rng(31)
    n, nb = 40, 60
    _, q, k, v = qkv(rng, n, 16, 2, 128, BF16)
    pos = positions(rng, n, 3)
    slots = up(runs(rng, "step", nb)[:n])
    src = torch.arange(n, dtype=torch.int32, device=DEV)

    def new_pool():
        if e4m3:
            return stale_pool(np.random.default_rng(5), nb, 2)
        return tuple(torch.full((nb, 2, BS, 128), 2.0, dtype=BF16, device=DEV) for _ in range(2))

    def tensors(p):
        return (p.k_codes, p.v_codes, p.k_scales, p.v_scales) if e4m3 else p

    def append(p, qd, stream=None):
        if e4m3:
            pa.padoc_append_rotary_inputs_e4m3(sp.dev, p, k, v, pos, slots, q, qd, src, stream=stream)
        else:
            pa.padoc_append_rotary_inputs(sp.dev, *p, k, v, pos, slots, q, qd, src, stream=stream)
    qd = [torch.zeros((n, 16, 128), dtype=BF16, device=DEV) for _ in range(4)]
    want = new_pool()
    append(want, qd[0])
    streams, pools = [torch.cuda.Stream() for _ in range(2)], [new_pool() for _ in range(2)]
    torch.cuda.synchronize()
    for s, p, d in zip(streams, pools, qd[1:]):
        append(p, d, s)
    torch.cuda.synchronize()
    for p, d in zip(pools, qd[1:]):
        assert all(torch.equal(a, b) for a, b in zip(tensors(p), tensors(want))) and torch.equal(d, qd[0])
    graph, held = torch.cuda.CUDAGraph(), new_pool()
    with torch.cuda.graph(graph):
        append(held, qd[3])
    src.copy_(src.flip(0))
    pos.add_(7)
    append(want, qd[0])
    for t, x in zip(tensors(held), tensors(pools[0])):
        t.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(tensors(held), tensors(want))) and torch.equal(qd[3], qd[0])
    # nothing to append
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    if e4m3:
        pa.padoc_append_rotary_inputs_e4m3(sp.dev, held, k, v, pos, none)
    else:
        pa.padoc_append_rotary_inputs(sp.dev, *held, k, v, pos, none)
    pa.padoc_check_device_errors()
    assert all(torch.equal(a, b) for a, b in zip(tensors(held), tensors(want)))


def test_runner_rotary_is_set_replaced_and_taken_off():
    sp = Spec(32, 128, 128, 1, False, True, BF16)
    mpd = pa.Mpd(8)
    pool = tuple(torch.zeros((8, 2, BS, 128), dtype=BF16, device=DEV) for _ in range(2))
    cfg = pa.make_decode_config(16, 2, 128)
    runner = pa.MpdRunner(mpd, cfg, pa.make_kv_pool(*pool))
    _, q, k, v = qkv(np.random.default_rng(32), 4, 16, 2, 128, BF16)
    q, k, v = (t.contiguous() for t in (q, k, v))
    pos = torch.arange(4, dtype=torch.int32, device=DEV)[:, None].contiguous()
    out, lse = torch.empty((4, 16, 128), dtype=BF16, device=DEV), torch.empty((4, 16), device=DEV)
    mpd.add_page(0, 0)
    row = np.zeros(4, np.int32)
    kr, qr = torch.empty_like(k), torch.empty_like(q)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qr, kr)

    def step(r):
        row[:] = r
        runner.step(k, v, q, row, 0.1, out, lse)
        mpd.end_step(num_streams=1)
        torch.cuda.synchronize()
    step(1)
    runner.set_rotary(sp.dev, pos)
    step(2)
    runner.set_rotary(sp.dev, pos[:3])
    row[:] = 1
    with pytest.raises(pa.PadocError) as e:              # four source rows, three positions
        runner.step(k, v, q, row, 0.1, out, lse)
    assert e.value.status == 1 and mpd.status()[1] == 1
    runner.set_rotary(None)
    step(3)
    pa.padoc_check_device_errors()
    got = pool[0][0, :, :3]
    assert torch.equal(got[:, 0], k[1]) and torch.equal(got[:, 1], kr[2]) and torch.equal(got[:, 2], k[3])
    small = Spec(32, 64, 64, 1, False, False, BF16)
    with pytest.raises(pa.PadocError):
        runner.set_rotary(small.dev, pos)                # another head_dim
    with pytest.raises(TypeError):
        runner.set_rotary(Spec(32, 128, 128, 1, False, True, F32).dev, pos)


# ------------------------------------------------------------------------------------------------
# Together: a training layer, and the decoding loop
# ------------------------------------------------------------------------------------------------

GRIDS = [(0, 3, 1, 6, 8), (1, 0, 2, 3, 4)]
PAGES = [PageSpec(60, 12, [0, 5, 12, 5], [17, 3, 30, 1]), PageSpec(26, 6, [6, 2], [9, 20])]


def test_training_layer_fp32_against_fp64():
    # projections -> norm, rotation -> ancestor attention -> its backward -> the rotation's and norm's
    # backward, against the chain in 64 bits. fp32 attention is held to 1e-4 forward, and backward to 1e-4 of the
    # row's largest plus 1e-5 of the root mean square (the fp32 path's own bounds). Rotated rows that are off by 3e-6
    # shift scores of up to 10 by 3e-5, which changes probabilities and gradients by as much relative to their
    # size: twice the bounds before the last step; the norm's Jacobian adds two such errors per value: four times.
    hq, hkv, d = 4, 1, 64
    sp = Spec(21, d, d, 3, False, True, F32)
    layer = RotaryPrefill(PAGES, sp.dev, hq, hkv, F32, DEV, GRIDS, training=True)
    T = layer.T
    rng = np.random.default_rng(21)
    _, q, k, v = qkv(rng, T, hq, hkv, d, F32)
    v = v.contiguous()
    scale = 1 / math.sqrt(d)
    out, lse = torch.empty((T, hq, d), device=DEV), torch.empty((T, hq), device=DEV)
    layer.run(q, k, v, scale, out, lse)
    dout = up(rng.standard_normal((T, hq, d)).astype(np.float32))
    dq, dk, dv = (torch.empty((T, h, d), device=DEV) for h in (hq, hkv, hkv))
    dqw, dkw = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    layer.run_bwd(q, k, v, out, dout, lse, scale, dq, dk, dv, dqw, dkw)
    pa.padoc_check_device_errors()
    pos = layer.pos
    np.testing.assert_array_equal(pos.cpu().numpy(), pa.padoc_build_rotary_positions(PAGES, GRIDS)[0])
    zq, zk = sp.forward(q, sp.qw, pos)[0], sp.forward(k, sp.kw, pos)[0]
    tq, tk = (torch.from_numpy(z.astype(np.float32)) for z in (zq, zk))
    ro, rl = oracle.prefill_dense(PAGES, tq, tk, v.cpu(), scale)
    assert np.abs(f64(out) - ro).max() <= 2e-4 and np.abs(f64(lse) - rl).max() <= 2e-4
    gq, gk, gv = oracle.prefill_bwd(PAGES, tq, tk, v.cpu(), dout.cpu(), scale)
    want_q, want_k = orot.backward(gq, f64(q), f64(sp.qw), sp.eps, sp.angle(pos)), orot.backward(gk, f64(k), f64(sp.kw), sp.eps, sp.angle(pos))
    for got, want in ((dq, want_q[0]), (dk, want_k[0]), (dv, gv)):
        rms = math.sqrt((want ** 2).mean())
        err = np.abs(f64(got) - want).reshape(T, -1).max(1)
        assert (err <= 4e-4 * np.abs(want).reshape(T, -1).max(1) + 4e-5 * rms).all()
    # the weights' gradients sum the rows': their bounds add up in the same way
    for got, want in ((dqw, want_q), (dkw, want_k)):
        assert (np.abs(f64(got) - want[2]) <= 4e-4 * want[3]).all()


def test_training_layer_bf16_runs_on_its_own_rotated_rows():
    hq, hkv, d = 16, 2, 128
    sp = Spec(22, d, d, 3, False, True, BF16)
    layer = RotaryPrefill(PAGES, sp.dev, hq, hkv, BF16, DEV, GRIDS, training=True)
    T = layer.T
    rng = np.random.default_rng(22)
    _, q, k, v = qkv(rng, T, hq, hkv, d, BF16)
    v = v.contiguous()
    scale = 1 / math.sqrt(d)
    out, lse = torch.empty((T, hq, d), dtype=BF16, device=DEV), torch.empty((T, hq), device=DEV)
    layer.run(q, k, v, scale, out, lse)
    pa.padoc_check_device_errors()
    check(layer.q, *sp.forward(q, sp.qw, layer.pos), FWD, "q")
    ro, rl = oracle.prefill_dense(PAGES, layer.q.cpu(), layer.k.cpu(), v.cpu(), scale)
    assert np.abs(f64(out) - ro).max() <= 1.5e-2 and np.abs(f64(lse) - rl).max() <= 1e-3
    dout = up(rng.standard_normal((T, hq, d))).to(BF16)
    new = lambda h: torch.empty((T, h, d), dtype=BF16, device=DEV)
    dq, dk, dv, zq, zk = new(hq), new(hkv), new(hkv), new(hq), new(hkv)
    dqw, dkw = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    layer.run_bwd(q, k, v, out, dout, lse, scale, dq, dk, dv, dqw, dkw)
    layer.bwd.run(layer.q, layer.k, v, out, dout, lse, scale, zq, zk, dv)
    pa.padoc_check_device_errors()
    for got, dz, x, w, gw, name in ((dq, zq, q, sp.qw, dqw, "dq"), (dk, zk, k, sp.kw, dkw, "dk")):
        dx, size, dw, terms = sp.backward(dz, x, w, layer.pos)
        check(got, dx, size, BWD, name)
        check(gw, dw, terms, DW, name + "_weight")


@pytest.mark.parametrize("e4m3", [False, True])
def test_prefix_and_chunk_appended_then_attended(e4m3):
    # a page's prefix and layout tokens go into the cache in one call, a branch's 21 tokens in another, which also
    # lays out their queries; then the chunk is prefilled (bf16), or its newest token decoded (FP8), against the oracle
    # over the rotated rows, resp. over what the codes stand for (the decode's own tolerances)
    P, L, f, n = 70, 10, 4, 21
    page = PageSpec(P, L, [f], [n])
    sp = Spec(33, 128, 128, 3, False, True, BF16)
    rng = np.random.default_rng(33)
    T, scale = P + L + n, 128 ** -0.5
    x, q, k, v = qkv(rng, T, 16, 2, 128, BF16)
    pos = up(pa.padoc_build_rotary_positions([page], [(0, 2, 1, 8, 8)])[0])
    blocks = rng.permutation(12).astype(np.int32)
    shared, private = blocks[:5], blocks[5:7]
    slots = np.concatenate([shared[np.arange(P + L) // BS] * BS + np.arange(P + L) % BS,
                            private[np.arange(n) // BS] * BS + np.arange(n) % BS]).astype(np.int32)
    rows = np.arange(T, dtype=np.int32)
    qd = torch.empty((n, 16, 128), dtype=BF16, device=DEV)
    if e4m3:
        pool = stale_pool(rng, 12, 2)
        append = lambda *a, **kw: pa.padoc_append_rotary_inputs_e4m3(sp.dev, pool, k, v, pos, *a, **kw)
    else:
        kp, vp = (torch.zeros((12, 2, BS, 128), dtype=BF16, device=DEV) for _ in range(2))
        append = lambda *a, **kw: pa.padoc_append_rotary_inputs(sp.dev, kp, vp, k, v, pos, *a, **kw)
    append(up(slots[:P + L]))
    append(up(slots[P + L:]), q, qd, up(rows[P + L:]))
    page_table, table = up(shared[None]), private[None]
    if e4m3:
        plan = DecodePlan([page], 16, 2, 128, DEV)
        out, lse = torch.empty((1, 16, 128), dtype=BF16, device=DEV), torch.empty((1, 16), device=DEV)
        newest = qd[n - 1:].contiguous()
        pa.padoc_branch_decode_attn_e4m3(pool, plan.info, plan.plan_dev, page_table, up(table), newest, scale, out, lse,
                                         plan.workspace)
        pa.padoc_check_device_errors()
        deq = [oracle.dequantize_kv_blocks(c.cpu().numpy(), s.cpu().numpy())
               for c, s in ((pool.k_codes, pool.k_scales), (pool.v_codes, pool.v_scales))]
        ro, rl = oracle.decode_paged([page], *deq, shared[None], table, newest.cpu(), scale)
        # and the codes stand for the rotated rows: half a step of the format at the block's largest magnitude
        want = sp.forward(k, sp.kw, pos)[0]
        held = np.stack([deq[0][s // BS, :, s % BS] for s in slots])
        step = np.stack([pool.k_scales.cpu().numpy()[s // BS] for s in slots])[..., None]
        assert (np.abs(held - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * step) * 1.001 + 1e-4).all()
    else:
        plan = ChunkPrefillPlan([P + L], [(0, P + f, 0, n)], table, 16, 2, 128, DEV)
        out, lse = torch.empty((n, 16, 128), dtype=BF16, device=DEV), torch.empty((n, 16), device=DEV)
        plan.run(kp, vp, page_table, qd, scale, out, lse)
        pa.padoc_check_device_errors()
        qr, kr = torch.empty((T, 16, 128), dtype=BF16, device=DEV), torch.empty((T, 2, 128), dtype=BF16, device=DEV)
        pa.padoc_qk_rotary(sp.dev, q, k, pos, qr, kr)
        ro, rl = oracle.prefill_dense([page], qr.cpu(), kr.cpu(), v.cpu(), scale)
        ro, rl = ro[P + L:], rl[P + L:]
    assert np.abs(f64(out) - ro).max() <= 1.5e-2 and np.abs(f64(lse) - rl).max() <= 1e-3


LOOP_PAGES = [PageSpec(60, 10, [0, 10, 3, 7], [17, 5, 33, 16]), PageSpec(130, 24, [24, 12, 8, 20, 4], [2, 40, 12, 30, 18])]


def loop(rows_q, rows_k, rows_v, rotary, pos, mode, act=None, dtype=BF16, num_blocks=64, events=None):
    """Runs Algorithm 1 over LOOP_PAGES; act(loop, step) after each step. Returns {packed row: (out, lse)}."""
    src = LoopTokenSource(LOOP_PAGES)
    hq, hkv, d = rows_q.shape[1], rows_k.shape[1], rows_k.shape[2]
    lp = MaskedParallelLoop(num_blocks, hq, hkv, d, dtype, DEV, block_order=np.random.default_rng(1).permutation(num_blocks),
                            rotary=rotary)
    for p in range(len(LOOP_PAGES)):
        P, nf, leos, prow = src.admission(p)
        _, new = lp.add_page(P, nf, leos, rows_k, rows_v, prow, pos_src=pos)
        src.admitted(p, new)
    cap = sum(1 + pg.num_branches for pg in LOOP_PAGES)   # every stream id the loop can create
    out = torch.empty((cap, hq, d), dtype=dtype, device=DEV)
    lse = torch.empty((cap, hq), dtype=torch.float32, device=DEV)
    row_of, got, step = np.zeros(cap, np.int32), {}, 0
    while lp.status()[1]:
        if mode == "runner":
            row_of[:] = src.peek_rows(np.arange(cap))
            n, ids = lp.run_step(rows_k, rows_v, rows_q, row_of, 1 / math.sqrt(d), out, lse, pos_src=pos)
            ids = ids.copy()
            src.rows(ids)
            o, l = out[:n], lse[:n]
        else:
            ids, o, l = lp.step(rows_k, rows_v, rows_q, src.rows, 1 / math.sqrt(d), pos_src=pos)
        for r, a, b in zip(src.token_rows(ids).tolist(), o.clone(), l.clone()):
            got[r] = (a, b)
        nf, eos = src.events(ids)
        src.forked(ids, nf, lp.end_step(nf, eos))
        step += 1
        if act is not None:
            act(lp, step)
    pa.padoc_check_device_errors()
    assert lp.status()[2] == lp.k_pool.shape[0]
    return got


@pytest.mark.parametrize("mode", ["step", "runner"])
def test_loop_with_rotary_equals_the_loop_over_rotated_rows(mode):
    # also with the pool compacted after every fifth step and replaced by larger and smaller ones
    sp = Spec(23, 128, 128, 3, False, True, BF16)
    T = sum(pg.packed_len for pg in LOOP_PAGES)
    pos = up(pa.padoc_build_rotary_positions(LOOP_PAGES, [(0, 3, 1, 6, 8), (1, 10, 1, 10, 10)])[0])
    _, q, k, v = qkv(np.random.default_rng(23), T, 16, 2, 128, BF16)
    q, k, v = (t.contiguous() for t in (q, k, v))
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qr, kr)
    want = loop(qr, kr, v, None, None, mode)
    got = loop(q, k, v, sp.dev, pos, mode)

    def act(lp, step):
        if step % 5 == 0:
            live = lp.compact()
            assert lp.status()[2] == lp.k_pool.shape[0] - live
        if step % 9 == 0:
            lp.resize({0: 64, 1: 41, 2: 77}[step // 9 % 3])
    moved = loop(q, k, v, sp.dev, pos, mode, act)
    assert set(want) == set(got) == set(moved)
    for r in want:
        for other in (got, moved):
            assert torch.equal(want[r][0], other[r][0]) and torch.equal(want[r][1], other[r][1])


@pytest.mark.parametrize("mode", ["step", "runner"])
def test_forked_candidates_decode_like_their_origin_and_then_apart(mode):
    # a branch with 21 rows is forked in three; every candidate goes on with its own inputs, and each equals
    # a branch that had that history from the start (oracle over the packed page)
    sp = Spec(24, 128, 128, 1, False, True, BF16)
    n, more = 21, 14
    first = PageSpec(50, 4, [2], [n])
    rng = np.random.default_rng(24)
    hist = 50 + 4 + n
    rows = hist + 3 * more
    _, q, k, v = qkv(rng, rows, 16, 2, 128, BF16)
    q, k, v = (t.contiguous() for t in (q, k, v))
    place = np.concatenate([np.arange(54), 52 + np.arange(n)] + [52 + n + np.arange(more)] * 3).astype(np.int32)
    pos = up(place[:, None])
    lp = MaskedParallelLoop(40, 16, 2, 128, BF16, DEV, rotary=sp.dev)
    _, new = lp.add_page(50, 0, False, k, v, np.arange(50), pos_src=pos)
    layout = int(new[0])
    out, lse = torch.empty((8, 16, 128), dtype=BF16, device=DEV), torch.empty((8, 16), device=DEV)
    row_of = np.zeros(16, np.int32)

    def step(rows_by_id, forks=None, eos=()):
        for s, r in rows_by_id.items():
            row_of[s] = r
        if mode == "runner":
            c, ids = lp.run_step(k, v, q, row_of, 128 ** -0.5, out, lse, pos_src=pos)
            ids, o = ids.copy(), out[:c].clone()
        else:
            ids, o, _ = lp.step(k, v, q, lambda i: row_of[i], 128 ** -0.5, pos_src=pos)
        res = dict(zip(ids.tolist(), o))
        made = lp.end_step(np.array([(forks or {}).get(int(i), 0) for i in ids], np.int32),
                           np.array([int(i) in eos for i in ids], np.uint8))
        return res, made.tolist()
    step({layout: 50})
    _, (a,) = step({layout: 51}, forks={layout: 1})
    step({layout: 52, a: 54})
    step({layout: 53, a: 55}, eos=(layout,))
    for j in range(2, n):
        step({a: 54 + j})
    b, c = (int(x) for x in lp.fork_stream(a, 2))
    assert lp.status()[1] == 3
    got = {a: [], b: [], c: []}
    for j in range(more):
        if j == 6:
            lp.compact()
        res, _ = step({s: hist + i * more + j for i, s in enumerate((a, b, c))})
        for s in got:
            got[s].append(res[s])
    lp.drop_stream(b)
    assert lp.status()[1] == 2
    lp.drop_page(0)
    assert lp.status() == (0, 0, 40)
    pa.padoc_check_device_errors()
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qr, kr)
    page = PageSpec(50, 4, [2], [n + more])
    for i, s in enumerate((a, b, c)):
        at = torch.cat([torch.arange(hist), hist + i * more + torch.arange(more)])
        ro, _ = oracle.prefill_dense([page], qr.cpu()[at], kr.cpu()[at], v.cpu()[at], 128 ** -0.5)
        assert np.abs(f64(torch.stack(got[s])) - ro[hist:]).max() <= 1.5e-2


def test_loop_without_positions_is_refused_and_positions_may_change_their_memory():
    sp = Spec(33, 128, 128, 1, False, True, BF16)
    _, q, k, v = qkv(np.random.default_rng(33), 4, 16, 2, 128, BF16)
    q, k, v = (t.contiguous() for t in (q, k, v))
    lp = MaskedParallelLoop(8, 16, 2, 128, BF16, DEV, rotary=sp.dev)
    lp.add_page(0, 0, False, k, v, np.zeros(0, np.int32))
    out, lse = torch.empty((4, 16, 128), dtype=BF16, device=DEV), torch.empty((4, 16), device=DEV)
    row = np.zeros(4, np.int32)
    with pytest.raises(ValueError):
        lp.run_step(k, v, q, row, 0.1, out, lse)
    pos = torch.arange(4, dtype=torch.int32, device=DEV)[:, None].contiguous()
    later = pos + 1000
    lp.run_step(k, v, q, row, 0.1, out, lse, pos_src=pos)
    lp.end_step(num_streams=1)
    kr, qr = [torch.empty_like(k) for _ in range(2)], torch.empty_like(q)
    pa.padoc_qk_rotary(sp.dev, q, k, pos, qr, kr[0])
    pa.padoc_qk_rotary(sp.dev, q, k, later, qr, kr[1])
    before = pos.data_ptr()
    pos.set_(later)                                       # the same object over other memory
    assert pos.data_ptr() != before
    lp.run_step(k, v, q, row, 0.1, out, lse, pos_src=pos)
    lp.end_step(num_streams=1)
    pa.padoc_check_device_errors()
    assert torch.equal(lp.k_pool[0, :, 0], kr[0][0]) and torch.equal(lp.k_pool[0, :, 1], kr[1][0])


@pytest.mark.parametrize("what", ["no positions", "positions short", "another dtype", "heads", "unaligned", "no rows"])
def test_loop_refuses_bad_sources_before_it_begins(what):
    # the refused call leaves the scheduler as it was, so the next one goes through
    sp = Spec(34, 128, 128, 1, False, False, BF16)
    _, q, k, v = qkv(np.random.default_rng(34), 6, 16, 2, 128, BF16)
    q, k, v = (t.contiguous() for t in (q, k, v))
    pos = torch.arange(6, dtype=torch.int32, device=DEV)[:, None].contiguous()
    bad = {"no positions": (k, v, q, None), "positions short": (k, v, q, pos[:5]),
           "another dtype": (k.float(), v.float(), q.float(), pos),
           "heads": (k[:, :1].contiguous(), v[:, :1].contiguous(), q, pos),
           "unaligned": (torch.zeros(6 * 256 + 4, dtype=BF16, device=DEV)[4:].view(6, 2, 128), v, q, pos),
           "no rows": (k[:0], v[:0], q[:0], pos[:0])}[what]
    lp = MaskedParallelLoop(8, 16, 2, 128, BF16, DEV, rotary=sp.dev)
    errors = (ValueError, TypeError, pa.PadocError)
    with pytest.raises(errors):
        lp.add_page(3, 0, False, bad[0], bad[1], np.arange(3), pos_src=bad[3])
    with pytest.raises(errors):
        lp.add_page(3, 0, False, k, v, np.arange(2), pos_src=pos)
    assert lp.status() == (0, 0, 8)
    lp.add_page(3, 0, False, k, v, np.arange(3), pos_src=pos)
    free = lp.status()
    out, lse = torch.empty((4, 16, 128), dtype=BF16, device=DEV), torch.empty((4, 16), device=DEV)
    row = np.full(4, 3, np.int32)
    with pytest.raises(errors):
        lp.step(*bad[:3], lambda i: row[i], 0.1, pos_src=bad[3])
    with pytest.raises(errors):
        lp.step(k, v, None, lambda i: row[i], 0.1, pos_src=pos)
    with pytest.raises(errors):
        lp.run_step(*bad[:3], row, 0.1, out, lse, pos_src=bad[3])
    assert lp.status() == free
    _, o, l = lp.step(k, v, q, lambda i: row[i], 0.1, pos_src=pos)
    lp.end_step(num_streams=1)
    row[:] = 4
    assert lp.run_step(k, v, q, row, 0.1, out, lse, pos_src=pos)[0] == 1
    lp.end_step(num_streams=1)
    pa.padoc_check_device_errors()
    assert torch.isfinite(o).all() and torch.isfinite(out[0]).all()


def test_gradients_of_a_layer_that_is_not_trained_are_refused():
    layer = RotaryPrefill(PAGES, Spec(35, 128, 128, 3, False, False, BF16).dev, 16, 2, BF16, DEV)
    with pytest.raises(ValueError):
        layer.run_bwd(*[None] * 6, 0.1, None, None, None)
