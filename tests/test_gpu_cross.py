"""Cross attention on the GPU against its definition in 64 bits, at the sizes and segments where it can go wrong.

Tolerances are oracle.cross's bounds (derived there), element by element."""
import math

import pytest
import torch

from oracle import cross as oc
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import CrossPlan

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32
NAN = math.nan


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def rows_of(n, heads, d, dtype, g, stride_heads=0):
    """[n][heads][d], a slice of a wider buffer (filled with NaN) when stride_heads is more than heads."""
    wide = torch.full((n, max(stride_heads, heads), d), NAN, dtype=dtype, device=DEV)
    at = (max(stride_heads, heads) - heads) // 2
    wide[:, at:at + heads] = torch.randn((n, heads, d), generator=g, device=DEV).to(dtype)
    return wide[:, at:at + heads]


def inputs(segments, hq, hkv, d, dtype, seed=0, rows=None, keys=None, wide=0, poison=True):
    """q, k, v, dout; rows that no segment names hold NaN and infinities."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows = rows or max([s[0] + s[1] for s in segments]) + 3
    keys = keys or max([s[2] + s[3] for s in segments]) + 2
    q, dout = rows_of(rows, hq, d, dtype, g, hq + wide), rows_of(rows, hq, d, dtype, g)
    k, v = rows_of(keys, hkv, d, dtype, g, hkv + 2 * wide), rows_of(keys, hkv, d, dtype, g, hkv + wide)
    if poison:
        nq, nk = torch.ones(rows, dtype=torch.bool), torch.ones(keys, dtype=torch.bool)
        for a, n, b, m in segments:
            nq[a:a + n] = False
            nk[b:b + (m if n else 0)] = False
        for t, bad in ((q, nq), (dout, nq), (k, nk), (v, nk)):
            t[bad.to(DEV)] = torch.tensor([NAN, math.inf], device=DEV, dtype=dtype).repeat(d // 2)
    return q, k, v, dout


def within(got, want, bound, rows=None):
    got, want = got.double(), want.clone()
    if rows is not None:
        got, want, bound = got[rows], want[rows], bound[rows]
    same = (got == want) | ((got - want).abs() <= bound)
    assert same.all(), f"{(~same).sum().item()} of {same.numel()} off, worst {((got - want).abs() / bound.clamp_min(1e-30)).nan_to_num(9e9).max().item():.3g} of the bound"


def check_forward(segments, hq, hkv, d, dtype, ctas=0, **kw):
    q, k, v, _ = inputs(segments, hq, hkv, d, dtype, **kw)
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV, ctas=ctas)
    out = torch.full((q.shape[0], hq, d), 77.0, dtype=dtype, device=DEV)
    lse = torch.full((q.shape[0], hq), 77.0, device=DEV)
    scale = 1 / math.sqrt(d)
    plan.workspace.fill_(255)     # NaN
    plan.run(q, k, v, scale, out, lse)
    pa.padoc_check_device_errors()
    want, wl, rows = oc.forward(segments, q, k, v, scale)
    bo, bl = oc.forward_bounds(segments, q, k, v, scale)
    within(out, want, bo, rows)
    within(lse, wl, bl, rows)
    assert (out[~rows] == 77).all() and (lse[~rows] == 77).all()
    first = out.clone()
    plan.run(q, k, v, scale, out, lse)
    assert torch.equal(first, out)
    return plan


def check_backward(segments, hq, hkv, d, dtype, ctas=0, **kw):
    q, k, v, dout = inputs(segments, hq, hkv, d, dtype, **kw)
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV, training=True, ctas=ctas)
    scale = 1 / math.sqrt(d)
    want, wl, rows = oc.forward(segments, q, k, v, scale)
    out, lse = want.to(dtype), wl.float()
    dq = torch.full_like(out, 77.0)
    dkv = torch.full((k.shape[0], 3 * hkv, d), 77.0, dtype=dtype, device=DEV)
    dk, dv = dkv[:, :hkv], dkv[:, 2 * hkv:]
    plan.bwd_workspace.fill_(255)
    plan.run_bwd(q, k, v, out, dout, lse, scale, dq, dk, dv)
    pa.padoc_check_device_errors()
    # NaN of unnamed rows does not reach the oracle either: it reads the segments' rows alone
    gq, gk, gv = oc.backward(segments, q, k, v, dout, scale)
    bq, bk, bv = oc.backward_bounds(segments, q, k, v, out, dout, scale)
    within(dq, gq, bq, rows)
    within(dk, gk, bk)
    within(dv, gv, bv)
    assert (dq[~rows] == 77).all() and (dkv[:, hkv:2 * hkv] == 77).all()
    first = [t.clone() for t in (dq, dk, dv)]
    plan.run_bwd(q, k, v, out, dout, lse, scale, dq, dk, dv)
    assert all(torch.equal(a, b) for a, b in zip(first, (dq, dk, dv)))
    return plan


HEADS = [(16, 2, 128), (16, 16, 64), (2, 2, 128), (7, 1, 64), (14, 2, 128), (64, 1, 128), (12, 4, 64), (33, 1, 64)]
EDGES = [
    [(0, 1, 0, 1)],
    [(0, 1, 3, 129)],
    [(2, 65, 5, 127)],
    [(0, 16, 0, 128), (16, 17, 128, 128)],
    [(0, 33, 1, 64), (33, 31, 66, 1), (70, 64, 70, 191)],
    [(0, 5, 0, 0), (5, 3, 0, 200), (9, 0, 0, 50), (9, 40, 3, 0)],           # rows without keys, a segment without rows
    [(0, 40, 10, 300), (40, 9, 20, 30), (49, 1, 309, 1), (50, 70, 10, 300), (120, 7, 250, 200)],   # shared key ranges
    [(0, 130, 0, 1), (130, 1, 0, 513)],
]


@pytest.mark.parametrize("segments", EDGES)
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward_edges(dtype, hq, hkv, d, segments):
    check_forward(segments, hq, hkv, d, dtype)


@pytest.mark.parametrize("segments", EDGES)
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_edges(dtype, hq, hkv, d, segments):
    check_backward(segments, hq, hkv, d, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("ctas", [1, 7, 0])
@pytest.mark.parametrize("keys", [2, 129, 1000, 4097])
def test_few_rows_over_long_keys(dtype, ctas, keys):
    # split over the chip and joined, or whole
    segments = [(0, 3, 1, keys), (3, 1, 0, keys + 1)]
    check_forward(segments, 16, 2, 128, dtype, ctas=ctas)
    check_backward(segments, 4, 2, 64, dtype, ctas=ctas)


@pytest.mark.parametrize("keys", [1, 15, 16, 17, 63, 64, 65, 129, 961, 20_000])
@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (16, 16, 64), (8, 8, 128), (32, 1, 64), (10, 2, 64), (3, 1, 128)])
def test_single_tokens(hq, hkv, d, keys):
    check_forward([(0, 1, 3, keys)], hq, hkv, d, BF16)
    check_forward([(1, 3, 2, keys), (4, 2, 0, 0), (6, 5, 1, keys + 7)], hq, hkv, d, BF16)


def test_every_way_of_few_rows():
    # a cluster of each size and keys cut into parts, tiles of 16 and of 32 rows
    seen = set()
    for heads in ((16, 2, 128), (4, 4, 64), (2, 2, 128)):
        for segments in ([(0, 2, 1, 900)], [(3 * i, 3, 40 * i, 30 + 9 * i) for i in range(20)], [(0, 1, 0, 30_000)],
                         [(17 * i, 17, 200 * i, 200) for i in range(40)], [(i, 1, 100 * i, 90) for i in range(90)],
                         [(i, 1, 0, 400) for i in range(16)]):
            info = check_forward(segments, *heads, BF16).info
            seen.add((info.few, info.num_slots > 0, info.unit_rows))
    assert {s[0] for s in seen} >= {0, 1, 2, 4, 8} and {s[2] for s in seen} >= {16, 32}, seen
    assert (1, True) in {s[:2] for s in seen}, seen


def test_document_of_many_states():
    check_forward([(0, 24, 7, 50_003)], 16, 2, 128, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_lie_apart(dtype):
    segments = [(1, 70, 2, 140), (71, 5, 30, 40)]
    check_forward(segments, 8, 2, 128, dtype, wide=4)
    check_backward(segments, 8, 2, 128, dtype, wide=4)


@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (16, 16, 64), (4, 4, 128)])
def test_many_rows(hq, hkv, d):
    # more units than SMs, several waves, every kind of launch
    segments = [(0, 1500, 0, 400), (1500, 1111, 400, 700), (2611, 300, 350, 100)]
    check_forward(segments, hq, hkv, d, BF16, poison=False)
    check_backward(segments, hq, hkv, d, BF16, poison=False)


@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (4, 1, 64), (7, 1, 128)])
def test_few_keys_that_many_rows_see(hq, hkv, d):
    # a key tile's rows shared out over the whole chip; key rows between that nobody sees
    plan = check_backward([(0, 900, 5, 70), (900, 60, 400, 200), (960, 3, 300, 10)], hq, hkv, d, BF16)
    assert plan.info.num_dkv_sums > 0 and plan.info.num_gap_tiles > 0
    for segments in ([(0, 900, 0, 700)], [(0, 130, 3, 128)], [(0, 2, 0, 100)]):
        check_backward(segments, hq, hkv, d, BF16)


@pytest.mark.parametrize("hq,hkv,d,dtype,rows,keys,ctas,cut", [
    (16, 2, 128, BF16, 700, 1490, 7, "fwd"), (16, 2, 128, BF16, 290, 2500, 7, "dq"), (4, 4, 64, BF16, 290, 1500, 5, "both"),
    (4, 4, 64, F32, 200, 501, 7, "dq")])
def test_the_last_round_is_cut(hq, hkv, d, dtype, rows, keys, ctas, cut):
    segments = [(3, rows, 10, keys)]
    check_forward(segments, hq, hkv, d, dtype, ctas=ctas)
    info = check_backward(segments, hq, hkv, d, dtype, ctas=ctas).info
    assert cut == "dq" or (info.num_ctas == 0 and info.num_slots > 0)
    assert cut == "fwd" or (info.num_dq_ctas == 0 and info.num_dq_slots > 0)


@pytest.mark.parametrize("hq,hkv,d", [(16, 16, 64), (16, 2, 128), (8, 8, 64)])
@pytest.mark.parametrize("keys", [1, 70, 130, 250])
def test_many_short_items(hq, hkv, d, keys):
    # items of a tile or two, each ending inside one, taken one after the other by every CTA; some with one tile of rows
    segments = [(40 * i, 40 if i % 3 else 7, keys * i % 900, keys) for i in range(60)]
    check_forward(segments, hq, hkv, d, BF16, poison=False)
    check_backward(segments, hq, hkv, d, BF16, poison=False)
    segments = [(600 * i, 600, keys * i, keys) for i in range(5)]
    check_forward(segments, hq, hkv, d, BF16, poison=False)
    check_backward(segments, hq, hkv, d, BF16, poison=False)


def test_many_rows_f32():
    segments = [(0, 700, 0, 400), (700, 311, 400, 300)]
    check_forward(segments, 4, 1, 64, F32)
    check_backward(segments, 4, 1, 64, F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_far_apart_sizes(dtype):
    # keys that grow by steps: the running maximum moves at every tile, and early weights vanish
    segments, hq, hkv, d = [(0, 20, 0, 700)], 8, 2, 128
    q, k, v, dout = inputs(segments, hq, hkv, d, dtype, rows=20, keys=700)
    k *= torch.arange(700, device=DEV)[:, None, None] // 100 * 2 + 0.25
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV, training=True, ctas=1)
    out, lse = torch.empty_like(q.contiguous()), torch.empty((20, hq), device=DEV)
    plan.run(q, k, v, 0.5, out, lse)
    want, wl, _ = oc.forward(segments, q, k, v, 0.5)
    bo, bl = oc.forward_bounds(segments, q, k, v, 0.5)
    within(out, want, bo)
    within(lse, wl, bl)
    dq, dk, dv = torch.empty_like(out), torch.empty_like(k.contiguous()), torch.empty_like(k.contiguous())
    plan.run_bwd(q, k, v, want.to(dtype), dout, wl.float(), 0.5, dq, dk, dv)
    for got, ref, bound in zip((dq, dk, dv), oc.backward(segments, q, k, v, dout, 0.5),
                               oc.backward_bounds(segments, q, k, v, want.to(dtype), dout, 0.5)):
        within(got, ref, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_past_32_bits(dtype):
    # the last rows of arrays of more than 2^31 elements, and the zeros of all key rows before them
    rows, stride, hq, hkv, d, scale = 36_000, 65_536, 8, 2, 128, 1 / math.sqrt(128)
    seg, near = [(rows - 20, 20, rows - 300, 300)], [(0, 20, 0, 300)]
    x = [torch.empty(rows * stride, dtype=dtype, device=DEV) for _ in range(2)]
    part = lambda b, at, h: x[b][at:].as_strided((rows, h, d), (stride, d, 1))
    q, k, v = part(0, 0, hq), part(0, hq * d, hkv), part(0, (hq + hkv) * d, hkv)
    dq, dk, dv = part(1, 0, hq), part(1, hq * d, hkv), part(1, (hq + hkv) * d, hkv)
    g = torch.Generator(device=DEV).manual_seed(5)
    nq, nk, nv, ng = (torch.randn((n, h, d), generator=g, device=DEV).to(dtype) for n, h in ((20, hq), (300, hkv), (300, hkv), (20, hq)))
    q[-20:], k[-300:], v[-300:] = nq, nk, nv
    dk.fill_(77)
    dv.fill_(77)
    out, dout = (torch.zeros((rows, hq, d), dtype=dtype, device=DEV) for _ in range(2))
    lse = torch.zeros((rows, hq), device=DEV)
    dout[-20:] = ng
    plan = CrossPlan(seg, hq, hkv, d, dtype, DEV, training=True)
    plan.run(q, k, v, scale, out, lse)
    pa.padoc_check_device_errors()
    want, wl, _ = oc.forward(near, nq, nk, nv, scale)
    bo, bl = oc.forward_bounds(near, nq, nk, nv, scale)
    within(out[-20:], want, bo)
    within(lse[-20:], wl, bl)
    out[-20:], lse[-20:] = want.to(dtype), wl.float()
    plan.run_bwd(q, k, v, out, dout, lse, scale, dq, dk, dv)
    pa.padoc_check_device_errors()
    for got, ref, bound in zip((dq[-20:], dk[-300:], dv[-300:]), oc.backward(near, nq, nk, nv, ng, scale),
                               oc.backward_bounds(near, nq, nk, nv, out[-20:], ng, scale)):
        within(got, ref, bound)
    assert not dk[:-300].any() and not dv[:-300].any()


def test_segments_without_keys_alone():
    segments = [(0, 4, 0, 0), (6, 2, 9, 0)]
    q, k, v, dout = inputs(segments, 16, 2, 128, BF16, keys=5)
    plan = CrossPlan(segments, 16, 2, 128, BF16, DEV, training=True)
    out, lse = torch.full_like(dout, 3.0), torch.full((q.shape[0], 16), 3.0, device=DEV)
    plan.run(q, k, v, 0.1, out, lse)
    assert (out[:4] == 0).all() and (out[6:8] == 0).all() and (out[4:6] == 3).all() and (out[8:] == 3).all()
    assert (lse[:4] == -math.inf).all() and (lse[4:6] == 3).all()
    dq, dk, dv = torch.full_like(dout, 3.0), torch.full_like(k.contiguous(), 3.0), torch.full_like(k.contiguous(), 3.0)
    plan.run_bwd(q, k, v, out, dout, lse, 0.1, dq, dk, dv)
    assert (dq[:4] == 0).all() and (dq[4:6] == 3).all() and (dk == 0).all() and (dv == 0).all()


def test_key_rows_behind_the_last_segment_have_zero_gradients():
    segments = [(0, 9, 3, 40)]
    q, k, v, dout = inputs(segments, 4, 2, 64, BF16, keys=400)
    plan = CrossPlan(segments, 4, 2, 64, BF16, DEV, training=True)
    out, lse = torch.zeros_like(dout), torch.zeros((q.shape[0], 4), device=DEV)
    plan.run(q, k, v, 0.125, out, lse)
    dq, dk, dv = (torch.full_like(t, 9.0) for t in (out, k.contiguous(), k.contiguous()))
    plan.run_bwd(q, k, v, out, dout, lse, 0.125, dq, dk, dv)
    for t in (dk, dv):
        assert (t[:3] == 0).all() and (t[43:] == 0).all() and (t[3:43] != 0).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nan_and_infinity_stay_with_the_rows_that_see_them(dtype):
    segments = [(0, 20, 0, 150), (20, 20, 150, 150)]
    q, k, v, dout = inputs(segments, 8, 2, 64, dtype, rows=40, keys=300)
    v[149] = math.inf
    k[140, 1] = NAN
    plan = CrossPlan(segments, 8, 2, 64, dtype, DEV, training=True)
    out, lse = torch.empty_like(dout), torch.empty((40, 8), device=DEV)
    plan.run(q, k, v, 0.125, out, lse)
    assert not torch.isfinite(out[:20]).any() and torch.isnan(out[:20, 4:]).all() and torch.isnan(lse[:20, 4:]).all()
    assert torch.isfinite(lse[:20, :4]).all()
    want, wl, _ = oc.forward(segments[1:], q, k, v, 0.125)
    bo, bl = oc.forward_bounds(segments[1:], q, k, v, 0.125)
    within(out[20:], want[20:], bo[20:])
    within(lse[20:], wl[20:], bl[20:])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_against_differences(dtype):
    # the forward's own change along a direction, in 64 bits' differences of the oracle at the same inputs
    segments, hq, hkv, d = [(0, 30, 0, 90), (30, 10, 50, 60)], 4, 2, 64
    q, k, v, dout = inputs(segments, hq, hkv, d, dtype, rows=40, keys=110)
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV, training=True)
    out, lse = torch.empty_like(dout), torch.empty((40, hq), device=DEV)
    plan.run(q, k, v, 0.125, out, lse)
    dq, dk, dv = torch.empty_like(out), torch.empty_like(k.contiguous()), torch.empty_like(k.contiguous())
    plan.run_bwd(q, k, v, out, dout, lse, 0.125, dq, dk, dv)
    bounds = oc.backward_bounds(segments, q, k, v, out, dout, 0.125)
    g = torch.Generator(device=DEV).manual_seed(5)
    for n, (got, bound) in enumerate(zip((dq, dk, dv), bounds)):
        args = [t.double() for t in (q, k, v)]
        way = torch.randn(args[n].shape, generator=g, device=DEV, dtype=torch.float64)
        ends = []
        for h in (1e-5, -1e-5):
            at = list(args)
            at[n] = args[n] + h * way
            ends.append((oc.forward(segments, *at, 0.125)[0] * dout.double()).sum().item())
        slope = (ends[0] - ends[1]) / 2e-5
        assert abs((got.double() * way).sum().item() - slope) <= (bound * way.abs()).sum().item() + 1e-6 * abs(slope) + 1e-6


@pytest.mark.parametrize("hq,hkv,d,dtype", [(16, 2, 128, BF16), (16, 16, 64, BF16), (4, 1, 64, F32)])
def test_a_training_step(hq, hkv, d, dtype):
    # forward, then the gradients with what it left; k and v, and dk and dv, as slices of fused projections
    segments = [(0, 200, 0, 150), (200, 30, 40, 60), (230, 77, 150, 301), (307, 9, 0, 0)]
    q, k, v, dout = inputs(segments, hq, hkv, d, dtype, rows=316, keys=460, wide=hkv)
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV, training=True)
    out, lse = torch.empty_like(dout), torch.empty((316, hq), device=DEV)
    scale = 1 / math.sqrt(d)
    plan.run(q, k, v, scale, out, lse)
    dq, dkv = torch.empty_like(dout), torch.empty((460, 2 * hkv, d), dtype=dtype, device=DEV)
    plan.run_bwd(q, k, v, out, dout, lse, scale, dq, dkv[:, :hkv], dkv[:, hkv:])
    pa.padoc_check_device_errors()
    off, _ = oc.forward_bounds(segments, q, k, v, scale)
    for got, want, bound in zip((dq, dkv[:, :hkv], dkv[:, hkv:]), oc.backward(segments, q, k, v, dout, scale),
                                oc.backward_bounds(segments, q, k, v, out, dout, scale, off)):
        within(got, want, bound)


@pytest.mark.parametrize("segments,hq,hkv,d", [
    ([(0, 1, 0, 961)], 16, 2, 128),                                         # a cluster
    ([(0, 24, 0, 9001)], 16, 2, 128),                                       # lists of items, joined parts
    ([(0, 3, 0, 30_000)], 4, 4, 64),                                        # few rows, joined parts
    ([(0, 700, 0, 300), (700, 40, 300, 1000)], 16, 16, 64),
    ([(0, 900, 5, 70)], 16, 2, 128)])
def test_captured_and_replayed(segments, hq, hkv, d):
    plan = CrossPlan(segments, hq, hkv, d, BF16, DEV, training=True)
    q, k, v, dout = inputs(segments, hq, hkv, d, BF16, poison=False)
    out, lse = torch.zeros_like(dout), torch.zeros(q.shape[:2], device=DEV)
    dq, dk, dv = torch.zeros_like(dout), torch.zeros_like(k), torch.zeros_like(k)

    def both():
        plan.run(q, k, v, 0.1, out, lse)
        plan.run_bwd(q, k, v, out, dout, lse, 0.1, dq, dk, dv)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
        both()
    for seed in (7, 8):
        for t, n in zip((q, k, v, dout), inputs(segments, hq, hkv, d, BF16, seed=seed, poison=False)):
            t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, dq, dk, dv)]
        both()
        pa.padoc_check_device_errors()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, dq, dk, dv)))


def test_two_streams_at_once():
    # a plan each: the workspaces are a plan's own
    segments, hq, hkv, d = [(0, 24, 0, 20_001), (24, 300, 20_001, 500)], 16, 2, 128
    sets = []
    for seed in (1, 2):
        q, k, v, dout = inputs(segments, hq, hkv, d, BF16, seed=seed, poison=False)
        sets.append((CrossPlan(segments, hq, hkv, d, BF16, DEV, training=True), torch.cuda.Stream(), q, k, v, dout,
                     torch.zeros_like(dout), torch.zeros(q.shape[:2], device=DEV), torch.zeros_like(dout),
                     torch.zeros_like(k), torch.zeros_like(k)))
    torch.cuda.synchronize()
    for _ in range(3):
        for plan, s, q, k, v, dout, out, lse, dq, dk, dv in sets:
            plan.run(q, k, v, 0.1, out, lse, stream=s)
            plan.run_bwd(q, k, v, out, dout, lse, 0.1, dq, dk, dv, stream=s)
    torch.cuda.synchronize()
    pa.padoc_check_device_errors()
    for plan, _, q, k, v, dout, *outs in sets:
        got = [t.clone() for t in outs]
        plan.run(q, k, v, 0.1, outs[0], outs[1])
        plan.run_bwd(q, k, v, outs[0], dout, outs[1], 0.1, *outs[2:])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))


def test_another_current_device_is_refused(monkeypatch):
    segments = [(0, 4, 0, 9)]
    plan = CrossPlan(segments, 4, 2, 64, BF16, DEV, training=True)
    q, k, v, dout = inputs(segments, 4, 2, 64, BF16)
    out, lse = torch.empty_like(dout), torch.empty(q.shape[:2], device=DEV)
    with monkeypatch.context() as m:
        m.setattr(pa, "_current_device", lambda: 1)   # (as if another GPU were current)
        with pytest.raises(ValueError, match="device"):
            plan.run(q, k, v, 0.1, out, lse)
        with pytest.raises(ValueError, match="device"):
            plan.run_bwd(q, k, v, out, dout, lse, 0.1, out.clone(), k.clone(), v.clone())


def test_python_refusals():
    segments = [(0, 4, 0, 9)]
    plan = CrossPlan(segments, 4, 2, 64, BF16, DEV)
    q, k, v, _ = inputs(segments, 4, 2, 64, BF16)
    out, lse = torch.empty_like(q.contiguous()), torch.empty(q.shape[:2], device=DEV)
    run = lambda **o: plan.run(**{**dict(q=q, k=k, v=v, scale=0.1, out=out, lse=lse), **o})
    run()
    with pytest.raises(ValueError):
        plan.run_bwd(q, k, v, out, out, lse, 0.1, out, k, v)
    for bad in (dict(q=q.cpu()), dict(q=q[:, :3]), dict(k=k[:, :1]), dict(v=v[:5]), dict(out=out[:3]), dict(out=out.float()),
                dict(lse=lse.double()), dict(lse=lse[:, :3]), dict(q=q.transpose(0, 1)), dict(q=q[..., :32])):
        with pytest.raises((ValueError, TypeError, pa.PadocError)):
            run(**bad)
    with pytest.raises(pa.PadocError):     # fewer rows than the plan names
        plan.run(q[:3], k, v, 0.1, out[:3], lse[:3])
    with pytest.raises(pa.PadocError):
        run(k=k[:8], v=v[:8])
    with pytest.raises(pa.PadocError):     # an output over an input
        run(out=q)
    with pytest.raises(TypeError):
        run(q=q.half(), k=k.half(), v=v.half())
