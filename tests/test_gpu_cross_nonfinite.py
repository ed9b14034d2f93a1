"""Gradients of cross attention with rows that are not finite, where segments share key tiles: what a row does not see
stays as the definition in 64 bits has it, within oracle.cross's bounds."""
import math

import pytest
import torch

from oracle import cross as oc
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import CrossPlan

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32

# a page's layout rows over all of its states, branches over crops of them, one row over a single state, rows without any
SEGMENTS = [(0, 40, 10, 300), (40, 9, 20, 30), (49, 1, 309, 1), (50, 70, 60, 190), (120, 7, 250, 200), (127, 3, 0, 0)]


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def _poison(q, dout, k, what, row, head):
    if what == "q nan":
        q[row, head] = math.nan
    elif what == "q nan in one dim":
        q[row, head, 5] = math.nan
    elif what == "q infinite":
        q[row, head, 3] = math.inf
    elif what == "scores -infinite":      # nothing is left of the row: its out is 0, its lse -inf
        k[..., 3] = -k[..., 3].abs() - 0.5
        q[row, head, 3] = math.inf
    elif what == "dout nan":
        dout[row, head] = math.nan
    elif what == "dout infinite in one dim":
        dout[row, head, 7] = -math.inf
    else:                                 # finite, of a size that leaves dV and dK finite in the bounds' own terms
        dout[row, head] *= 1024


@pytest.mark.parametrize("what", ["q nan", "q nan in one dim", "q infinite", "scores -infinite", "dout nan",
                                  "dout infinite in one dim", "dout large"])
@pytest.mark.parametrize("row", [41, 49, 60, 119, 126])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(16, 2, 128, BF16), (4, 4, 64, BF16), (7, 1, 64, BF16), (33, 1, 128, BF16),
                                            (4, 2, 64, F32), (4, 1, 128, F32)])
def test_rows_that_are_not_finite_reach_the_keys_they_see_alone(hq, hkv, d, dtype, row, what):
    g = torch.Generator(device=DEV).manual_seed(row)
    rows, keys, scale, head = 130, 470, 1 / math.sqrt(d), hq - 1
    new = lambda n, h: torch.randn((n, h, d), generator=g, device=DEV).to(dtype)   # noqa: E731
    q, k, v, dout = new(rows, hq), new(keys, hkv), new(keys, hkv), new(rows, hq)
    _poison(q, dout, k, what, row, head)
    plan = CrossPlan(SEGMENTS, hq, hkv, d, dtype, DEV, training=True)
    out, lse = torch.empty_like(q), torch.empty((rows, hq), device=DEV)
    plan.run(q, k, v, scale, out, lse)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    plan.run_bwd(q, k, v, out, dout, lse, scale, dq, dk, dv)
    pa.padoc_check_device_errors()
    want = oc.backward(SEGMENTS, q, k, v, dout, scale)
    off, _ = oc.forward_bounds(SEGMENTS, q, k, v, scale)
    bounds = oc.backward_bounds(SEGMENTS, q, k, v, out, dout, scale, off)
    first, number = [s[2:] for s in SEGMENTS if s[0] <= row < s[0] + s[1]][0]
    others = torch.ones((rows, hq), dtype=torch.bool, device=DEV)
    unseen = torch.ones((keys, hkv), dtype=torch.bool, device=DEV)
    if what != "dout large":
        others[row, head] = False
        unseen[first:first + number, -1] = False
    for got, ref, bound, held in zip((dq, dk, dv), want, bounds, (others, unseen, unseen)):
        error = (got.double() - ref).abs()[held]
        assert torch.isfinite(ref[held]).all() and (error <= bound[held]).all(), \
            f"{(~(error <= bound[held])).sum().item()} of {error.numel()} off"
    # What the definition has as not finite is not finite here. (Where every score of the row is -inf, as an infinite q
    # makes its only one when the key's value there is negative, nothing is left of it: out 0, lse -inf, no gradients.)
    if what != "dout large" and lse[row, head] != -math.inf:
        for got, ref in ((dk, want[1]), (dv, want[2])):
            assert not torch.isfinite(got[~torch.isfinite(ref)]).any()


@pytest.mark.parametrize("hq,hkv,d,dtype,segments", [
    (16, 2, 128, BF16, [(0, 1, 0, 300)]), (16, 16, 64, BF16, [(0, 3, 0, 5000)]), (16, 2, 128, BF16, [(0, 90, 0, 300)]),
    (4, 4, 64, BF16, [(0, 700, 0, 1000)]), (4, 1, 64, F32, [(0, 40, 0, 700)])])
def test_a_row_whose_scores_are_all_minus_infinity_is_a_row_without_keys(hq, hkv, d, dtype, segments):
    # one head of one row, by clusters, in joined parts, in tiles, in fp32; the others as without it
    rows, keys = segments[0][1], segments[0][3]
    g = torch.Generator(device=DEV).manual_seed(keys)
    new = lambda n, h: torch.randn((n, h, d), generator=g, device=DEV).to(dtype)   # noqa: E731
    q, k, v = new(rows, hq), new(keys, hkv), new(keys, hkv)
    k[..., 3] = -k[..., 3].abs() - 0.5
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV)
    want, wl = torch.empty_like(q), torch.empty((rows, hq), device=DEV)
    plan.run(q, k, v, 0.1, want, wl)
    row, head = rows // 2, hq - 1
    q[row, head, 3] = math.inf
    out, lse = torch.empty_like(q), torch.empty_like(wl)
    plan.run(q, k, v, 0.1, out, lse)
    pa.padoc_check_device_errors()
    assert (out[row, head] == 0).all() and lse[row, head] == -math.inf
    want[row, head], wl[row, head] = 0, -math.inf
    assert torch.equal(out, want) and torch.equal(lse, wl)
