"""A decoding step whose streams each see a crop of their page's states: many segments of one row, so that an item's tiles
hold a token or none, in both kernels that may take them. Tolerances are oracle.cross's bounds."""
import math
import random

import pytest
import torch

from oracle import cross as oc
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.engine import CrossPlan

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def _crops(streams, shortest, longest, seed):
    rng = random.Random(seed)
    return [(i, 1, 4096 * (i // 21) + rng.randint(0, 2000), rng.randint(shortest, longest)) for i in range(streams)]


def _check(segments, hq, hkv, d, dtype):
    rows, keys, scale = segments[-1][0] + 1, max(s[2] + s[3] for s in segments), 1 / math.sqrt(d)
    g = torch.Generator(device=DEV).manual_seed(rows)
    q = torch.randn((rows, hq, d), generator=g, device=DEV).to(dtype)
    k, v = (torch.randn((keys, hkv, d), generator=g, device=DEV).to(dtype) for _ in range(2))
    plan = CrossPlan(segments, hq, hkv, d, dtype, DEV)
    out, lse = torch.full_like(q, 77.0), torch.full((rows, hq), 77.0, device=DEV)
    plan.workspace.fill_(255)
    plan.run(q, k, v, scale, out, lse)
    pa.padoc_check_device_errors()
    want, wl, _ = oc.forward(segments, q, k, v, scale)
    bo, bl = oc.forward_bounds(segments, q, k, v, scale)
    assert ((out.double() - want).abs() <= bo).all() and ((lse.double() - wl).abs() <= bl).all()
    return plan.info


@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (8, 8, 128), (16, 16, 64)])
@pytest.mark.parametrize("streams,shortest,longest", [(160, 60, 200), (160, 300, 1200), (330, 800, 1200)])
def test_streams_over_crops(hq, hkv, d, streams, shortest, longest):
    _check(_crops(streams, shortest, longest, streams + hq), hq, hkv, d, BF16)


def test_streams_over_crops_in_fp32():
    _check(_crops(90, 60, 700, 1), 4, 1, 64, F32)


def test_tiles_of_one_token_in_items_of_256_rows():
    # a segment of many rows among them rules out the kernel for few rows: the other items are a token each
    segments = [(i, 1, 40 * i, 100 + i) for i in range(60)] + [(60, 3000, 0, 900)] + [(3060 + i, 1, 30 * i, 333) for i in range(60)]
    info = _check(segments, 8, 8, 128, BF16)
    assert info.few == 0 and info.unit_rows == 256
    info = _check(segments, 8, 8, 64, BF16)
    assert info.few == 0 and info.unit_rows == 128
