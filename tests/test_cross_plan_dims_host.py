"""The cross-attention planner with heads of 64 dims beside those of 128 (other items, lists and costs): every visible pair
in one item, every row written once, parts joined in the keys' order, key tiles and their steps each once."""
import random

import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa

from .test_cross_host import _random_segments

BF16, F32 = torch.bfloat16, torch.float32
SMS = 152


@pytest.fixture(scope="module", autouse=True)
def lib():
    pbuild.build()
    return pa.load_library()


def _records(plan, off, n):
    return plan[off:off + 8 * n].reshape(n, 8)


def _check_items(plan, info, dq, per, lists, want, empty, hkv):
    """The items of the forward, or of the dq pass, and what joins their parts."""
    off, n, coff, ctas, moff, mn, slots, most = (
        (info.off_dq_units, info.num_dq_units, info.off_dq_ctas, info.num_dq_ctas, info.off_dq_merges, info.num_dq_merges,
         info.num_dq_slots, info.max_dq_parts) if dq else
        (info.off_units, info.num_units, info.off_ctas, info.num_ctas, info.off_merges, info.num_merges, info.num_slots,
         info.max_parts))
    pairs, written = np.zeros((hkv,) + want.shape, np.int32), np.zeros((hkv, want.shape[0]), np.int32)
    parts = {}
    for tok, nt, k0, nk, g, slot, _, _ in _records(plan, off, n):
        assert 1 <= nt <= per and nk >= 1
        pairs[g, tok:tok + nt, k0:k0 + nk] += 1
        if slot < 0:
            written[g, tok:tok + nt] += 1
        else:
            assert slot not in parts
            parts[int(slot)] = (tok, nt, g, k0, nk)
    assert (pairs == want).all() and sorted(parts) == list(range(slots))
    if ctas:
        ends = plan[coff:coff + ctas + 1]
        assert ends[0] == 0 and ends[-1] == n and (np.diff(ends) > 0).all() and ctas <= lists
    else:
        assert (np.diff(_records(plan, off, n)[:, 3]) <= 0).all()     # longest first
    joined = []
    for tok, nt, slot, count, g in _records(plan, moff, mn)[:, :5]:
        assert 1 <= nt <= per
        written[g, tok:tok + nt] += 1
        joined.append(int(count))
        mine = [parts[p] for p in range(slot, slot + count)]
        assert count != 1 and all(m[:3] == (tok, nt, g) for m in mine)
        assert all(a[3] + a[4] == b[3] for a, b in zip(mine, mine[1:]))
        if count == 0:
            assert empty[tok:tok + nt].all()
    assert max(joined, default=0) == most and sum(joined) == slots
    assert (written == (want.any(1) | empty)).all()


def _check(heads, d, dtype, segments, ctas):
    hq, hkv = heads
    cfg = pa.make_cross_config(hq, hkv, d, dtype, True, ctas)
    plan, info = pa.padoc_build_cross_plan(segments, cfg)
    assert pa.padoc_cross_plan_size(segments, cfg) == info.plan_ints == plan.size
    rows = max([s[0] + s[1] for s in segments if s[1]], default=0)
    keys = max([s[2] + s[3] for s in segments if s[1] and s[3]], default=0)
    assert (info.query_rows, info.key_rows) == (rows, keys)
    want, empty = np.zeros((rows, keys), np.int32), np.zeros(rows, bool)
    for a, n, b, m in segments:
        want[a:a + n, b:b + m] += 1
        empty[a:a + n] |= m == 0
    want = want.astype(bool)
    group, lanes = hq // hkv, ctas or SMS
    block, an_sm = 64 // group, 2 if d == 64 and dtype == BF16 else 1
    assert info.unit_rows in (16, 32, 256 // an_sm)
    assert info.few in (0, 1, 2, 4, 8) and (info.unit_rows < 64) == (info.few > 0)
    per = info.unit_rows // group if info.few else 4 // an_sm * block
    _check_items(plan, info, False, per, an_sm * lanes, want, empty, hkv)
    _check_items(plan, info, True, 2 * block, lanes, want, empty, hkv)
    # key tiles, and with bf16 the items that walk their steps
    tiles = _records(plan, info.off_key_tiles, info.num_key_tiles)
    seen, tiled = np.zeros((rows, keys), np.int32), np.zeros(keys, np.int32)
    covers = _records(plan, info.off_covers, info.num_covers)
    for k0, nk, c0, nc, steps, _, _, _ in tiles:
        tiled[k0:k0 + nk] += 1
        assert steps == sum(-(-int(c[1]) // block) for c in covers[c0:c0 + nc])
        for tok, nt, _, nsub, ck, cn, _, _ in covers[c0:c0 + nc]:
            assert nsub == -(-nt // block) and k0 <= ck and ck + cn <= k0 + nk
            seen[tok:tok + nt, ck:ck + cn] += 1
    assert (tiled == 1).all() and (seen == want).all()
    if dtype == F32:
        return info
    steps = {int(t[0]): int(t[4]) for t in tiles if t[4]}
    done, slots = {}, set()
    for k0, _, _, first, number, g, slot, _ in _records(plan, info.off_dkv, info.num_dkv_units):
        done.setdefault((int(k0), int(g)), []).append((int(first), int(number)))
        if slot >= 0:
            assert slot not in slots
            slots.add(int(slot))
    assert len(done) == hkv * len(steps) and slots == set(range(info.num_dkv_slots))
    for (k0, _), runs in done.items():
        runs.sort()
        assert runs[0][0] == 0 and all(a + n == b for (a, n), (b, _) in zip(runs, runs[1:])) and sum(runs[-1]) == steps[k0]
    assert info.num_dkv_ctas <= lanes
    sums = _records(plan, info.off_dkv_sums, info.num_dkv_sums)
    assert sorted(len(r) for r in done.values() if len(r) > 1) == sorted(int(s[4]) for s in sums)
    return info


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(16, 16), (16, 2), (7, 1), (40, 1), (64, 1), (12, 4)])
@pytest.mark.parametrize("seed", range(10))
def test_every_pair_row_and_tile_once(heads, d, seed):
    rng = random.Random(1000 * seed + heads[0] + d)
    _check(heads, d, rng.choice([BF16, BF16, F32]), _random_segments(rng), rng.choice([0, 0, 1, 10, SMS]))


def test_heads_of_64_dims_take_every_kind_of_plan():
    kinds = set()
    for segments, ctas in (([(0, 900, 0, 700)], 0), ([(0, 2300, 0, 300)], 7), ([(0, 40, 0, 9000), (40, 3, 5, 0)], 0),
                           ([(0, 1, 0, 900)], 0), ([(i, 1, 20 * i, 200) for i in range(40)], 0), ([(0, 3, 0, 20_000)], 0),
                           ([(17 * i, 17, 200 * i, 200) for i in range(40)], 0)):
        info = _check((16, 16), 64, BF16, segments, ctas)
        kinds.add((info.unit_rows, info.num_ctas > 0, info.num_slots > 0))
    assert {k[0] for k in kinds} == {16, 32, 128} and {(128, False), (128, True)} <= {k[:2] for k in kinds}
    assert any(k[2] for k in kinds) and not all(k[2] for k in kinds), kinds
