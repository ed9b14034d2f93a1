"""Cross attention's host side: the planner against a plain count, the refusals, and the oracle itself (its gradients
against differences and autograd)."""
import ctypes
import math
import random

import numpy as np
import pytest
import torch

from oracle import cross as oc
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    pbuild.build()
    return pa.load_library()


def _units(plan, off, n):
    return plan[off:off + 8 * n].reshape(n, 8)


def _random_segments(rng):
    segments, q = [], 0
    for _ in range(rng.randint(0, 7)):
        q += rng.choice([0, 0, 1, 5])
        n = rng.choice([0, 1, 3, 17, 64, 130, 700])
        k0, kn = rng.choice([0, 0, 40, 256, 1000]), rng.choice([0, 1, 63, 64, 127, 128, 129, 300, 5000])
        segments.append((q, n, k0, kn))
        q += n
    return segments


@pytest.mark.parametrize("heads", [(16, 2), (4, 4), (7, 1), (64, 1), (12, 4)])
@pytest.mark.parametrize("seed", range(12))
def test_plan_covers_every_pair_once(heads, seed):
    rng = random.Random(100 * seed + heads[0])
    segments = _random_segments(rng)
    cfg = pa.make_cross_config(*heads, 128, rng.choice([BF16, F32]), True, rng.choice([0, 1, 10, 152]))
    plan, info = pa.padoc_build_cross_plan(segments, cfg)
    assert pa.padoc_cross_plan_size(segments, cfg) == info.plan_ints == plan.size
    live = [s for s in segments if s[1] and s[3]]
    rows = max([s[0] + s[1] for s in segments if s[1]], default=0)
    keys = max([s[2] + s[3] for s in live], default=0)
    assert (info.query_rows, info.key_rows) == (rows, keys)
    hkv = heads[1]
    want = np.zeros((rows, keys), np.int32)
    for a, n, b, m in segments:
        want[a:a + n, b:b + m] += 1
    assert info.pairs == want.sum()
    assert want.max(initial=0) <= 1
    empty = np.zeros(rows, bool)
    for a, n, _, m in segments:
        if m == 0:
            empty[a:a + n] = True
    block = 64 // (heads[0] // hkv)
    assert info.unit_rows in (16, 32, 256) and info.few in (0, 1, 2, 4, 8)
    # statistics: each block of rows that sees keys has one place
    place = {}
    for a, n, _, m in live:
        for t in range(0, n, block):
            place[a + t] = len(place)
    assert info.num_subs == len(place)
    for off, n, coff, ctas, moff, mn, slots, most, blocks, dq in (
            (info.off_units, info.num_units, info.off_ctas, info.num_ctas, info.off_merges, info.num_merges, info.num_slots,
             info.max_parts, 4 * block if info.unit_rows == 256 else info.unit_rows // (heads[0] // hkv), False),
            (info.off_dq_units, info.num_dq_units, info.off_dq_ctas, info.num_dq_ctas, info.off_dq_merges,
             info.num_dq_merges, info.num_dq_slots, info.max_dq_parts, 2 * block, True)):
        got, written = np.zeros((hkv,) + want.shape, np.int32), np.zeros((hkv, rows), np.int32)
        parts, seen = {}, set()
        units = _units(plan, off, n)
        for tok, nt, k0, nk, g, slot, sub, _ in units:
            assert 1 <= nt <= blocks and 1 <= nk and 0 <= g < hkv
            got[g, tok:tok + nt, k0:k0 + nk] += 1
            if slot >= 0:
                assert slot not in parts
                parts[slot] = (tok, nt, g, k0, nk)
            else:
                written[g, tok:tok + nt] += 1
            if dq and sub >= 0:
                for i, t in enumerate(range(0, nt, block)):
                    assert place[tok + t] == sub + i
                    assert (g, sub + i) not in seen
                    seen.add((g, sub + i))
        assert (got == want).all()
        assert not dq or len(seen) == hkv * len(place)
        assert sorted(parts) == list(range(slots))
        if ctas:     # a list for each CTA, none empty
            ends = plan[coff:coff + ctas + 1]
            assert ends[0] == 0 and ends[-1] == n and (np.diff(ends) > 0).all()
            assert ctas <= max(1, cfg.ctas or 152)
        else:
            assert (np.diff(units[:, 3]) <= 0).all()
        top = 0
        for tok, nt, slot, np_, g in plan[moff:moff + 8 * mn].reshape(mn, 8)[:, :5]:
            written[g, tok:tok + nt] += 1
            assert np_ == 0 or np_ > 1
            top = max(top, np_)
            end = None
            for p in range(slot, slot + np_):     # the parts in the keys' order, one behind the other
                assert parts[p][:3] == (tok, nt, g) and (end is None or parts[p][3] == end)
                end = parts[p][3] + parts[p][4]
            if np_ == 0:
                assert empty[tok:tok + nt].all()
        assert top == most
        assert (written == (want.sum(1) > 0) + empty.astype(np.int32)).all()
    # key tiles: every key once, each segment's keys of it
    got, tiled = np.zeros((rows, keys), np.int32), np.zeros(keys, np.int32)
    covers = _units(plan, info.off_covers, info.num_covers)
    last = 1 << 30
    for k0, nk, c0, nc, steps, _, _, _ in _units(plan, info.off_key_tiles, info.num_key_tiles):
        assert 1 <= nk <= 128 and steps <= last
        last = steps
        tiled[k0:k0 + nk] += 1
        mine = covers[c0:c0 + nc]
        assert steps == sum(-(-c[1] // block) for c in mine) == sum(c[3] for c in mine)
        assert (np.diff(mine[:, 0]) > 0).all()
        for tok, nt, sub, nsub, ck, cn, _, _ in mine:
            assert cn >= 1 and k0 <= ck and ck + cn <= k0 + nk and sub == place[tok]
            got[tok:tok + nt, ck:ck + cn] += 1
    assert (tiled == 1).all() and (got == want).all()
    gaps = [t for t in _units(plan, info.off_key_tiles, info.num_key_tiles) if t[4] == 0]
    assert len(gaps) == info.num_gap_tiles
    if cfg.dtype == pa.PADOC_DTYPE_F32:
        assert info.cluster in (1, 2, 4, 8) and info.num_dkv_units == 0
        return
    # dk/dv items: every step of every tile and KV head once, parts joined in the steps' order
    tiles = {(int(t[0]), int(t[1])): t for t in _units(plan, info.off_key_tiles, info.num_key_tiles) if t[4]}
    items = _units(plan, info.off_dkv, info.num_dkv_units)
    ends = plan[info.off_dkv_ctas:info.off_dkv_ctas + info.num_dkv_ctas + 1] if info.num_dkv_ctas else np.zeros(1, np.int32)
    assert ends[0] == 0 and ends[-1] == info.num_dkv_units and (np.diff(ends) > 0).all()
    assert info.num_dkv_ctas <= max(1, cfg.ctas or 152)
    done, parts = {}, {}
    for k0, nk, cover, first, steps, g, slot, _ in items:
        t = tiles[int(k0), int(nk)]
        assert cover == t[2] and steps >= 1 and 0 <= first and first + steps <= t[4]
        done.setdefault((k0, g), []).append((first, steps))
        if slot >= 0:
            assert slot not in parts
            parts[slot] = (k0, nk, g, first)
        else:
            assert steps == t[4]
    assert len(done) == len(tiles) * hkv
    for (k0, g), runs in done.items():
        at = 0
        for first, steps in sorted(runs):
            assert first == at
            at += steps
        assert at == [t for t in tiles.values() if t[0] == k0][0][4]
    assert sorted(parts) == list(range(info.num_dkv_slots))
    joined = 0
    for k0, nk, g, slot, n in _units(plan, info.off_dkv_sums, info.num_dkv_sums)[:, :5]:
        assert n == len(done[k0, g]) > 1
        mine = [parts[p] for p in range(slot, slot + n)]
        assert all(m[:3] == (k0, nk, g) for m in mine) and [m[3] for m in mine] == sorted(m[3] for m in mine)
        joined += n
    assert joined == info.num_dkv_slots


def test_few_rows_are_split_over_the_chip():
    cfg = pa.make_cross_config(16, 2, 128, BF16, False, 152)
    _, one = pa.padoc_build_cross_plan([(0, 1, 0, 961)], cfg)
    _, document = pa.padoc_build_cross_plan([(0, 24, 0, 150_001)], cfg)
    _, packed = pa.padoc_build_cross_plan([(4096 * i, 4096, 2560 * i, 2560) for i in range(8)], cfg)
    assert one.few == 8 and one.num_slots == 0 and document.num_slots >= 140 and packed.num_units == 2048
    assert pa.padoc_cross_workspace_size(document) > 0


def test_plan_refusals(lib):
    good = dict(num_q_heads=16, num_kv_heads=2, head_dim=128, dtype=BF16)
    cfg = lambda **k: pa.make_cross_config(**{**good, **k})

    def status(segments, c):
        with pytest.raises(pa.PadocError) as e:
            pa.padoc_build_cross_plan(segments, c)
        return e.value.status
    seg = [(0, 4, 0, 9)]
    assert status([(4, 4, 0, 9), (0, 4, 0, 9)], cfg()) == 1          # out of order
    assert status([(0, 4, 0, 9), (3, 4, 0, 9)], cfg()) == 1          # a row in two segments
    assert status([(2 ** 31 - 1000, 10, 0, 9)], cfg()) == 1          # past the rows' range
    assert status([(0, 4, 2 ** 31 - 1000, 10)], cfg()) == 1
    assert status([(0, 4, 2 ** 30, 10)], cfg(backward=True)) == 2
    assert status([(0, 2 ** 30, 0, 10)], cfg()) == 2
    for bad in (dict(num_q_heads=0), dict(num_kv_heads=0), dict(num_q_heads=15), dict(ctas=-1), dict(ctas=65536)):
        assert status(seg, cfg(**bad)) == 1
    for bad in (dict(head_dim=96), dict(num_q_heads=130), dict(dtype=7)):
        assert status(seg, cfg(**bad)) == 2
    with pytest.raises(ValueError):
        pa.padoc_build_cross_plan([(-1, 4, 0, 9)], cfg())
    with pytest.raises(TypeError):
        cfg(dtype=torch.float16)
    n = ctypes.c_int64()
    info = pa.padoc_cross_plan()
    buf = np.zeros(8, np.int32)
    s = np.array(seg, np.int32)
    p = buf.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    c = ctypes.byref(cfg())
    assert lib.padoc_cross_plan_size(s.ctypes.data, 1, c, None) == 1
    assert lib.padoc_cross_plan_size(None, 1, c, ctypes.byref(n)) == 1
    assert lib.padoc_build_cross_plan(s.ctypes.data, 1, c, p, 8, ctypes.byref(info)) == 6 and info.plan_ints > 8
    assert lib.padoc_build_cross_plan(s.ctypes.data, 1, c, None, 0, ctypes.byref(info)) == 6
    assert lib.padoc_build_cross_plan(s.ctypes.data, 1, c, p, 8, None) == 1
    with pytest.raises(pa.PadocError):   # no backward in this plan
        pa.padoc_cross_bwd_workspace_size(pa.padoc_build_cross_plan(seg, cfg())[1])


@pytest.mark.skipif(torch.cuda.is_available(), reason="stand-in addresses are for machines without a GPU")
def test_calls_are_refused_before_any_launch(lib):
    A = 1 << 20
    # one token, split: the call needs a workspace
    plan, info = pa.padoc_build_cross_plan([(0, 1, 0, 961)], pa.make_cross_config(16, 2, 128, F32, True, 152))
    need, bneed = pa.padoc_cross_workspace_size(info), pa.padoc_cross_bwd_workspace_size(info)

    def fwd(i=info, plan=A, q=A, k=4 * A, v=5 * A, qs=2048, ks=256, vs=256, qn=1, kn=961, scale=0.1, out=2 * A, lse=3 * A, ws=64 * A,
            n=need):
        rows = pa.padoc_cross_rows(q, k, v, qs, ks, vs, qn, kn)
        return lib.padoc_cross_attn(ctypes.byref(i) if i else None, plan, ctypes.byref(rows), scale, out, lse, ws, n, None)

    def bwd(i=info, q=A, k=4 * A, v=5 * A, kn=961, out=2 * A, dout=6 * A, lse=3 * A, dq=7 * A, dk=8 * A, dv=9 * A, dqs=2048,
            dks=256, dvs=256, ws=64 * A, n=bneed):
        rows = pa.padoc_cross_rows(q, k, v, 2048, 256, 256, 1, kn)
        grads = pa.padoc_cross_grads(dq, dk, dv, dqs, dks, dvs)
        return lib.padoc_cross_attn_bwd(ctypes.byref(i), A, ctypes.byref(rows), out, dout, lse, 0.1, ctypes.byref(grads), ws, n, None)

    assert fwd(i=None) == 1 and fwd(plan=None) == 1 and fwd(plan=A + 4) == 1
    for name in ("q", "k", "v", "out", "lse"):
        assert fwd(**{name: None}) == 1
        assert fwd(**{name: A + 2}) == 1
    assert fwd(qs=2040) == 1 and fwd(qs=2050) == 1 and fwd(ks=128) == 1 and fwd(vs=0) == 1 and fwd(ks=-256) == 1
    assert fwd(qn=0) == 1 and fwd(kn=960) == 1 and fwd(kn=2 ** 31) == 1
    assert fwd(qs=2 ** 62) == 1 and fwd(ks=2 ** 37, kn=2 ** 30) == 1 and bwd(dqs=2 ** 62) == 1 and bwd(dvs=2 ** 37, kn=2 ** 30) == 1
    assert fwd(scale=0.0) == 1 and fwd(scale=math.nan) == 1 and fwd(scale=math.inf) == 1
    assert fwd(ws=None) == 1 and fwd(ws=64 * A + 16) == 1 and fwd(n=need - 1) == 3
    assert fwd(out=A) == 1 and fwd(out=4 * A + 512 * 960) == 1 and fwd(lse=5 * A) == 1 and fwd(lse=2 * A) == 1   # overlaps
    for name in ("q", "k", "v", "out", "dout", "lse", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == 1
        assert bwd(**{name: A + 2}) == 1
    assert bwd(dqs=2040) == 1 and bwd(dks=128) == 1 and bwd(dvs=258) == 1 and bwd(kn=960) == 1
    assert bwd(ws=None) == 1 and bwd(n=bneed - 1) == 3
    assert bwd(dk=9 * A) == 1 and bwd(dv=8 * A + 512 * 500) == 1 and bwd(dq=A) == 1 and bwd(dk=4 * A) == 1 and bwd(dq=6 * A) == 1
    # side by side in one buffer: not an overlap, but rows reaching into the neighbour's are
    assert bwd(dk=8 * A, dv=8 * A + 256, dks=512, dvs=512) == 1
    no = pa.padoc_build_cross_plan([(0, 1, 0, 961)], pa.make_cross_config(16, 2, 128, BF16, False, 152))[1]
    assert bwd(i=no) == 1
    nothing = pa.padoc_build_cross_plan([], pa.make_cross_config(16, 2, 128, BF16, True))[1]
    assert fwd(i=nothing) == 0 and bwd(i=nothing, kn=0) == 0     # nothing to do


def test_the_oracle():
    g = torch.Generator().manual_seed(1)
    segments = [(0, 3, 2, 5), (3, 2, 0, 0), (6, 4, 4, 6), (10, 1, 0, 1)]
    q = torch.randn(12, 4, 8, generator=g, dtype=torch.float64)
    k, v = (torch.randn(11, 2, 8, generator=g, dtype=torch.float64) for _ in range(2))
    dout = torch.randn(12, 4, 8, generator=g, dtype=torch.float64)
    out, lse, rows = oc.forward(segments, q, k, v, 0.3)
    assert rows.tolist() == [i != 5 and i != 11 for i in range(12)]
    # a row written out by hand
    s = [0.3 * float(q[7, 3] @ k[j, 1]) for j in range(4, 10)]
    w = [math.exp(x) for x in s]
    assert abs(float(lse[7, 3]) - math.log(sum(w))) < 1e-12
    assert torch.allclose(out[7, 3], sum(x * v[4 + j, 1] for j, x in enumerate(w)) / sum(w), atol=1e-12)
    assert (out[3:5] == 0).all() and (lse[3:5] == -math.inf).all()
    grads = oc.backward(segments, q, k, v, dout, 0.3)
    for n, (x, got) in enumerate(zip((q, k, v), grads)):
        for at in ((0, 0, 0), (3, 1, 4), (7, 1, 2), (10, 0, 5)):
            d = []
            for h in (1e-6, -1e-6):
                y = x.clone()
                y[at] += h
                args = [q, k, v]
                args[n] = y
                d.append(float((oc.forward(segments, *args, 0.3)[0] * dout).sum()))
            assert abs((d[0] - d[1]) / 2e-6 - float(got[at])) < 1e-7
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    total = 0
    for a, n, b, m in segments:
        if m:
            kk, vv = (t[b:b + m].repeat_interleave(2, 1) for t in leaves[1:])
            p = torch.softmax(0.3 * torch.einsum("ihd,jhd->hij", leaves[0][a:a + n], kk), -1)
            total = total + (torch.einsum("hij,jhd->ihd", p, vv) * dout[a:a + n]).sum()
    for got, want in zip(grads, torch.autograd.grad(total, leaves)):
        assert torch.allclose(got, want, atol=1e-12)
