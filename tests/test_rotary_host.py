"""CPU tests of the rotary calls' host side (the table, the positions, refusals) and of the scheduler's
forks with history, drops, compaction and resizing, against plain models."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import rotary as orot
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa
from paper_2608_06146_gb300.inputs import PageSpec

BS = 16
# pi to 50 digits, for angles without a rounding
PI = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


@pytest.fixture(scope="module", autouse=True)
def lib():
    pbuild.build()
    return pa.load_library()


# ------------------------------------------------------------------------------------------------
# Oracle pins
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_oracle_backward_against_differences(adjacent, norm):
    rng = np.random.default_rng(4)
    x, dz = rng.standard_normal((3, 2, 16)), rng.standard_normal((3, 2, 16))
    w = rng.standard_normal(16) if norm else None
    ang = rng.standard_normal((3, 4)) * 3
    f = lambda x, w: (orot.forward(x, w, 1e-3, ang, adjacent, 1.25)[0] * dz).sum()
    dx, _, dw, _ = orot.backward(dz, x, w, 1e-3, ang, adjacent, 1.25)
    # central differences with step 1e-5: truncation 1e-10 x third derivative, rounding 1e-16 / 1e-5 x |f|
    h = 1e-5
    for at in [(0, 0, 0), (1, 1, 5), (2, 0, 7), (2, 1, 15)]:
        e = np.zeros_like(x)
        e[at] = h
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[at]) < 1e-7
    if norm:
        for j in (0, 6, 15):
            e = np.zeros(16)
            e[j] = h
            assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[j]) < 1e-7


# ------------------------------------------------------------------------------------------------
# Table and positions
# ------------------------------------------------------------------------------------------------

def test_table_turns_far_positions_exactly():
    inv = [1.0, 0.5 ** 0.25, 1e-3, 5e6 ** (-63 / 64), 7.25, -0.3, 0.0]
    table = pa.padoc_build_rotary_table(inv, [0, 1, 2, 0, 1, 2, 0], 3)
    for p in (0, 1, -1, 12345, 1_000_003, -(2 ** 24), 2 ** 31 - 1, -2 ** 31):
        for f, entry, axis in zip(inv, table.tolist(), (0, 1, 2, 0, 1, 2, 0)):
            assert entry & 3 == axis
            turns = Fraction((entry & ~3) * p % 2 ** 64, 2 ** 64)
            want = Fraction(f) * p / (2 * PI) % 1
            off = abs(turns - want)
            # f / 2 pi in fp64: two roundings (the quotient and 2 pi), 2^-53 each, relative; the 62-bit
            # fraction: half of 2^-62 (and 2^-53 where the fraction is near a whole turn, of a negative f)
            bound = abs(p) * (2 * abs(f) / 6.28 * 2.0 ** -53 + 2.0 ** -63 + (2.0 ** -53 if f < 0 or f > 6 else 0))
            assert min(off, 1 - off) <= bound


def test_table_refusals():
    for args in (([1.0], None, 2), ([float("inf")], None, 1), ([float("nan")], None, 1), ([1.0], [1], 1),
                 ([1.0], [-1], 2), ([1.0], None, 0), ([1.0], [0], 5), ([], None, 1)):
        with pytest.raises(pa.PadocError) as e:
            pa.padoc_build_rotary_table(*args)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        pa.padoc_build_rotary_table([1.0, 2.0], [0], 1)


def _positions(pages, grids):
    pos, ends = [], []
    for i, pg in enumerate(pages):
        by = {g[1]: g[2:] for g in grids if g[0] == i}
        p = q = 0
        while q < pg.prefix_len:
            if q in by:
                t, h, w = by[q]
                pos += [(p + a, p + b, p + c) for a in range(t) for b in range(h) for c in range(w)]
                q, p = q + t * h * w, p + max(t, h, w)
            else:
                pos.append((p,) * 3)
                q, p = q + 1, p + 1
        ends.append(p)
        pos += [(p + j,) * 3 for j in range(pg.layout_len)]
        pos += [(p + f + j,) * 3 for f, n in zip(pg.fork_offset, pg.branch_len) for j in range(n)]
    return np.array(pos, np.int32).reshape(-1, 3), ends


def test_positions_of_pages_with_grids():
    pages = [PageSpec(40, 5, [0, 3, 5], [4, 1, 7]), PageSpec(0, 2, [1], [3]), PageSpec(24, 0, [0], [2]), PageSpec(9, 0)]
    for grids in ([], [(0, 2, 1, 4, 6), (0, 26, 2, 3, 2), (2, 0, 1, 4, 6)], [(0, 0, 10, 2, 2)], [(3, 8, 1, 1, 1)],
                  [(0, 0, 1, 1, 40), (2, 23, 1, 1, 1)]):
        pos, end = pa.padoc_build_rotary_positions(pages, grids)
        want, want_end = _positions(pages, grids)
        np.testing.assert_array_equal(pos, want)
        assert end.tolist() == want_end


@pytest.mark.parametrize("grids", [[(0, 0, 1, 7, 6)], [(0, -1, 1, 1, 1)], [(4, 0, 1, 1, 1)], [(0, 0, 0, 1, 1)],
                                   [(0, 0, 1, 2, 2), (0, 3, 1, 1, 1)], [(2, 0, 1, 1, 1), (0, 0, 1, 1, 1)],
                                   [(0, 0, 2 ** 30, 2 ** 30, 16)], [(0, 41, 1, 1, 1)], [(0, 40, 1, 1, 1)],
                                   [(1, 0, 1, 1, 1)], [(-1, 0, 1, 1, 1)]])
def test_positions_refuse_bad_grids(grids):
    pages = [PageSpec(40, 5, [0], [4]), PageSpec(0, 2, [1], [3]), PageSpec(24, 0, [0], [2])]
    with pytest.raises(pa.PadocError) as e:
        pa.padoc_build_rotary_positions(pages, grids)
    assert e.value.status == 1


# ------------------------------------------------------------------------------------------------
# Refusals of the device calls (stand-in addresses: nothing here reaches a launch)
# ------------------------------------------------------------------------------------------------

A, MIS = 1 << 20, (1 << 20) + 8
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="stand-in addresses are for machines without a GPU")
BF16, F32 = pa.PADOC_DTYPE_BF16, pa.PADOC_DTYPE_F32


def _rot(freq=A, qw=None, kw=None, d=128, rot=128, axes=3, adjacent=0, eps=1e-6, amp=1.0):
    return pa.padoc_rotary(freq, qw, kw, d, rot, axes, adjacent, eps, amp)


def _rows(q=A, k=A, v=A, qs=2048, ks=256, vs=256, pos=A, rows=10, hq=16, hkv=2, dtype=BF16):
    return pa.padoc_qkv_rows(q, k, v, qs, ks, vs, pos, rows, hq, hkv, dtype)


BAD_SPECS = [(dict(freq=None), 1), (dict(freq=A + 4), 1), (dict(axes=0), 1), (dict(axes=5), 1), (dict(adjacent=2), 1),
             (dict(amp=float("nan")), 1), (dict(amp=float("inf")), 1), (dict(qw=A), 1), (dict(kw=A), 1),
             (dict(qw=A, kw=MIS), 1), (dict(qw=A, kw=A, eps=-1.0), 1), (dict(qw=A, kw=A, eps=float("nan")), 1),
             (dict(rot=136), 1), (dict(rot=0), 1), (dict(d=0), 1), (dict(d=264, rot=64), 2), (dict(rot=12), 2),
             (dict(d=100, rot=64), 2)]
BAD_ROWS = [(dict(rows=-1), 1), (dict(hkv=0), 1), (dict(hq=0), 1), (dict(dtype=5), 1), (dict(pos=None), 1),
            (dict(pos=A + 2), 1), (dict(q=MIS), 1), (dict(k=None), 1), (dict(qs=2047), 1), (dict(qs=2052), 1),
            (dict(ks=255), 1), (dict(ks=-256), 1), (dict(qs=1 << 62), 1), (dict(rows=1 << 31), 2)]


@no_gpu
def test_qk_rotary_refusals(lib):
    def call(spec=None, rows=None, qo=A, qos=2048, ko=A, kos=256):
        s, r = spec or _rot(), rows or _rows()
        return lib.padoc_qk_rotary(ctypes.byref(s), ctypes.byref(r), qo, qos, ko, kos, None)
    assert lib.padoc_qk_rotary(None, ctypes.byref(_rows()), A, 2048, A, 256, None) == 1
    assert lib.padoc_qk_rotary(ctypes.byref(_rot()), None, A, 2048, A, 256, None) == 1
    for kw, st in BAD_SPECS:
        assert call(spec=_rot(**kw)) == st, kw
    for kw, st in BAD_ROWS:
        assert call(rows=_rows(**kw)) == st, kw
    assert call(rows=_rows(q=None)) == 1
    assert call(qo=None) == 1 and call(ko=MIS) == 1 and call(qos=2040) == 1 and call(kos=260) == 1
    assert call(rows=_rows(rows=0)) == 0


@no_gpu
def test_qk_rotary_bwd_refusals(lib):
    norm = dict(qw=A, kw=A)

    def call(spec, rows=None, dqo=A, dko=A, dq=A, dk=A, dqw=A, dkw=A, ws=A, wsb=1 << 20, s=256):
        r = rows or _rows()
        return lib.padoc_qk_rotary_bwd(ctypes.byref(spec), ctypes.byref(r), dqo, 2048, dko, 256, dq, 2048, dk, s, dqw,
                                       dkw, ws, wsb, None)
    for kw, st in BAD_SPECS:
        assert call(_rot(**kw)) == st, kw
    for kw, st in BAD_ROWS:
        assert call(_rot(**norm), rows=_rows(**kw)) == st, kw
    spec = _rot(**norm)
    assert call(spec, dqw=None) == 1 and call(spec, dkw=A + 2) == 1 and call(spec, rows=_rows(q=None)) == 1
    assert call(spec, dqo=None) == 1 and call(spec, dko=MIS) == 1 and call(spec, dq=None) == 1 and call(spec, s=248) == 1
    assert call(spec, ws=None) == 1 and call(spec, ws=A + 16) == 1
    need = ctypes.c_size_t()
    assert lib.padoc_qk_rotary_bwd_workspace_size(ctypes.byref(spec), 10, ctypes.byref(need)) == 0 and need.value > 0
    assert call(spec, wsb=need.value - 1) == 3
    assert lib.padoc_qk_rotary_bwd_workspace_size(ctypes.byref(_rot()), 10, ctypes.byref(need)) == 0 and need.value == 0
    assert lib.padoc_qk_rotary_bwd_workspace_size(ctypes.byref(spec), -1, ctypes.byref(need)) == 1
    assert lib.padoc_qk_rotary_bwd_workspace_size(ctypes.byref(spec), 1 << 31, ctypes.byref(need)) == 2
    assert lib.padoc_qk_rotary_bwd_workspace_size(ctypes.byref(spec), 10, None) == 1
    # the rotation alone needs no rows, weights or workspace
    assert call(_rot(), rows=_rows(q=None, k=None, rows=0), dqw=None, dkw=None, ws=None, wsb=0) == 0
    assert call(_rot(), rows=_rows(q=None, k=None), dko=None, dqw=None) == 1


@no_gpu
def test_append_rotary_refusals(lib):
    def pool(k=A, v=A, nb=64, bs=16, hkv=2, d=128, dtype=BF16):
        return pa.padoc_kv_pool(k, v, nb, bs, hkv, d, dtype)

    def pool8(k=A, v=A, ks=A, vs=A, nb=64, bs=16, hkv=2, d=128):
        return pa.padoc_kv_pool_e4m3(k, v, ks, vs, nb, bs, hkv, d)

    for name, mk in (("padoc_append_rotary_inputs", pool), ("padoc_append_rotary_inputs_e4m3", pool8)):
        def call(p=None, spec=None, rows=None, qd=A, slots=A, count=4):
            p, s, r = p or mk(), spec or _rot(), rows or _rows()
            return getattr(lib, name)(ctypes.byref(p), ctypes.byref(s), ctypes.byref(r), qd, None, slots, count, None)
        assert getattr(lib, name)(None, ctypes.byref(_rot()), ctypes.byref(_rows()), A, None, A, 4, None) == 1
        for kw, st in BAD_SPECS:
            assert call(spec=_rot(**kw)) == st, (name, kw)
        for kw, st in BAD_ROWS:
            assert call(rows=_rows(**kw)) == st, (name, kw)
        assert call(rows=_rows(v=None)) == 1 and call(rows=_rows(vs=250)) == 1
        assert call(slots=None) == 1 and call(count=-1) == 1 and call(qd=None) == 1 and call(qd=MIS) == 1
        assert call(p=mk(k=None)) == 1 and call(p=mk(hkv=4)) == 1 and call(p=mk(d=64)) == 1 and call(p=mk(nb=0)) == 1
        assert call(p=mk(v=MIS)) == 1 and call(rows=_rows(rows=0)) == 1
        assert call(count=0) == 0
    call8 = lambda p, r: lib.padoc_append_rotary_inputs_e4m3(ctypes.byref(p), ctypes.byref(_rot()), ctypes.byref(r), A,
                                                             None, A, 4, None)
    assert call8(pool8(), _rows(dtype=F32)) == 1 and call8(pool8(bs=8), _rows()) == 2
    assert call8(pool8(ks=None), _rows()) == 1 and call8(pool8(vs=A + 2), _rows()) == 1
    d64 = _rot(d=64, rot=64)
    assert lib.padoc_append_rotary_inputs_e4m3(ctypes.byref(pool8(d=64)), ctypes.byref(d64), ctypes.byref(_rows()), A, None,
                                               A, 4, None) == 2
    assert lib.padoc_append_rotary_inputs(ctypes.byref(pool(dtype=F32)), ctypes.byref(_rot()), ctypes.byref(_rows()), A,
                                          None, A, 4, None) == 1


@no_gpu
def test_copy_blocks_refusals(lib):
    def pools(n=2, **kw):
        a = dict(k=A, v=A, nb=64, bs=16, hkv=2, d=128, dtype=BF16)
        a.update(kw)
        return (pa.padoc_kv_pool * n)(*[pa.padoc_kv_pool(*a.values()) for _ in range(n)])

    def pools8(n=2, **kw):
        a = dict(k=A, v=A, ks=A, vs=A, nb=64, bs=16, hkv=2, d=128)
        a.update(kw)
        return (pa.padoc_kv_pool_e4m3 * n)(*[pa.padoc_kv_pool_e4m3(*a.values()) for _ in range(n)])

    for f, mk in ((lib.padoc_copy_kv_blocks, pools), (lib.padoc_copy_kv_blocks_e4m3, pools8)):
        call = lambda d=None, s=None, n=2, sb=A, db=A, c=3: f(d or mk(), s or mk(), n, sb, db, c, None)
        assert f(None, mk(), 2, A, A, 3, None) == 1 and f(mk(), None, 2, A, A, 3, None) == 1
        assert call(n=-1) == 1 and call(c=-1) == 1 and call(c=0) == 0 and call(n=0) == 0
        assert call(sb=None) == 1 and call(db=A + 2) == 1
        for bad in (dict(k=None), dict(v=MIS), dict(nb=0), dict(hkv=0), dict(hkv=3), dict(d=64), dict(bs=8)):
            assert call(s=mk(**bad)) == 1, bad
        mixed = mk()
        mixed[1].num_blocks = 32
        assert call(d=mixed) == 1 and call(s=mixed) == 1
        assert call(s=mk(nb=32), c=0) == 0          # another size is allowed
    assert lib.padoc_copy_kv_blocks(pools(dtype=F32), pools(), 2, A, A, 3, None) == 1
    assert lib.padoc_copy_kv_blocks(pools(dtype=7), pools(dtype=7), 2, A, A, 3, None) == 1
    odd = lambda: pools(bs=1, hkv=1, d=4)
    assert lib.padoc_copy_kv_blocks(odd(), odd(), 2, A, A, 3, None) == 2
    assert lib.padoc_copy_kv_blocks_e4m3(pools8(d=64), pools8(d=64), 2, A, A, 3, None) == 2
    assert lib.padoc_copy_kv_blocks_e4m3(pools8(ks=None), pools8(), 2, A, A, 3, None) == 1


# ------------------------------------------------------------------------------------------------
# The scheduler: forks with history, drops, compaction, resizing
# ------------------------------------------------------------------------------------------------

class Model:
    """A host pool written only through the scheduler's slots and copies, and what every stream must read."""

    def __init__(self, num_blocks, order=None):
        self.mpd = pa.Mpd(num_blocks, BS, order)
        self.nb = num_blocks
        self.pool, self.want, self.shared, self.page_of, self.cut = {}, {}, {}, {}, {}
        self.token = 0

    def add_page(self, prefix, forks):
        pid, slots, new = self.mpd.add_page(prefix, forks, False)
        self.shared[pid] = [self._write(s) for s in slots]
        for i, s in enumerate(new.tolist()):
            self.page_of[s] = pid
            self.want[s], self.cut[s] = [], (None if i == 0 else prefix)
        return pid, new.tolist()

    def _write(self, slot):
        self.token += 1
        self.pool[int(slot)] = self.token
        return self.token

    def step(self, forks=None, eos=None):
        ids, slots = self.mpd.begin_step()
        page_len, streams, pt, st = self.mpd.step_tables()
        for s, slot in zip(ids.tolist(), slots.tolist()):
            t = self._write(slot)
            (self.shared[self.page_of[s]] if self.cut[s] is None else self.want[s]).append(t)
        for i, s in enumerate(ids.tolist()):
            pi, cut, priv = (int(x) for x in streams[i])
            sh = self.shared[self.page_of[s]]
            assert [self.pool[int(pt[pi][j // BS]) * BS + j % BS] for j in range(cut)] == sh[:cut]
            assert cut == (len(sh) if self.cut[s] is None else self.cut[s])
            got = [self.pool[int(st[i][j // BS]) * BS + j % BS] for j in range(priv)]
            assert got == self.want[s], f"stream {s} reads rows that are not its own"
        assert (pt < self.nb).all() and (st < self.nb).all()
        nf = np.array([(forks or {}).get(int(s), 0) for s in ids], np.int32)
        end = np.array([int(s) in (eos or ()) for s in ids], np.uint8)
        new = self.mpd.end_step(nf, end).tolist()
        for s, n in zip(ids.tolist(), nf.tolist()):
            for _ in range(n):
                b = new.pop(0)
                self.page_of[b], self.want[b], self.cut[b] = self.page_of[s], [], len(self.shared[self.page_of[s]])
        return ids.tolist()

    def copy(self, src, dst):
        assert not set(src.tolist()) & set(dst.tolist()) and len(set(dst.tolist())) == len(dst)
        for a, b in zip(src.tolist(), dst.tolist()):
            for j in range(BS):
                if a * BS + j in self.pool:
                    self.pool[b * BS + j] = self.pool[a * BS + j]

    def fork(self, s, n):
        new, src, dst = self.mpd.fork_stream(s, n)
        assert len(set(src.tolist())) <= 1
        for a, b in zip(src.tolist(), dst.tolist()):
            self.copy(np.array([a]), np.array([b]))
        for b in new.tolist():
            self.page_of[b], self.want[b], self.cut[b] = self.page_of[s], list(self.want[s]), self.cut[s]
        return new.tolist()

    def compact(self):
        live = self.nb - self.mpd.status()[2]
        src, dst = self.mpd.compact()
        self.copy(src, dst)
        for b in range(live, self.nb):
            for j in range(BS):
                self.pool.pop(b * BS + j, None)   # nothing above is read again
        assert self.nb - self.mpd.status()[2] == live
        return live


def test_fork_stream_shares_full_blocks_and_copies_the_tail():
    m = Model(32, np.random.default_rng(1).permutation(32))
    pid, (layout, a) = m.add_page(20, 1)
    for _ in range(16):
        m.step()
    free = m.mpd.status()[2]
    b, c = m.fork(a, 2)                         # 16 rows: a full block, shared, nothing to copy
    assert m.mpd.status() == (1, 4, free)
    for _ in range(5):
        m.step()
    free = m.mpd.status()[2]
    d, = m.fork(b, 1)                           # 21 rows: one shared block, a tail of 5 rows copied
    assert m.mpd.status()[2] == free - 1
    m.step(eos={a})                             # the first owner goes; the shared block stays
    m.step()
    m.mpd.drop_stream(c)
    m.step(eos={b})
    for _ in range(14):
        m.step()
    m.mpd.drop_stream(d)
    m.step(eos={layout})
    assert m.mpd.status() == (0, 0, 32)


def test_fork_of_an_empty_branch_and_of_a_fork():
    m = Model(16)
    pid, (layout, a) = m.add_page(3, 1)
    b, = m.fork(a, 1)                           # no rows yet
    m.step()
    c, d = m.fork(b, 2)
    e, = m.fork(c, 1)
    for _ in range(40):
        m.step(eos=None)
        if m.mpd.status()[2] < 6:
            break
    m.mpd.drop_page(pid)
    assert m.mpd.status() == (0, 0, 16)


def test_scheduler_refusals():
    mpd = pa.Mpd(4, BS)
    pid, slots, (layout, a) = mpd.add_page(16, 1)
    def refuse(status, f, *args):
        with pytest.raises(pa.PadocError) as e:
            f(*args)
        assert e.value.status == status
    refuse(1, mpd.fork_stream, layout, 1)
    refuse(1, mpd.fork_stream, a, -1)
    refuse(1, mpd.fork_stream, 99, 1)
    refuse(1, mpd.fork_stream, -1, 1)
    refuse(1, mpd.drop_stream, 99)
    refuse(1, mpd.drop_page, pid + 1)
    assert mpd.fork_stream(a, 0)[0].size == 0
    mpd.begin_step()
    for f, args in ((mpd.fork_stream, (a, 1)), (mpd.drop_stream, (a,)), (mpd.drop_page, (pid,)), (mpd.resize, (8,))):
        refuse(1, f, *args)
    refuse(1, mpd.compact)
    mpd.end_step(num_streams=2)
    refuse(6, mpd.fork_stream, a, 2)            # one free block, two tails
    assert mpd.status() == (1, 2, 1)
    refuse(6, mpd.resize, 2)                    # live blocks beyond
    refuse(1, mpd.resize, -1)
    refuse(1, mpd.resize, 1 << 30)
    mpd.drop_stream(a)
    refuse(1, mpd.drop_stream, a)
    refuse(1, mpd.fork_stream, a, 1)
    mpd.drop_stream(layout)
    assert mpd.status() == (0, 0, 4)
    refuse(1, mpd.drop_page, pid)
    mpd.resize(0)
    assert mpd.status() == (0, 0, 0)
    assert mpd.compact()[0].size == 0
    mpd.resize(3)
    assert mpd.status() == (0, 0, 3)


@pytest.mark.parametrize("seed", range(6))
def test_random_serving_with_forks_drops_compaction_and_resizing(seed):
    rng = np.random.default_rng(seed)
    nb = 96
    m = Model(nb, rng.permutation(nb))
    pages, streams = [], {}
    for step in range(120):
        if len(pages) < 3 and m.mpd.status()[2] > 30:
            pid, new = m.add_page(int(rng.integers(0, 50)), int(rng.integers(0, 4)))
            pages.append(pid)
        live = set(m.step()) if m.mpd.status()[2] >= m.mpd.status()[1] else None   # (a block each at most)
        if live is None:                        # room is short: give some up
            p = pages.pop(int(rng.integers(len(pages))))
            m.mpd.drop_page(p)
            for s in [s for s in m.want if m.page_of[s] == p]:
                del m.want[s]
            continue
        branches = [s for s in live if m.cut[s] is not None and s in m.want]
        act = rng.random()
        if act < 0.25 and branches and m.mpd.status()[2] > 20:
            m.fork(int(rng.choice(branches)), int(rng.integers(1, 4)))
        elif act < 0.4 and branches:
            s = int(rng.choice(branches))
            m.mpd.drop_stream(s)
            del m.want[s]
        elif act < 0.6:
            live_blocks = m.compact()
            if rng.random() < 0.5:
                m.nb = int(rng.integers(live_blocks + 12, 130))
                m.mpd.resize(m.nb)
        pages = [p for p in pages if any(m.page_of[s] == p for s in m.want)]
    for p in pages:
        m.mpd.drop_page(p)
    assert m.mpd.status() == (0, 0, m.nb)
