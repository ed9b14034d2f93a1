"""The decoding loop's cross attention: each step's tokens over their page's states, or a branch's own range of them.

Outputs are held to oracle.cross's bounds, with each stream's states tracked here."""
import numpy as np
import pytest
import torch

from oracle import cross as oc
from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import engine
from paper_2608_06146_gb300 import padoc_attn as pa

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda:0", torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def check(ids, states, q, k, v, out, lse, scale):
    segments = [(i, 1) + states[int(s)] for i, s in enumerate(ids)]
    want, wl, _ = oc.forward(segments, q, k, v, scale)
    bo, bl = oc.forward_bounds(segments, q, k, v, scale)
    assert ((out.double() - want).abs() <= bo).all()
    assert ((lse.double() == wl) | ((lse.double() - wl).abs() <= bl)).all()


@pytest.mark.parametrize("run_step", [False, True])
@pytest.mark.parametrize("hq,hkv,d,ekv,dtype", [(16, 2, 128, 2, BF16), (16, 2, 128, 16, BF16), (4, 1, 64, 1, F32)])
def test_loop(hq, hkv, d, ekv, dtype, run_step):
    g = torch.Generator(DEV).manual_seed(3)
    new = lambda n, h: torch.randn((n, h, d), generator=g, device=DEV).to(dtype)   # noqa: E731
    loop = engine.MaskedParallelLoop(400, hq, hkv, d, dtype, DEV)
    q, k, v = new(64, hq), new(64, hkv), new(64, hkv)
    kv = new(3000, 2 * ekv)
    ek, ev = kv[:, :ekv], kv[:, ekv:]
    states = {}

    def admit(prefix, forks, at):
        pid, ids = loop.add_page(prefix, forks, False, k, v, np.arange(prefix), states=at)
        states.update({int(i): at for i in ids})
        return pid, ids
    admit(20, 2, (0, 700))
    admit(7, 1, (700, 0))                   # a page without an image
    pid, last = admit(33, 3, (1000, 1301))
    loop.set_states(int(last[2]), 1100, 77)       # a branch over its region's crop
    states[int(last[2])] = (1100, 77)
    rows = np.arange(256, dtype=np.int32) % 64
    uploads = []
    for step in range(6):
        if run_step:
            o, l = torch.empty((64, hq, d), dtype=dtype, device=DEV), torch.empty((64, hq), device=DEV)
            n, ids = loop.run_step(k, v, q, rows, 0.2, o, l)
            self_out = o[:n]
        else:
            ids, self_out, _ = loop.step(k, v, q, lambda i: rows[i], 0.2)
        before = loop._cross_plan
        out, lse = loop.cross_step(ids, self_out, ek, ev, 0.2)
        uploads.append(loop._cross_plan is not before)
        check(ids, states, self_out, ek, ev, out, lse, 0.2)
        forks, eos = np.zeros(len(ids), np.int32), np.zeros(len(ids), np.uint8)
        if step == 1:                       # the last page's layout stream forks two branches, another stream ends
            at = [i for i, s in enumerate(ids) if int(s) == int(last[0])][0]
            forks[at], eos[0] = 2, 1
        made = loop.end_step(forks, eos)
        for i in made:
            states[int(i)] = states[int(last[0])]
        if step == 2:
            for i in loop.fork_stream(int(last[2]), 2):
                states[int(i)] = (1100, 77)
        if step == 3:
            loop.drop_page(pid)
            admit(5, 0, (2500, 500))
    pa.padoc_check_device_errors()
    assert uploads == [True, False, True, True, True, False]


def test_a_loop_without_states():
    loop = engine.MaskedParallelLoop(100, 16, 2, 128, BF16, DEV)
    q, k, v = (torch.randn((8, h, 128), device=DEV).to(BF16) for h in (16, 2, 2))
    loop.add_page(4, 1, False, k, v, np.arange(4))
    ids, o, _ = loop.step(k, v, q, lambda i: i % 8, 0.1)
    out, lse = loop.cross_step(ids, o, k, v, 0.1)
    assert (out == 0).all() and (lse == -float("inf")).all()
    loop.end_step(num_streams=len(ids))
    loop.set_states(int(ids[1]), 2, 6)
    ids, o, _ = loop.step(k, v, q, lambda i: i % 8, 0.1)
    out, lse = loop.cross_step(ids, o, k, v, 0.1)
    check(ids, {int(ids[0]): (0, 0), int(ids[1]): (2, 6)}, o, k, v, out, lse, 0.1)
    with pytest.raises(pa.PadocError):      # fewer rows than a stream's states
        loop.cross_step(ids, o, k[:5], v[:5], 0.1)
    with pytest.raises(ValueError):
        loop.cross_step(ids, o[:1], k, v, 0.1)
    with pytest.raises(ValueError):
        loop.set_states(0, -1, 4)
    with pytest.raises(ValueError):
        loop.add_page(4, 1, False, k, v, np.arange(4), states=(0, 2 ** 31))
