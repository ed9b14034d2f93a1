"""GPU tests of the cache block copies: every bit against an index copy, in pools of several layers, within a
cache and between caches of different sizes."""
import numpy as np
import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _build():
    pbuild.build()
    pa.load_library()


def pools(rng, layers, nb, hkv, d, dtype, e4m3=False):
    g = torch.Generator(device=DEV).manual_seed(int(rng.integers(1 << 30)))
    whole = lambda: torch.randint(-2 ** 31, 2 ** 31 - 1, (layers, nb, hkv, 16, d), generator=g, device=DEV).to(torch.int32)
    if e4m3:
        return [(*(whole()[i].to(torch.uint8) for _ in range(2)), *(torch.rand((nb, hkv), generator=g, device=DEV) for _ in range(2)))
                for i in range(layers)]
    make = lambda: whole().view(torch.float32) if dtype == torch.float32 else whole().to(torch.int16).view(torch.bfloat16)
    k, v = make(), make()
    return [(k[i], v[i]) for i in range(layers)]


def bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def wrap(ps, e4m3):
    return (pa.KvPoolsE4M3 if e4m3 else pa.KvPools)(ps)


CASES = [(1, 1, 2, 128, torch.bfloat16, False, 1), (3, 40, 2, 128, torch.bfloat16, False, 17),
         (2, 300, 1, 64, torch.float32, False, 150), (33, 12, 2, 128, torch.bfloat16, False, 5),
         (65, 9, 1, 8, torch.bfloat16, False, 4), (1, 5000, 2, 128, torch.bfloat16, False, 2400),
         (2, 7, 3, 80, torch.bfloat16, False, 3), (1, 30, 2, 128, None, True, 14), (40, 9, 5, 128, None, True, 4),
         (4, 64, 1, 128, torch.float32, False, 0), (1, 50, 300, 8, torch.bfloat16, False, 20)]


@pytest.mark.parametrize("layers,nb,hkv,d,dtype,e4m3,count", CASES)
def test_copies_within_and_between_pools(layers, nb, hkv, d, dtype, e4m3, count):
    rng = np.random.default_rng(nb + layers)
    copy = pa.padoc_copy_kv_blocks_e4m3 if e4m3 else pa.padoc_copy_kv_blocks
    ps = pools(rng, layers, nb, hkv, d, dtype, e4m3)
    perm = rng.permutation(nb).astype(np.int32)
    src, dst = perm[:count], perm[count:2 * count] if nb > 1 else perm[:count]
    want = [tuple(t.clone() for t in p) for p in ps]
    for p in want:
        for t in p:
            t[dst.astype(np.int64)] = t[src.astype(np.int64)]
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    copy(wrap(ps, e4m3), up(src), up(dst))
    pa.padoc_check_device_errors()
    for p, w in zip(ps, want):
        for t, x in zip(p, w):
            assert torch.equal(bits(t), bits(x))
    # into a cache of another size; a block may be copied to several places
    other = pools(rng, layers, nb + 7, hkv, d, dtype, e4m3)
    want = [tuple(t.clone() for t in p) for p in other]
    dst = rng.permutation(nb + 7).astype(np.int32)[:count + 2]
    src = rng.integers(0, nb, count + 2).astype(np.int32)
    for p, w in zip(ps, want):
        for t, x in zip(p, w):
            x[dst.astype(np.int64)] = t[src.astype(np.int64)]
    copy(wrap(other, e4m3), up(src), up(dst), wrap(ps, e4m3))
    pa.padoc_check_device_errors()
    for p, w in zip(other, want):
        for t, x in zip(p, w):
            assert torch.equal(bits(t), bits(x))


def test_copy_past_32_bits():
    nb = (9 << 30) // (2 * 16 * 128 * 2) // 2
    k, v = (torch.zeros((nb, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[nb - 1], v[nb - 1], k[3], v[3] = 1.5, 2.5, 3.5, 4.5
    src = torch.tensor([nb - 1, 3], dtype=torch.int32, device=DEV)
    dst = torch.tensor([0, nb - 2], dtype=torch.int32, device=DEV)
    pa.padoc_copy_kv_blocks(pa.KvPools([(k, v)]), src, dst)
    pa.padoc_check_device_errors()
    assert bool((k[0] == 1.5).all()) and bool((v[0] == 2.5).all()) and bool((k[nb - 2] == 3.5).all()) and bool((v[nb - 2] == 4.5).all())
    assert int((k.view(torch.int16).flatten(1) != 0).any(1).sum()) == 4


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("bad", [(0, -1), (0, 20), (1, -2), (1, 25)])
def test_bad_ids_are_reported_and_skipped(e4m3, bad):
    rng = np.random.default_rng(2)
    ps, other = pools(rng, 2, 20, 2, 128, torch.bfloat16, e4m3), pools(rng, 2, 25, 2, 128, torch.bfloat16, e4m3)
    ids = [np.array([3, 4, 5], np.int32), np.array([24, 0, 7], np.int32)]
    ids[bad[0]][1] = bad[1]
    before = [tuple(t.clone() for t in p) for p in other]
    up = lambda a: torch.from_numpy(a).to(DEV)
    copy = pa.padoc_copy_kv_blocks_e4m3 if e4m3 else pa.padoc_copy_kv_blocks
    copy(wrap(other, e4m3), up(ids[0]), up(ids[1]), wrap(ps, e4m3))
    with pytest.raises(pa.PadocError) as e:
        pa.padoc_check_device_errors()
    assert e.value.device_code == 1 and e.value.device_detail == bad[1]
    for p, w, s in zip(other, before, ps):
        for t, x, y in zip(p, w, s):
            x[24], x[7] = y[3], y[5]
            assert torch.equal(bits(t), bits(x))


def test_on_a_side_stream_and_in_a_graph():
    rng = np.random.default_rng(3)
    ps = pools(rng, 3, 60, 2, 128, torch.bfloat16)
    kp = pa.KvPools(ps)
    src, dst = (torch.from_numpy(x.astype(np.int32)).to(DEV) for x in np.split(rng.permutation(60), 2))
    want = [tuple(t.clone() for t in p) for p in ps]
    for p in want:
        for t in p:
            t[dst.long()] = t[src.long()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pa.padoc_copy_kv_blocks(kp, src, dst, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(bits(a), bits(b)) for p, w in zip(ps, want) for a, b in zip(p, w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.padoc_copy_kv_blocks(kp, dst, src)       # the captured copy goes the other way
    for p in ps:
        for t in p:
            t[src.long()] = 0
    graph.replay()
    torch.cuda.synchronize()
    for p, w in zip(ps, want):
        for t, x in zip(p, w):
            assert torch.equal(bits(t[src.long()]), bits(x[dst.long()]))


def test_python_refusals():
    rng = np.random.default_rng(4)
    a, b = pools(rng, 2, 6, 2, 128, torch.bfloat16), pools(rng, 1, 6, 2, 128, torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        pa.padoc_copy_kv_blocks(pa.KvPools(a), i, i, pa.KvPools(b))
    with pytest.raises(ValueError):
        pa.padoc_copy_kv_blocks(pa.KvPools(a), i.long(), i)
    with pytest.raises(ValueError):
        pa.padoc_copy_kv_blocks(pa.KvPools(a), i, i, count=4)
    with pytest.raises(ValueError):
        pa.KvPools([(a[0][0], a[0][1][:5])])
    with pytest.raises(pa.PadocError) as e:
        pa.padoc_copy_kv_blocks(pa.KvPools(a), i, i, pa.KvPools(pools(rng, 2, 6, 1, 128, torch.bfloat16)))
    assert e.value.status == 1
