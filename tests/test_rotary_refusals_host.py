"""CPU tests of further calls that the rotary entry points refuse (with stand-in addresses, so on machines without a GPU)."""
import ctypes

import pytest
import torch

from paper_2608_06146_gb300 import build as pbuild
from paper_2608_06146_gb300 import padoc_attn as pa

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="stand-in addresses are for machines without a GPU")
A = 1 << 20
BF16 = pa.PADOC_DTYPE_BF16


@pytest.fixture(scope="module")
def lib():
    pbuild.build()
    return pa.load_library()


def rot(**kw):
    a = dict(freq=A, qw=A, kw=A, d=128, rot=128, axes=1, adjacent=0, eps=1e-6, amp=1.0)
    a.update(kw)
    return pa.padoc_rotary(*a.values())


def rows(n=10):
    return pa.padoc_qkv_rows(A, A, A, 2048, 256, 256, A, n, 16, 2, BF16)


@pytest.mark.parametrize("n", [0, 10])
def test_weight_gradients_that_overlap(lib, n):
    def call(dqw, dkw):
        return lib.padoc_qk_rotary_bwd(ctypes.byref(rot()), ctypes.byref(rows(n)), A, 2048, A, 256, A, 2048, A, 256, dqw, dkw, A,
                                       1 << 24, None)
    for off in (0, 4, 127 * 4):
        assert call(A, A + off) == 1 and call(A + off, A) == 1
    assert call(A, A + 512) not in (0, 1) and call(A + 512, A) not in (0, 1)   # (the launch, that finds no GPU)


@pytest.mark.parametrize("e4m3", [False, True])
def test_append_lists_off_a_4_byte_boundary(lib, e4m3):
    if e4m3:
        pool, f = pa.padoc_kv_pool_e4m3(A, A, A, A, 64, 16, 2, 128), lib.padoc_append_rotary_inputs_e4m3
    else:
        pool, f = pa.padoc_kv_pool(A, A, 64, 16, 2, 128, BF16), lib.padoc_append_rotary_inputs
    call = lambda src, slots: f(ctypes.byref(pool), ctypes.byref(rot()), ctypes.byref(rows()), A, src, slots, 4, None)
    for off in (1, 2, 3):
        assert call(None, A + off) == 1 and call(A + off, A) == 1
    assert call(None, A + 4) not in (0, 1) and call(A + 4, A) not in (0, 1)    # (no GPU to launch on)
