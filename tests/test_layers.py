"""On the CPU: the masks' generator against published numbers, and what the layers' and answers' calls refuse."""
import ctypes as C

import numpy as np
import pytest

from tests import layers_util as lu

recd = pytest.importorskip("paper_2211_05239_amd.recd")


# known answers that the generator's authors publish with it
@pytest.mark.parametrize("ctr,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_generator(ctr, key, want):
    assert tuple(int(v) for v in lu.philox(np.array(ctr, dtype=np.uint64), key)) == want


def test_a_mask_keeps_its_share():
    """300 000 draws: the share kept is within five deviations."""
    for p in (0.1, 0.5, 0.9):
        kept = lu.keep(1000, 300, p, 123, 5).double()
        assert abs(float(kept.mean()) - (1 - p)) < 5 * (p * (1 - p) / kept.numel()) ** 0.5
    a, b = lu.keep(100, 80, 0.5, 1, 2), lu.keep(100, 80, 0.5, 1, 3)
    assert 0.4 < float((a == b).double().mean()) < 0.6


def _dense_bytes(n=4, inner=64, outer=64, dtype=0, act=0, p=None):
    mask = C.pointer(recd._Mask(p, 1, 2, None)) if p is not None else None
    out = C.c_size_t(7)
    st = recd._lib.recd_dense_workspace_bytes(0, C.byref(recd._Dense(n, inner, outer, dtype, act, 0, 0, 0, mask)), C.byref(out))
    assert st == recd.RECD_OK or out.value == 7
    return st


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=1 << 31), dict(inner=0), dict(outer=-4), dict(inner=6), dict(inner=4, dtype=2),
                                 dict(outer=65540), dict(dtype=3), dict(dtype=-1), dict(act=4), dict(act=-1), dict(p=1.0), dict(p=-0.1),
                                 dict(p=float("nan")), dict(p=0.99999999), dict(p=float("inf"))])
def test_layers_that_are_refused(bad):
    assert _dense_bytes(**bad) == recd.RECD_EINVAL


def test_null_arguments():
    lib, bad, out = recd._lib, recd.RECD_EINVAL, C.c_size_t(7)
    assert lib.recd_dense_workspace_bytes(0, None, C.byref(out)) == bad
    assert lib.recd_dense_workspace_bytes(0, C.byref(recd._Dense(4, 64, 64)), None) == bad
    assert lib.recd_dense(None, C.byref(recd._Dense(4, 64, 64)), None, None, None, None, None, None) == bad
    assert lib.recd_dense_backward(None, C.byref(recd._Dense(4, 64, 64)), None, None, None, None, None, 0, None, 0, None, None) == bad
    assert lib.recd_dropout(None, 4, 64, 0, None, None, None, None) == bad
    assert lib.recd_dropout_backward(None, 4, 64, 0, None, None, None) == bad
    assert lib.recd_vocab_answers(None, 4, 8, 64, 0, None, None, 1.0, None, 0, None, None, None, None, None) == bad
    assert lib.recd_vocab_answers_workspace_bytes(0, 4, 8, 64, 0, 1, None) == bad


@pytest.mark.parametrize("n,V,D,dt,k", [(-1, 8, 64, 0, 1), (1 << 31, 8, 64, 0, 1), (4, -1, 64, 0, 0), (4, 1 << 31, 64, 0, 1), (4, 8, 0, 0, 1),
                                        (4, 8, 6, 0, 1), (4, 8, 4, 1, 1), (4, 8, 260, 0, 1), (4, 8, 64, 3, 1), (4, 8, 64, 0, -1),
                                        (4, 8, 64, 0, 9), (4, 80, 64, 0, 65)])
def test_answers_that_are_refused(n, V, D, dt, k):
    out = C.c_size_t(7)
    assert recd._lib.recd_vocab_answers_workspace_bytes(0, n, V, D, dt, k, C.byref(out)) == recd.RECD_EINVAL and out.value == 7
