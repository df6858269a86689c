"""Argument checks of the step's entry points: everything wrong is refused on
the host before a launch (no GPU needed; the addresses are never used)."""

import pytest
import torch

from conftest import ensure_library

FAKE, OFF = 0x10000, 0x10008
ARG, SHAPE, ALIGN, FORMAT, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    return ensure_library()


def _call(f, args, kw):
    assert set(kw) <= set(args), kw
    return f(*{**args, **kw}.values())


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), SHAPE), (dict(K=0), SHAPE), (dict(E=0), SHAPE), (dict(E=2049), SHAPE), (dict(T=1 << 28, K=8), SHAPE),
    (dict(bytes=2), ARG), (dict(ids=None), ARG), (dict(offsets=None), ARG), (dict(token=None), ARG), (dict(slot=None), ARG),
    (dict(ids=FAKE + 4), ALIGN), (dict(offsets=FAKE + 2), ALIGN), (dict(slot=FAKE + 1), ALIGN), (dict(token=FAKE + 2), ALIGN),
    (dict(T=1 << 20), WORKSPACE), (dict(T=1 << 20, ws=FAKE, size=64), WORKSPACE),
    (dict(T=1 << 20, ws=FAKE + 2, size=1 << 30), ALIGN),
])
def test_sort_refusals(lib, kw, status):
    args = dict(T=16, K=8, E=32, ids=FAKE, bytes=8, offsets=FAKE, token=FAKE, slot=FAKE, ws=None, size=0, stream=None)
    assert _call(lib.sq_moe_sort, args, kw) == status


def test_sort_workspace(lib):
    assert lib.sq_moe_sort_workspace(4, 2, 8) == 0
    assert lib.sq_moe_sort_workspace(1 << 20, 8, 64) >= (1 << 23) // 4096 * 65 * 4
    assert lib.sq_moe_sort_workspace(1 << 20, 8, 5000) == 0            # invalid


ROWS = [(dict(T=-1), SHAPE), (dict(K=0), SHAPE), (dict(E=0), SHAPE), (dict(H=12), SHAPE), (dict(H=0), SHAPE),
        (dict(T=1 << 30, K=4), SHAPE), (dict(slot=None), ARG), (dict(offsets=None), ARG), (dict(slot=FAKE + 2), ALIGN),
        (dict(offsets=FAKE + 1), ALIGN)]


@pytest.mark.parametrize("kw,status", ROWS + [(dict(X=None), ARG), (dict(Xs=None), ARG), (dict(dtype=2), ARG),
                                              (dict(X=OFF), ALIGN), (dict(Xs=OFF), ALIGN)])
def test_gather_refusals(lib, kw, status):
    args = dict(T=16, K=8, E=32, H=64, X=FAKE, dtype=1, slot=FAKE, offsets=FAKE, Xs=FAKE, stream=None)
    assert _call(lib.sq_moe_gather, args, kw) == status


@pytest.mark.parametrize("kw,status", ROWS + [(dict(Ys=None), ARG), (dict(out=None), ARG), (dict(yd=2), ARG),
                                              (dict(od=-1), ARG), (dict(Ys=OFF), ALIGN), (dict(out=OFF), ALIGN),
                                              (dict(w=FAKE + 2), ALIGN)])
def test_combine_refusals(lib, kw, status):
    args = dict(T=16, K=8, E=32, H=64, Ys=FAKE, yd=1, slot=FAKE, offsets=FAKE, w=FAKE, out=FAKE, od=0, stream=None)
    assert _call(lib.sq_moe_combine, args, kw) == status


@pytest.mark.parametrize("kw,status", ROWS + [(dict(d=None), ARG), (dict(Ys=None), ARG), (dict(w=None), ARG), (dict(g=None), ARG),
                                              (dict(dw=None), ARG), (dict(dd=3), ARG), (dict(yd=3), ARG), (dict(gd=3), ARG),
                                              (dict(d=OFF), ALIGN), (dict(Ys=OFF), ALIGN), (dict(g=OFF), ALIGN),
                                              (dict(w=FAKE + 1), ALIGN), (dict(dw=FAKE + 2), ALIGN)])
def test_combine_bwd_refusals(lib, kw, status):
    args = dict(T=16, K=8, E=32, H=64, d=FAKE, dd=1, Ys=FAKE, yd=1, slot=FAKE, offsets=FAKE, w=FAKE, g=FAKE, gd=1, dw=FAKE,
                stream=None)
    assert _call(lib.sq_moe_combine_bwd, args, kw) == status


def test_empty_batches_launch_nothing(lib):
    assert lib.sq_moe_gather(0, 8, 32, 64, None, 1, None, FAKE, None, None) == 0
    assert lib.sq_moe_combine(0, 8, 32, 64, None, 1, None, FAKE, None, None, 1, None) == 0
    assert lib.sq_moe_combine_bwd(0, 8, 32, 64, None, 1, None, 1, None, FAKE, None, None, 1, None, None) == 0


def test_binding_refuses_what_the_library_cannot_see():
    """Wrong dtypes, shapes, strides and host tensors raise before the call."""
    ensure_library()
    from paper_2609_04526_amd import sq
    slot = torch.zeros((4, 2), dtype=torch.int32)
    offsets = torch.zeros(9, dtype=torch.int32)
    X = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors"):
        sq.sq_moe_gather(X, slot, offsets)
    with pytest.raises(ValueError, match="ids"):
        sq.sq_moe_sort(torch.zeros((4, 2)), 8)
    with pytest.raises(ValueError, match="slot"):
        sq.sq_moe_gather(X, slot.long(), offsets)
    with pytest.raises(ValueError, match="offsets"):
        sq.sq_moe_gather(X, slot, offsets.view(3, 3))
    with pytest.raises(ValueError, match="contiguous"):
        sq.sq_moe_gather(torch.zeros((64, 4), dtype=torch.bfloat16).t(), slot, offsets)
    with pytest.raises(ValueError, match="shape"):
        sq.sq_moe_combine(X, slot, offsets)                  # 4 rows for 8 pairs
    with pytest.raises(ValueError, match="weights"):
        sq.sq_moe_combine(torch.zeros((8, 64)), slot, offsets, torch.zeros((4, 2), dtype=torch.float64))
