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


# ---------------------------------------------------------------- 8-bit activations
@pytest.mark.parametrize("name", ["sq_act_pack", "sq_act_unpack"])
@pytest.mark.parametrize("kw,status", [
    (dict(act=2), ARG), (dict(T=-1), SHAPE), (dict(I=0), SHAPE), (dict(I=48), SHAPE), (dict(T=1 << 30, I=1 << 20), SHAPE),
    (dict(a=None), ARG), (dict(b=None), ARG), (dict(c=None), ARG), (dict(a=OFF), ALIGN),
])
def test_act_refusals(lib, name, kw, status):
    args = dict(act=0, T=16, I=64, a=FAKE, b=FAKE, c=FAKE, stream=None)
    assert _call(getattr(lib, name), args, kw) == status
    assert _call(getattr(lib, name), args, dict(T=0, a=None, b=None, c=None)) == 0


@pytest.mark.parametrize("name", ["sq_act_pack", "sq_act_unpack"])
@pytest.mark.parametrize("T,I", [(1 << 21, 1 << 16), ((1 << 26) + 1, 1 << 10), (1 << 30, 128)])
def test_more_values_than_a_launch_holds(lib, name, T, I):
    assert getattr(lib, name)(0, T, I, FAKE, FAKE, FAKE, None) == SHAPE

def test_act_alignment_of_the_second_plane(lib):
    assert lib.sq_act_pack(0, 16, 64, FAKE, OFF, FAKE, None) == ALIGN
    assert lib.sq_act_unpack(0, 16, 64, FAKE, FAKE, OFF, None) == ALIGN


DS8 = [(dict(fmt=2), FORMAT), (dict(act=-1), ARG), (dict(O=12), SHAPE), (dict(I=48), SHAPE), (dict(fmt=1, I=48), SHAPE),
       (dict(T=-1), SHAPE), (dict(x=None), ARG), (dict(xs=None), ARG), (dict(dY=None), ARG), (dict(codes=None), ARG),
       (dict(dS=None), ARG), (dict(x=OFF), ALIGN), (dict(dY=OFF), ALIGN), (dict(codes=FAKE + 2), ALIGN),
       (dict(dS=FAKE + 2), ALIGN)]


@pytest.mark.parametrize("kw,status", DS8 + [
    (dict(T=1 << 17, I=1 << 13), SHAPE), (dict(T=4096, O=1024, I=4096), WORKSPACE),
    (dict(T=4096, O=1024, I=4096, ws=FAKE, size=100), WORKSPACE), (dict(T=4096, O=1024, I=4096, ws=OFF, size=1 << 22), ALIGN)])
def test_dscale_act8_refusals(lib, kw, status):
    args = dict(fmt=0, act=0, T=64, O=256, I=512, x=FAKE, xs=FAKE, dY=FAKE, codes=FAKE, dS=FAKE, ws=None, size=0, stream=None)
    assert _call(lib.sq_bwd_dscale_act8, args, kw) == status


def test_dscale_act8_workspace(lib):
    assert lib.sq_bwd_dscale_act8_workspace(0, 1024, 4096, 4096) == 0
    assert lib.sq_bwd_dscale_act8_workspace(0, 4096, 4096, 4096) == 4096 * 4096 * 2 + lib.sq_bwd_dscale_workspace(0, 4096, 4096, 4096)
    assert lib.sq_bwd_dscale_act8_workspace(0, 4096, 1024, 4096) == lib.sq_bwd_dscale_workspace(0, 4096, 1024, 4096) > 0
    assert lib.sq_bwd_dscale_act8_workspace(1, 4096, 1024, 4112) == 0          # not whole blocks of 32


@pytest.mark.parametrize("kw,status", DS8 + [
    (dict(E=0), SHAPE), (dict(E=8193), SHAPE), (dict(N=-1), SHAPE), (dict(N=1 << 30), SHAPE), (dict(rows=None), ARG),
    (dict(offsets=None), ARG), (dict(rows=FAKE + 2), ALIGN), (dict(offsets=FAKE + 1), ALIGN), (dict(T=1 << 26), SHAPE),
    (dict(T=1 << 21), SHAPE), (dict(ws=None), WORKSPACE), (dict(size=64 * 512 * 2 - 1), WORKSPACE), (dict(ws=OFF), ALIGN)])
def test_dscale_act8_batched_refusals(lib, kw, status):
    args = dict(fmt=0, act=0, E=4, T=64, N=128, O=256, I=512, x=FAKE, xs=FAKE, rows=FAKE, offsets=FAKE, dY=FAKE, codes=FAKE,
                dS=FAKE, ws=FAKE, size=64 * 512 * 2 + 16 + 8 * 256, stream=None)
    assert _call(lib.sq_bwd_dscale_act8_batched, args, kw) == status


# ---------------------------------------------------------------- cross entropy
CE = [(dict(head=3), FORMAT), (dict(head=-1), FORMAT), (dict(T=-1), SHAPE), (dict(V=0), SHAPE), (dict(I=12), SHAPE),
      (dict(head=0, I=48), SHAPE), (dict(head=1, I=40), SHAPE), (dict(T=1 << 20, I=2048), SHAPE), (dict(V=1 << 31), SHAPE),
      (dict(X=None), ARG), (dict(W=None), ARG), (dict(y=None), ARG), (dict(yb=2), ARG), (dict(head=0, scales=None), ARG),
      (dict(head=1, ws2=0.0), ARG), (dict(head=1, ws2=float("inf")), ARG), (dict(X=OFF), ALIGN), (dict(W=OFF), ALIGN),
      (dict(head=0, W=FAKE + 2), ALIGN), (dict(y=FAKE + 4), ALIGN), (dict(ws=None), WORKSPACE), (dict(size=100), WORKSPACE),
      (dict(ws=FAKE + 16), ALIGN)]


@pytest.mark.parametrize("kw,status", CE + [(dict(loss=None), ARG), (dict(lse=None), ARG), (dict(loss=FAKE + 2), ALIGN),
                                            (dict(lse=FAKE + 1), ALIGN)])
def test_ce_fwd_refusals(lib, kw, status):
    args = dict(head=2, T=64, V=1000, I=512, X=FAKE, W=FAKE, scales=FAKE, ws2=1.0, y=FAKE, yb=8, loss=FAKE, lse=FAKE, ws=FAKE,
                size=1 << 40, stream=None)
    assert _call(lib.sq_ce_fwd, args, kw) == status


@pytest.mark.parametrize("kw,status", CE + [(dict(lse=None), ARG), (dict(dl=None), ARG), (dict(dX=None), ARG), (dict(dt=2), ARG),
                                            (dict(lse=FAKE + 2), ALIGN), (dict(dl=FAKE + 2), ALIGN), (dict(dX=OFF), ALIGN)])
def test_ce_bwd_refusals(lib, kw, status):
    args = dict(head=2, T=64, V=1000, I=512, X=FAKE, W=FAKE, scales=FAKE, ws2=1.0, y=FAKE, yb=8, lse=FAKE, dl=FAKE, dX=FAKE,
                dt=1, ws=FAKE, size=1 << 40, stream=None)
    assert _call(lib.sq_ce_bwd, args, kw) == status


def test_ce_without_tokens(lib):
    assert lib.sq_ce_fwd(2, 0, 1000, 512, None, FAKE, None, 1.0, None, 8, None, None, None, 0, None) == 0
    assert lib.sq_ce_bwd(2, 0, 1000, 512, None, FAKE, None, 1.0, None, 8, None, None, None, 0, None, 0, None) == 0
    assert lib.sq_ce_fwd_workspace(2, 0, 1000, 512) == 0


@pytest.mark.parametrize("head", [0, 1, 2])
def test_ce_workspace_stays_bounded(lib, head):
    """No workspace holds the logits: a large batch over a large vocabulary stays under a gigabyte and a half."""
    T, V, I = 8192, 160000, 8192
    assert 0 < lib.sq_ce_fwd_workspace(head, T, V, I) < 3 << 29
    assert 0 < lib.sq_ce_bwd_workspace(head, T, V, I) < 3 << 29
    assert lib.sq_ce_fwd_workspace(head, T, V, 12) == 0


def test_binding_refuses_a_head_it_cannot_read():
    from paper_2609_04526_amd import sq
    X, y = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="W"):
        sq.sq_ce_fwd("bf16", X, torch.zeros((10, 32), dtype=torch.bfloat16), y)
    with pytest.raises(ValueError, match="scales"):
        sq.sq_ce_fwd("mx", X, torch.zeros((10, 32), dtype=torch.uint8), y)
    with pytest.raises(ValueError, match="targets"):
        sq.sq_ce_fwd("bf16", X, torch.zeros((10, 64), dtype=torch.bfloat16), y.float())
    with pytest.raises(ValueError, match="device tensors"):
        sq.sq_ce_fwd("bf16", X, torch.zeros((10, 64), dtype=torch.bfloat16), y)
