"""Argument checks of a 4-bit student's entry points: everything wrong is refused
on the host before a launch (no GPU needed; the addresses are never used)."""

import math
import subprocess
import sys

import pytest
import torch

from conftest import ROOT, ensure_library

FAKE, OFF = 0x10000, 0x10008
ARG, SHAPE, ALIGN, FORMAT, WORKSPACE, UNIMPLEMENTED = -1, -2, -3, -4, -5, -7
MX, NV, BF = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    return ensure_library()


def _call(f, args, kw):
    assert set(kw) <= set(args), kw
    return f(*{**args, **kw}.values())


# ---------------------------------------------------------------- 4-bit activations
@pytest.mark.parametrize("kw,status", [
    (dict(fmt=2), FORMAT), (dict(T=-1), SHAPE), (dict(I=0), SHAPE), (dict(I=48), SHAPE), (dict(fmt=NV, I=40), SHAPE),
    (dict(T=1 << 21, I=1 << 16), SHAPE), (dict(T=1 << 30, I=128), SHAPE), (dict(fmt=NV, ws2=0.0), ARG),
    (dict(fmt=NV, ws2=-1.0), ARG), (dict(fmt=NV, ws2=math.inf), ARG), (dict(fmt=NV, ws2=math.nan), ARG),
    (dict(X=None), ARG), (dict(c=None), ARG), (dict(s=None), ARG), (dict(X=OFF), ALIGN), (dict(c=FAKE + 2), ALIGN),
])
def test_pack_refusals(lib, kw, status):
    args = dict(fmt=MX, T=16, I=64, X=FAKE, ws2=1.0, c=FAKE, s=FAKE, stream=None)
    assert _call(lib.sq_act4_pack, args, kw) == status
    assert _call(lib.sq_act4_pack, args, dict(T=0, X=None, c=None, s=None)) == 0
    args = dict(fmt=MX, T=16, I=64, c=FAKE, s=FAKE, ws2=1.0, X=FAKE, stream=None)
    assert _call(lib.sq_act4_unpack, args, kw) == status
    assert _call(lib.sq_act4_unpack, args, dict(T=0, X=None, c=None, s=None)) == 0


FWD = [(dict(fmt=2), FORMAT), (dict(T=-1), SHAPE), (dict(O=0), SHAPE), (dict(O=12), SHAPE), (dict(I=48), SHAPE),
       (dict(T=1 << 25, I=64), SHAPE), (dict(xc=None), ARG), (dict(xs=None), ARG), (dict(c=None), ARG), (dict(s=None), ARG),
       (dict(Y=None), ARG), (dict(yd=2), ARG), (dict(xc=OFF), ALIGN), (dict(c=OFF), ALIGN), (dict(xs=FAKE + 2), ALIGN),
       (dict(s=FAKE + 1), ALIGN), (dict(Y=OFF), ALIGN)]


@pytest.mark.parametrize("kw,status", FWD + [
    (dict(fmt=NV), WORKSPACE), (dict(fmt=NV, ws=FAKE, size=16 * 64 * 2 - 1), WORKSPACE),
    (dict(fmt=NV, ws=FAKE + 16, size=1 << 20), ALIGN), (dict(fmt=NV, xw=0.0), ARG), (dict(fmt=NV, w2=math.nan), ARG),
    (dict(fmt=NV, xw=1e-30, w2=1e-30), ARG), (dict(fmt=NV, xw=1e30, w2=1e30), ARG)])
def test_fwd_refusals(lib, kw, status):
    args = dict(fmt=MX, T=128, O=64, I=128, xc=FAKE, xs=FAKE, xw=1.0, c=FAKE, s=FAKE, w2=1.0, Y=FAKE, yd=1, ws=None, size=0,
                stream=None)
    assert _call(lib.sq_fwd_act4, args, kw) == status


def test_fwd_of_no_tokens(lib):
    assert lib.sq_fwd_act4(MX, 0, 64, 96, None, None, 1.0, FAKE, FAKE, 1.0, None, 1, None, 0, None) == 0


@pytest.mark.parametrize("kw,status", FWD + [
    (dict(fmt=NV), UNIMPLEMENTED), (dict(E=0), SHAPE), (dict(E=8193), SHAPE), (dict(N=-1), SHAPE), (dict(N=1 << 31), SHAPE),
    (dict(E=8192, N=1 << 20, O=1 << 18, I=32), SHAPE), (dict(off=None), ARG), (dict(rows=None, N=130), ARG),
    (dict(rows=FAKE + 2), ALIGN), (dict(off=FAKE + 1), ALIGN)])
def test_experts_refusals(lib, kw, status):
    args = dict(fmt=MX, E=4, T=128, N=256, O=64, I=128, xc=FAKE, xs=FAKE, rows=FAKE, off=FAKE, c=FAKE, s=FAKE, Y=FAKE, yd=1,
                ws=None, size=0, stream=None)
    assert _call(lib.sq_fwd_act4_batched, args, kw) == status
    assert _call(lib.sq_fwd_act4_batched, args, dict(T=0, N=0, xc=None, xs=None, rows=None, Y=None)) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(), 0), (dict(N=1 << 18), 0), (dict(N=1 << 20, T=1 << 20), 0),                    # T*O*2 and N*O*2 of 2.2 GB and more
    (dict(T=(1 << 25) - 1), 0), (dict(T=1 << 25), SHAPE), (dict(I=1 << 12, T=8, N=8, O=1 << 20), SHAPE),
    (dict(I=1 << 12, T=8, N=8, O=(1 << 20) - 8), 0), (dict(O=8444), SHAPE), (dict(I=48), SHAPE), (dict(T=-1), SHAPE), (dict(O=0), SHAPE)])
def test_experts_refuse_what_lies_beyond_32_bits_only(lib, kw, status):
    """The kept rows and one expert's codes are limited, not the rows times the outputs, which nothing holds."""
    args = dict(E=4, T=131072, N=131072, O=8448, I=32)
    a = {**args, **kw}
    st = lib.sq_fwd_act4_batched(MX, *a.values(), FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1, None, 0, None)
    assert st == (status or ARG)                               # without offsets, where the shape is taken


# ---------------------------------------------------------------- distillation
HEAD = [(dict(head=3), FORMAT), (dict(T=-1), SHAPE), (dict(V=0), SHAPE), (dict(I=0), SHAPE), (dict(I=12), SHAPE),
        (dict(head=MX, I=48), SHAPE), (dict(K=0), SHAPE), (dict(K=257), SHAPE), (dict(T=1 << 25), SHAPE), (dict(I=1 << 22), SHAPE),
        (dict(X=None), ARG), (dict(W=None), ARG), (dict(head=MX, sc=None), ARG), (dict(head=NV, ws2=0.0), ARG),
        (dict(ids=None), ARG), (dict(ib=2), ARG), (dict(z=None), ARG), (dict(zd=2), ARG), (dict(tau=0.0), ARG),
        (dict(tau=-1.0), ARG), (dict(tau=math.nan), ARG), (dict(tau=math.inf), ARG), (dict(tau=2.0 ** -21), ARG),
        (dict(lse=None), ARG), (dict(picked=None), ARG), (dict(X=OFF), ALIGN), (dict(W=OFF), ALIGN),
        (dict(head=MX, W=FAKE + 2), ALIGN), (dict(ids=FAKE + 4), ALIGN), (dict(z=FAKE + 2), ALIGN), (dict(zd=1, z=FAKE + 1), ALIGN),
        (dict(lse=FAKE + 2), ALIGN), (dict(picked=FAKE + 2), ALIGN), (dict(), WORKSPACE), (dict(ws=FAKE, size=64), WORKSPACE),
        (dict(ws=FAKE + 16, size=1 << 40), ALIGN)]


@pytest.mark.parametrize("kw,status", HEAD + [(dict(loss=None), ARG), (dict(loss=FAKE + 2), ALIGN)])
def test_distill_fwd_refusals(lib, kw, status):
    args = dict(head=BF, T=16, V=100, I=64, K=4, X=FAKE, W=FAKE, sc=FAKE, ws2=1.0, ids=FAKE, ib=8, z=FAKE, zd=0, tau=1.0, loss=FAKE,
                lse=FAKE, picked=FAKE, ws=None, size=0, stream=None)
    assert _call(lib.sq_distill_fwd, args, kw) == status
    assert _call(lib.sq_distill_fwd, args, dict(T=0, X=None, ids=None, z=None, loss=None, lse=None, picked=None)) == 0


@pytest.mark.parametrize("kw,status", HEAD + [(dict(dl=None), ARG), (dict(dX=None), ARG), (dict(dxd=2), ARG), (dict(dX=OFF), ALIGN),
                                              (dict(dl=FAKE + 1), ALIGN)])
def test_distill_bwd_refusals(lib, kw, status):
    args = dict(head=BF, T=16, V=100, I=64, K=4, X=FAKE, W=FAKE, sc=FAKE, ws2=1.0, ids=FAKE, ib=8, z=FAKE, zd=0, tau=1.0, lse=FAKE,
                picked=FAKE, dl=FAKE, dX=FAKE, dxd=0, ws=None, size=0, stream=None)
    assert _call(lib.sq_distill_bwd, args, kw) == status


# ---------------------------------------------------------------- embedding
@pytest.mark.parametrize("kw,status", [
    (dict(head=3), FORMAT), (dict(T=-1), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 31) - 1), SHAPE), (dict(I=12), SHAPE),
    (dict(head=MX, I=48), SHAPE), (dict(ids=None), ARG), (dict(ib=3), ARG), (dict(W=None), ARG), (dict(head=MX, sc=None), ARG),
    (dict(head=NV, ws2=0.0), ARG), (dict(f=math.nan), ARG), (dict(f=math.inf), ARG), (dict(out=None), ARG), (dict(od=2), ARG),
    (dict(ids=FAKE + 4), ALIGN), (dict(W=OFF), ALIGN), (dict(head=MX, W=FAKE + 2), ALIGN), (dict(out=OFF), ALIGN),
])
def test_embed_refusals(lib, kw, status):
    args = dict(head=BF, T=16, V=100, I=64, ids=FAKE, ib=8, W=FAKE, sc=FAKE, ws2=1.0, f=1.0, out=FAKE, od=1, stream=None)
    assert _call(lib.sq_embed_fwd, args, kw) == status
    assert _call(lib.sq_embed_fwd, args, dict(T=0, ids=None, out=None)) == 0


BWD = [(dict(T=-1), SHAPE), (dict(V=0), SHAPE), (dict(I=12), SHAPE), (dict(ids=None), ARG), (dict(ib=3), ARG), (dict(d=None), ARG),
       (dict(dd=2), ARG), (dict(f=math.inf), ARG), (dict(grad=None), ARG), (dict(ids=FAKE + 4), ALIGN), (dict(d=OFF), ALIGN),
       (dict(grad=OFF), ALIGN), (dict(), WORKSPACE), (dict(ws=FAKE, size=16), WORKSPACE), (dict(ws=FAKE + 16, size=1 << 30), ALIGN)]


@pytest.mark.parametrize("kw,status", BWD + [(dict(gd=2), ARG)])
def test_embed_bwd_refusals(lib, kw, status):
    args = dict(T=16, V=100, I=64, ids=FAKE, ib=8, d=FAKE, dd=1, f=1.0, grad=FAKE, gd=0, ws=None, size=0, stream=None)
    assert _call(lib.sq_embed_bwd, args, kw) == status


@pytest.mark.parametrize("kw,status", BWD + [(dict(fmt=2), FORMAT), (dict(I=16), SHAPE), (dict(c=None), ARG), (dict(c=FAKE + 2), ALIGN)])
def test_embed_bwd_dscale_refusals(lib, kw, status):
    args = dict(fmt=MX, T=16, V=100, I=64, ids=FAKE, ib=8, d=FAKE, dd=1, f=1.0, c=FAKE, grad=FAKE, ws=None, size=0, stream=None)
    assert _call(lib.sq_embed_bwd_dscale, args, kw) == status


# ---------------------------------------------------------------- the largest sizes
@pytest.mark.parametrize("kw,status", [(dict(T=1 << 30), WORKSPACE), (dict(T=(1 << 30) + 1), SHAPE), (dict(I=1 << 26), WORKSPACE),
                                       (dict(I=(1 << 26) + 8), SHAPE)])
def test_embed_largest(lib, kw, status):
    args = dict(T=16, V=100, I=64, ids=FAKE, ib=8, d=FAKE, dd=1, f=1.0, grad=FAKE, gd=0, ws=None, size=0, stream=None)
    assert _call(lib.sq_embed_bwd, args, kw) == status
    assert (_call(lib.sq_embed_bwd_workspace, dict(T=16, V=100, I=64), kw) > 0) == (status == WORKSPACE)
    if status == SHAPE:
        args = dict(head=BF, T=16, V=100, I=64, ids=FAKE, ib=8, W=FAKE, sc=FAKE, ws2=1.0, f=1.0, out=FAKE, od=1, stream=None)
        assert _call(lib.sq_embed_fwd, args, kw) == SHAPE


@pytest.mark.parametrize("ws2,tau,status", [(1.0, 2.0 ** 20, WORKSPACE), (1.0, 2.0 ** -20, WORKSPACE), (2.0 ** 120, 2.0 ** -20, ARG),
                                            (2.0 ** 120, 2.0 ** 20, ARG), (2.0 ** -140, 2.0 ** 20, ARG), (2.0 ** -140, 2.0 ** -20, ARG)])
def test_distill_factors_stay_numbers(lib, ws2, tau, status):
    args = dict(head=NV, T=16, V=100, I=64, K=4, X=FAKE, W=FAKE, sc=FAKE, ws2=ws2, ids=FAKE, ib=8, z=FAKE, zd=0, tau=tau, loss=FAKE,
                lse=FAKE, picked=FAKE, ws=None, size=0, stream=None)
    assert _call(lib.sq_distill_fwd, args, {}) == status


# ---------------------------------------------------------------- binding
def test_binding_refuses_what_the_library_cannot_see():
    ensure_library()
    from paper_2609_04526_amd import sq
    u8, bf, i32 = torch.uint8, torch.bfloat16, torch.int32
    X = torch.zeros((4, 64), dtype=bf)
    x, xs = torch.zeros((4, 32), dtype=u8), torch.zeros((4, 2), dtype=u8)
    c, s = torch.zeros((8, 32), dtype=u8), torch.zeros((8, 2), dtype=u8)
    with pytest.raises(ValueError, match="device tensors"):
        sq.sq_act4_pack("mx", X)
    with pytest.raises(ValueError, match="bfloat16"):
        sq.sq_act4_pack("mx", X.float())
    with pytest.raises(ValueError, match="multiple"):
        sq.sq_act4_pack("mx", torch.zeros((4, 48), dtype=bf))
    with pytest.raises(ValueError, match="contiguous"):
        sq.sq_act4_pack("mx", torch.zeros((64, 4), dtype=bf).t())
    with pytest.raises(ValueError, match="scales"):
        sq.sq_act4_unpack("mx", x, xs[:, :1])
    with pytest.raises(ValueError, match="unknown format"):
        sq.sq_act4_unpack("fp4", x, xs)
    with pytest.raises(ValueError, match="codes"):
        sq.sq_fwd_act4("mx", x, xs, c[:, :16].contiguous(), s)
    with pytest.raises(ValueError, match="Y"):
        sq.sq_fwd_act4("mx", x, xs, c, s, out_dtype=torch.float16)
    with pytest.raises(ValueError, match="x_scales"):
        sq.sq_fwd_act4("nv", x, xs, c, s)
    with pytest.raises(ValueError, match="3-D"):
        sq.sq_fwd_act4_batched("mx", x, xs, None, torch.zeros(2, dtype=i32), c, s)
    with pytest.raises(ValueError, match="offsets"):
        sq.sq_fwd_act4_batched("mx", x, xs, None, torch.zeros(3, dtype=i32), c[None], s[None])
    with pytest.raises(ValueError, match="rows"):
        sq.sq_fwd_act4_batched("mx", x, xs, torch.zeros(4), torch.zeros(2, dtype=i32), c[None], s[None])
    W, ids, z = torch.zeros((10, 64), dtype=bf), torch.zeros((4, 3), dtype=torch.int64), torch.zeros((4, 3))
    with pytest.raises(ValueError, match="device tensors"):
        sq.sq_distill_fwd("bf16", X, W, ids, z)
    with pytest.raises(ValueError, match="logits"):
        sq.sq_distill_fwd("bf16", X, W, ids, z[:, :2].contiguous())
    with pytest.raises(ValueError, match="ids"):
        sq.sq_distill_fwd("bf16", X, W, ids.float(), z)
    with pytest.raises(ValueError, match="scales"):
        sq.sq_distill_fwd("mx", X, c, ids, z)
    with pytest.raises(ValueError, match="picked"):
        sq.sq_distill_bwd("bf16", X, W, ids, z, torch.zeros(4), torch.zeros(4), torch.zeros(4))
    with pytest.raises(ValueError, match="ids"):
        sq.sq_embed_fwd("bf16", ids, W)
    with pytest.raises(ValueError, match="device tensors"):
        sq.sq_embed_fwd("bf16", ids[:, 0].contiguous(), W)
    with pytest.raises(ValueError, match="out"):
        sq.sq_embed_fwd("bf16", ids[:, 0].contiguous(), W, out_dtype=torch.float16)
    with pytest.raises(ValueError, match="dOut"):
        sq.sq_embed_bwd(ids[:, 0].contiguous(), X[:3], 10)
    with pytest.raises(ValueError, match="dW"):
        sq.sq_embed_bwd(ids[:, 0].contiguous(), X, 10, dW=torch.zeros((9, 64)))
    with pytest.raises(ValueError, match="codes"):
        sq.sq_embed_bwd_dscale("mx", ids[:, 0].contiguous(), X, c[:, :8].contiguous())


def test_binding_imports_under_a_torch_without_a_gpu_build():
    """Such a torch lacks the runtime's own calls; the host's checks work there all the same."""
    code = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2609_04526_amd import sq
try:
    sq.sq_act4_pack("mx", torch.zeros((4, 64), dtype=torch.bfloat16))
except ValueError as e:
    print("refused:", e)
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr
    assert "refused: libscaleqlora takes device tensors" in done.stdout
