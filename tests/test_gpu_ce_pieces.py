"""Cross entropy over a vocabulary of several pieces, in each form that takes
pieces: the gradient from bf16 rows and from MXFP4 codes, both directions of a
4-bit head written out in bf16, the logits of the layer's own products.  Targets
lie on both sides of every multiple of 256, so on both sides of every piece's
ends, the last piece is ragged, and some tokens are ignored.

The tokens compared are those whose targets lie there and some others; bounds as
for one piece: a logit is an fp32 sum of I exact products, off by a = gamma_I sum
|x w| at most, lse by max a and its own steps (|top| + 64) 2^-22, loss by the
target's logit too; a logit's gradient by c p (2 a + the same) and its rounding to
bf16, dX by its fp32 sum over V and the rounding of its type."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from paper_2609_04526_amd import inputs
from parity_check import gamma

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16, F64 = torch.bfloat16, torch.float64
BLOCK = {"mx": 32, "nv": 16}
WS2 = float(np.float32(1.0 / 448.0))
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _head(head, V, I, offset):
    """Operands of a head whose logits are a few units wide, its codes `offset` bytes past an aligned address, and its values."""
    gen = inputs.device_generator(V)
    if head == "bf16":
        W = (torch.randn((V, I), generator=gen, device="cuda") * (2 / I ** 0.5)).to(BF16)
        return W, None, W
    base = torch.randint(0, 256, (V * I // 2 + 16,), generator=gen, device="cuda", dtype=torch.uint8)
    codes = base[offset:offset + V * I // 2].view(V, I // 2)
    if head == "mx":
        e = int(np.round(np.log2(1 / np.sqrt(I))))
        scales = torch.randint(e + 126, e + 129, (V, I // 32), generator=gen, device="cuda", dtype=torch.uint8)
        eff = torch.exp2(scales.to(F64) - 127)
    else:
        s = torch.rand((V, I // 16), generator=gen, device="cuda") * (448.0 / I ** 0.5)
        scales = s.to(torch.float8_e4m3fn).view(torch.uint8)
        eff = scales.view(torch.float8_e4m3fn).to(F64) * WS2
    table = torch.tensor(E2M1 + [-v for v in E2M1], dtype=F64, device="cuda")
    w = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).view(V, -1, BLOCK[head])
    return codes, scales, (w * eff[..., None]).view(V, I)


def _targets(T, V):
    """Both sides of every multiple of 256 first, then any; every 7th ignored."""
    edges = np.arange(0, V + 256, 256)
    edges = np.unique(np.clip(np.concatenate([edges - 1, edges]), 0, V - 1))
    g = inputs.rng(T)
    y = np.concatenate([g.permutation(edges), g.integers(0, V, T)])[:T]
    y[::7] = np.where(np.arange(0, T, 7) % 2 == 0, -100, V)
    return y


@pytest.mark.parametrize("head,T,V,I,offset", [
    ("bf16", 5000, 60001, 256, 0),        # gradient: 26624 rows a piece
    ("mx", 4000, 70001, 512, 0),          # gradient from codes
    ("mx", 4000, 70001, 512, 4),          # the same written out in bf16
    ("mx", 600, 300001, 1056, 0),         # both directions written out
    ("mx", 600, 300001, 1024, 4),
    ("nv", 600, 300001, 1024, 0),
    ("nv", 256, 200001, 64, 0),           # the layer's products, logits in pieces
    ("mx", 200, 300003, 96, 0),
])
def test_pieces(sq, head, T, V, I, offset):
    W, scales, w = _head(head, V, I, offset)
    if T > 256:
        assert T * V * 2 > 256 << 20                           # the logits' gradients of more than one piece
    if head != "bf16" and (T <= 256 or I > 512):               # less than all of the logits, or than the head in bf16
        assert sq.sq_ce_fwd_workspace(head, T, V, I) < (T * V * 4 if T <= 256 else V * I * 2)
    X, y = inputs.device_bf16_normal(T, (T, I)), _targets(T, V)
    yd = torch.from_numpy(y).cuda()
    dloss = torch.randn(T, generator=inputs.device_generator(T + 1), device="cuda")
    loss, lse = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    sq.sq_ce_fwd(head, X, W, yd, scales=scales, ws2=WS2, loss=loss, lse=lse)
    dX = torch.full((T, I), float("nan"), device="cuda")
    sq.sq_ce_bwd(head, X, W, yd, lse, dloss, scales=scales, ws2=WS2, dX=dX)

    valid = (yd >= 0) & (yd < V)
    assert (loss[~valid] == 0).all() and (lse[~valid] == 0).all() and (dX[~valid] == 0).all()
    assert torch.isfinite(dX).all()
    edges = np.flatnonzero((y >= 0) & (y < V) & ((y % 256 == 0) | (y % 256 == 255)))
    pick = torch.from_numpy(np.unique(np.concatenate([edges[:500], np.arange(0, T, T // 100), [T - 1]]))).cuda()
    pick = pick[valid[pick]]
    for p in pick.split(64):
        x, t = X[p].to(F64), yd[p][:, None]
        l = torch.zeros((len(p), V), dtype=F64, device="cuda")
        mag = torch.zeros(len(p), dtype=F64, device="cuda")
        rows = [w[a:a + 65536].to(F64) for a in range(0, V, 65536)]
        for a, r in zip(range(0, V, 65536), rows):
            l[:, a:a + 65536] = x @ r.t().contiguous()
            mag = torch.maximum(mag, (x.abs() @ r.abs().t().contiguous()).amax(1))
        z = torch.logsumexp(l, 1)
        at = l.gather(1, t)[:, 0]
        a_err, own = 2 * gamma(I + 2) * mag, (l.abs().amax(1) + 64) * 2.0 ** -22
        assert ((lse[p] - z).abs() <= a_err + own).all()
        assert ((loss[p] - (z - at)).abs() <= 2 * a_err + 2 * own).all()
        q = torch.exp(l - z[:, None])
        hot = torch.zeros_like(q).scatter_(1, t, 1.0)
        c = dloss[p].to(F64)[:, None]
        d_err = c.abs() * (q * (2 * a_err + 2 * own)[:, None] + (2.0 ** -8 + 2.0 ** -20) * (q - hot).abs() + 2 * gamma(V + 100) * (q + hot))
        want, bound = torch.zeros_like(x), torch.zeros_like(x)
        for a, r in zip(range(0, V, 65536), rows):
            want += (c * (q - hot))[:, a:a + 65536].contiguous() @ r
            bound += d_err[:, a:a + 65536].contiguous() @ r.abs()
        assert ((dX[p] - want).abs() <= bound + 2.0 ** -22 * want.abs() + 1e-30).all()


def test_gradient_of_codes_in_pieces_equals_that_of_bf16_values(sq):
    T, V, I = 4000, 70001, 512
    codes, scales, w = _head("mx", V, I, 0)
    X, yd = inputs.device_bf16_normal(3, (T, I)), torch.from_numpy(_targets(T, V)).cuda()
    W = w.to(BF16)
    assert torch.equal(W.to(F64), w)
    _, lse = sq.sq_ce_fwd("bf16", X, W, yd)
    dloss = torch.randn(T, generator=inputs.device_generator(4), device="cuda")
    assert torch.equal(sq.sq_ce_bwd("mx", X, codes, yd, lse, dloss, scales=scales), sq.sq_ce_bwd("bf16", X, W, yd, lse, dloss))
