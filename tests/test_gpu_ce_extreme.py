"""Cross entropy where logits reach the end of fp32's range, are infinite or are
NaN, through every form of the kernels: tiles of 64 tokens and of more, heads
read as bf16, from their codes, by the layer's own products, and sums over the
width in planes.

Each logit here is one product of two bf16 values beside zeros, so it is exact,
and a token's logits are x times one column of W.

Bounds.  l - top is rounded once (2^-24 of it), the exponential's argument twice
more: p is off by 2^-22 |d| e^-|d| < 2^-23 of 1 and by its own steps, the sum by
that and its depth; log adds its own.  So lse is off by 2^-22 |lse| + 2^-16 and
loss by 2^-22 |loss| + 2^-16.  The gradient takes lse as it is held, 2^-24 of it
off, which moves p by p 2^-22 |lse| as long as that is small: 2^-6 for |lse| up to
2^16.  Beyond that p is 0 or 1 here: the logits nearest the largest differ from it
by a tenth of it and more."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import linear, step
from paper_2609_04526_amd import inputs
from parity_check import gamma

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16 = torch.bfloat16
WS2 = 2.0
# few tokens and compact rows; widths of codes, of the layer's products and of planes
FORMS = [("bf16", 7, 300, 32), ("bf16", 300, 700, 96), ("bf16", 1500, 5000, 64), ("bf16", 40, 513, 1088), ("bf16", 400, 513, 1088),
         ("mx", 7, 299, 96), ("mx", 300, 3003, 512), ("mx", 130, 33333, 512), ("mx", 400, 700, 96),
         ("nv", 7, 299, 96), ("nv", 300, 3003, 512), ("nv", 400, 513, 1088)]


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _head(head, V, I):
    """Operands of a head whose column 0 is 3/4 at row V // 3, 1 at row V // 2 and 7/8 elsewhere (4-bit: 3/8, 3/4 and 1/2), its
    other columns at most 3/4, and its fp64 values."""
    g = inputs.rng(V + I)
    if head == "bf16":
        w = g.integers(-8, 9, (V, I)) / 64.0
        w[:, 0] = 0.875
        w[V // 3, 0], w[V // 2, 0] = 0.75, 1.0
        return torch.from_numpy(w).to(BF16).cuda(), None, w
    codes = inputs.codes_uniform(V, V, I)
    first = np.full(V, 6, np.uint8)                            # 4
    first[V // 3], first[V // 2] = 5, 7                        # 3 and 6
    codes[:, 0] = codes[:, 0] & 0xF0 | first
    if head == "mx":
        sc = np.full((V, I // 32), 127 - 3, np.uint8)          # 1/8
        w = linear.dequant("mx", codes, sc)
    else:
        sc = torch.full((V, I // 16), 0.0625).to(torch.float8_e4m3fn).view(torch.uint8).numpy()    # ws2 / 16 = 1/8
        w = linear.dequant("nv", codes, sc, WS2)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(sc).cuda(), w


def _run(sq, head, X, W, scales, y, dloss, ws2=WS2):
    Xd, yd = X.to(BF16).cuda(), torch.from_numpy(y).cuda()
    loss, lse = sq.sq_ce_fwd(head, Xd, W, yd, scales=scales, ws2=ws2)
    dX = sq.sq_ce_bwd(head, Xd, W, yd, lse, torch.from_numpy(dloss).cuda(), scales=scales, ws2=ws2)
    return loss.double().cpu().numpy(), lse.double().cpu().numpy(), dX.double().cpu().numpy()


@pytest.mark.parametrize("head,T,V,I", FORMS)
def test_large_finite_logits(sq, head, T, V, I):
    """Logits of +-1 to +-3.2e38, the largest of them past 2^128 / log2(e)."""
    W, scales, w = _head(head, V, I)
    top = w[V // 2, 0]
    size = np.array([1.0, 30.0, 1e4, 1e6, 1e10, 1e30, 3.2e38 / max(top, 1.0)])
    x = torch.from_numpy(np.concatenate([size, -size])[np.arange(T) % 14]).to(BF16).double().numpy()
    X = np.zeros((T, I))
    X[:, 0] = x
    y = np.array([V // 2, V // 3, 0, V - 1])[np.arange(T) // 2 % 4]
    y[::9] = -1
    dloss = inputs.rng(T).standard_normal(T).astype(np.float32)
    loss, lse, dX = _run(sq, head, torch.from_numpy(X), W, scales, y, dloss)
    r_loss, r_lse = step.ce_fwd(X, w, y)
    assert (np.abs(lse - r_lse) <= 2.0 ** -22 * np.abs(r_lse) + 2.0 ** -16).all()
    assert (np.abs(loss - r_loss) <= 2.0 ** -22 * np.abs(r_loss) + 2.0 ** -16).all()
    l = X @ w.T
    valid = y >= 0
    soft = np.where(np.abs(l).max(1) <= 2.0 ** 16, 2.0 ** -22 * np.abs(l).max(1), 0.0)     # p through lse as fp32 holds it
    p = np.exp(l - l.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    p[np.flatnonzero(valid), y[valid]] += 1.0
    d = (2.0 ** -8 + 2.0 ** -16 + 2 * gamma(V + 70) + soft)[:, None] * p
    bound = np.abs(dloss)[:, None] * (d @ np.abs(w)) * 1.01 + 1e-30
    assert (np.abs(dX - step.ce_bwd(X, w, y, dloss)) <= np.where(valid[:, None], bound, 0)).all()


@pytest.mark.parametrize("head,T,V,I", FORMS)
def test_logits_that_are_not_finite(sq, head, T, V, I):
    """A NaN and an infinite logit give NaN in their own token's loss, lse and gradient, and nothing else changes."""
    W, scales, w = _head(head, V, I)
    g = inputs.rng(T + 1)
    X = torch.from_numpy(g.integers(-8, 9, (T, I)) / 8.0).to(BF16)
    y, dloss = g.integers(0, V, T), g.standard_normal(T).astype(np.float32)
    base = _run(sq, head, X, W, scales, y, dloss)
    assert all(np.isfinite(b).all() for b in base)
    bad = X.clone()
    bad[1, 0], bad[T - 1, 3], bad[4, 0] = float("nan"), float("-inf"), float("inf")
    got = _run(sq, head, bad, W, scales, y, dloss)
    rows = np.array([1, 4, T - 1])
    rest = np.setdiff1d(np.arange(T), rows)
    for a, b in zip(got, base):
        assert np.isnan(a[rows]).all() and np.array_equal(a[rest], b[rest])


@pytest.mark.parametrize("T", [5, 300])
def test_a_logit_of_minus_infinity_beside_finite_ones(sq, T):
    """A product past fp32's range: probability 0, an infinite loss where it is the target, and a finite gradient."""
    V, I = 300, 32
    w = inputs.rng(2).integers(-8, 9, (V, I)) / 64.0
    w[:, 1] = 0.0
    w[7, 1] = -(2.0 ** 120)
    W = torch.from_numpy(w).to(BF16).cuda()
    X = np.zeros((T, I))
    X[:, 0], X[:, 1] = 1.0, 0.0
    X[0, 1] = X[T - 1, 1] = 2.0 ** 120
    y = np.arange(T) % V
    y[0] = 7
    loss, lse, dX = _run(sq, "bf16", torch.from_numpy(X), W, None, y, np.ones(T, np.float32))
    keep = np.arange(V) != 7
    l = (X @ w.T)[:, keep]
    want = np.log(np.exp(l[[0, T - 1]]).sum(1))
    assert np.abs(lse[[0, T - 1]] - want).max() <= 2.0 ** -16 + 2.0 ** -22 * want.max()
    assert loss[0] == np.inf and np.isfinite(loss[1:]).all() and np.isfinite(dX).all()


@pytest.mark.parametrize("T", [5, 300])
def test_ws2_that_takes_logits_past_the_range(sq, T):
    """The sums are finite, the logits, ws2 times that, are not: NaN, as for any infinite logit."""
    V, I = 300, 64
    W, scales, w = _head("nv", V, I)
    X = np.zeros((T, I))
    X[:, 0] = 1.0
    X[1, 0] = 2.0 ** 120
    loss, lse, dX = _run(sq, "nv", torch.from_numpy(X), W, scales, np.arange(T) % V, np.ones(T, np.float32), ws2=1024.0)
    for a in (loss, lse, dX):
        assert np.isnan(a[1]).all() and np.isfinite(np.delete(a, 1, 0)).all()
