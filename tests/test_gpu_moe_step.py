"""The example's training step (sort, gather, grouped products, combine, loss
and back, with the products' inputs kept in 8 bits) against the oracle's chain
in 64 bits.

Bound, by norm.  The chain rounds to bf16 at most ten times on the way to any
result (Z, dZ, the logits' gradients, Ys, dYs, U, A, dA, dU, dXs), each 2^-8 of
its value at most; the squares of U count twice, and an error e of Z moves a
logit by e of its size and the probabilities by that: logits here stay below 8.
The hidden rows that are kept hold 8 bits: int8 blocks are off by half a step of
2^-6 of their largest value, so by about 2^-7 of 3 standard deviations at most;
E4M3 by 2^-4 of a value."""

import importlib.util
import os

import numpy as np
import pytest
import torch

from conftest import ROOT, ensure_library, gpu_ready
from oracle import linear, step

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BOUND = 12 * 2.0 ** -8 + 8 * 2.0 ** -8
KEPT = {"int8": 3 * 2.0 ** -7, "e4m3": 2.0 ** -4}


@pytest.fixture(scope="module")
def example():
    ensure_library()
    spec = importlib.util.spec_from_file_location("moe_step", os.path.join(ROOT, "examples", "moe_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _np(t):
    return t.double().cpu().numpy()


def _values(codes, scales):
    return np.stack([linear.dequant("mx", c, s) for c, s in zip(codes.cpu().numpy(), scales.cpu().numpy())])


def _off(got, want):
    return np.linalg.norm(_np(got) - want) / np.linalg.norm(want)


@pytest.mark.parametrize("T,K,E,H,F,V,head,act", [(60, 2, 5, 128, 96, 301, "mx", "int8"), (333, 3, 8, 96, 160, 1000, "mx", "e4m3"),
                                                  (20, 1, 24, 64, 32, 77, "bf16", "int8")])
def test_step(example, T, K, E, H, F, V, head, act):
    layer, X, ids, w, y = example.synthetic(T, T, K, E, H, F, V, head)
    ids[::7, 0] = -1                                     # dropped pairs
    loss, g = example.step(layer, X, ids, w, y, act)

    up, down = _values(layer.up, layer.up_scales), _values(layer.down, layer.down_scales)
    W = _np(layer.W) if head == "bf16" else linear.dequant("mx", layer.W.cpu().numpy(), layer.head_scales.cpu().numpy())
    x, yn, wn = _np(X), y.cpu().numpy(), _np(w)
    offsets, token, slot = step.moe_sort(ids.cpu().numpy(), E)
    R = offsets[E]
    xs = step.moe_gather(x, slot, R)
    U, Ys = np.zeros((T * K, F)), np.zeros((T * K, H))
    spans = [slice(a, b) for a, b in zip(offsets[:-1], offsets[1:])]
    for e, s in enumerate(spans):
        U[s] = xs[s] @ up[e].T
        Ys[s] = np.maximum(U[s], 0) ** 2 @ down[e].T
    A = np.maximum(U, 0) ** 2
    z = x + step.moe_combine(Ys, slot, R, wn)
    losses, _ = step.ce_fwd(z, W, yn)
    live = (yn >= 0) & (yn < V)
    share = live / max(live.sum(), 1)
    assert abs(loss.item() - (losses * share).sum()) <= 8 * 2.0 ** -8 * 8
    dz = step.ce_bwd(z, W, yn, share)
    dYs, dw = step.moe_combine_bwd(dz, Ys, slot, R, wn)
    kept = step.act_unpack(act, *step.act_pack(act, x))
    dU, dxs = np.zeros_like(U), np.zeros_like(Ys)
    d_up, d_down = [], []
    for e, s in enumerate(spans):
        d_down.append(linear.backward_dscale("mx", A[s], dYs[s], layer.down[e].cpu().numpy()))
        dU[s] = dYs[s] @ down[e] * 2 * np.maximum(U[s], 0)
        d_up.append(linear.backward_dscale("mx", kept[token[s]], dU[s], layer.up[e].cpu().numpy()))
        dxs[s] = dU[s] @ up[e]
    assert _off(g.weights, dw) <= BOUND
    assert _off(g.down_scales, np.stack(d_down)) <= BOUND + KEPT[act]
    assert _off(g.up_scales, np.stack(d_up)) <= BOUND
    assert _off(g.X, dz + step.moe_combine(dxs, slot, R)) <= BOUND
    assert (_np(g.weights)[::7, 0] == 0).all()
