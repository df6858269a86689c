"""Oracle of a 4-bit student's operators (test infrastructure only), plain numpy
in float64 from the definitions:

  act4      an activation in the layer's 4-bit storage: the nearest-even
            re-quantisation of each block, a block with an Inf or NaN as the NaN
            scale and zero codes
  experts   rows [offsets[e], offsets[e+1]) of Y are picked rows of x^ times
            expert e's weight; rows that no expert has are zeros
  distill   s = X W^T / tau; q = softmax over the entries that count of z / tau;
            loss = tau^2 sum q (log q - s[id] + lse);
            dX = dloss tau (softmax(s) - scatter(q)) W
  embed     rows of the table times a factor, and the sums of dOut by id
"""

import numpy as np

from . import codec, linear, rtn


# ---------------------------------------------------------------- 4-bit activations
def act4_pack(fmt, X, ws2=1.0):
    """codes uint8 [T, I/2], scale bytes uint8 [T, I/B] of X [T, I] (values exact in bf16)."""
    X = np.asarray(X, np.float32)
    B = codec.BLOCK[fmt]
    T, I = X.shape
    bad = ~np.isfinite(X.reshape(T, I // B, B)).all(-1)
    clean = np.where(np.repeat(bad, B, axis=1), np.float32(0), X)
    codes, scales, _ = rtn.quantize(fmt, clean, rtn.TIE_EVEN, ws2=np.float32(ws2))
    scales = np.where(bad, 0xFF if fmt == "mx" else 0x7F, scales).astype(np.uint8)
    codes = np.where(np.repeat(bad, B // 2, axis=1), 0, codes).astype(np.uint8)
    return codes, scales


def act4_values(fmt, codes, scales, ws2=1.0):
    return linear.dequant(fmt, codes, scales, ws2)


def experts(x, rows, offsets, W):
    """x [T, I] values, rows int [N], W [E, O, I] values -> Y [N, O]."""
    Y = np.zeros((len(rows), W.shape[1]))
    for e in range(W.shape[0]):
        a, b = (min(max(int(v), 0), len(rows)) for v in offsets[e:e + 2])
        for s in range(a, b):
            if 0 <= rows[s] < len(x):
                Y[s] = W[e] @ x[rows[s]]
    return Y


# ---------------------------------------------------------------- distillation
def teacher(ids, z, tau, V):
    """(which entries count [T, K], their probabilities [T, K])."""
    counts = (ids >= 0) & (ids < V) & ~np.isneginf(z)
    s = np.where(counts, np.asarray(z, np.float64) / tau, -np.inf)
    top = np.where(counts.any(1), s.max(1), 0.0)[:, None]
    q = np.where(counts, np.exp(s - top), 0.0)
    return counts, q / np.where(counts.any(1), q.sum(1), 1.0)[:, None]


def distill_fwd(X, W, ids, z, tau):
    """(loss [T], lse [T], picked [T, K])."""
    s = np.asarray(X, np.float64) @ np.asarray(W, np.float64).T / tau
    counts, q = teacher(ids, z, tau, len(W))
    top = s.max(1, keepdims=True)
    lse = (top + np.log(np.exp(s - top).sum(1, keepdims=True)))[:, 0]
    picked = np.where(counts, np.take_along_axis(s, np.where(counts, ids, 0), 1), 0.0)
    log_q = np.log(np.where(q > 0, q, 1.0))
    loss = tau ** 2 * np.where(q > 0, q * (log_q - picked + lse[:, None]), 0.0).sum(1)
    live = counts.any(1)
    return np.where(live, loss, 0.0), np.where(live, lse, 0.0), picked


def distill_bwd(X, W, ids, z, tau, dloss):
    W = np.asarray(W, np.float64)
    s = np.asarray(X, np.float64) @ W.T / tau
    counts, q = teacher(ids, z, tau, len(W))
    p = np.exp(s - s.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    for t, k in zip(*np.nonzero(counts)):
        p[t, ids[t, k]] -= q[t, k]
    return np.where(counts.any(1), np.asarray(dloss, np.float64) * tau, 0.0)[:, None] * (p @ W)


# ---------------------------------------------------------------- embedding
def embed_fwd(ids, W, factor):
    W = np.asarray(W, np.float64)
    live = (ids >= 0) & (ids < len(W))
    return np.where(live[:, None], factor * W[np.where(live, ids, 0)], 0.0)


def embed_bwd(ids, dOut, V, factor):
    dW = np.zeros((V, dOut.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < V:
            dW[v] += np.asarray(dOut[t], np.float64)
    return factor * dW


def embed_bwd_dscale(fmt, ids, dOut, codes, factor):
    c = linear.code_values(codes)
    return (c * embed_bwd(ids, dOut, len(c), factor)).reshape(len(c), -1, codec.BLOCK[fmt]).sum(-1)
