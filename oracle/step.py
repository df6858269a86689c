"""Oracle of what a training step runs around the frozen-code products (test
infrastructure only): tokens sorted by expert and back, 8-bit activation
checkpoints, and softmax cross entropy of a language-model head.

Plain numpy in float64, written from the definitions:

  sort      key(p) = ids[p] if it is an expert, else E; a stable sort of the
            pairs p = t*K + k by key; slot[p] is pair p's place
  gather    Xs[slot[p]] = X[p // K] for routed pairs, else 0
  combine   out[t] = sum_k w[t,k] Ys[slot[t,k]] over routed pairs
  keep      blocks of 32 columns with a power-of-two scale 2^k: int8
            k = floor(log2 amax) - 6, or E4M3 k = ceil(log2(amax / 448)), k
            held in [-126, 127]; a block with an Inf or NaN reads as NaN
  ce        l = X W^T; lse = log sum exp l; loss = lse - l[target];
            dX = dloss (softmax(l) - onehot(target)) W; rows whose target is
            not in the vocabulary give zeros
"""

import numpy as np

from . import codec

ACT_BLOCK = 32


# ---------------------------------------------------------------- experts
def moe_sort(ids, E):
    """(offsets [E+1], token [N], slot [T, K])."""
    T, K = ids.shape
    pairs = [[] for _ in range(E + 1)]
    for p, e in enumerate(np.asarray(ids).reshape(-1).tolist()):
        pairs[e if 0 <= e < E else E].append(p)
    order = [p for group in pairs for p in group]
    slot = np.empty(T * K, np.int32)
    slot[order] = np.arange(T * K)
    offsets = np.concatenate([[0], np.cumsum([len(g) for g in pairs[:E]])]).astype(np.int32)
    return offsets, (np.array(order, np.int64) // K).astype(np.int32), slot.reshape(T, K)


def moe_gather(X, slot, routed):
    T, K = slot.shape
    out = np.zeros((T * K, X.shape[1]))
    for t in range(T):
        for k in range(K):
            if slot[t, k] < routed:
                out[slot[t, k]] = X[t]
    return out


def moe_combine(Ys, slot, routed, w=None):
    T, K = slot.shape
    out = np.zeros((T, Ys.shape[1]))
    for t in range(T):
        for k in range(K):
            if slot[t, k] < routed:
                out[t] += (1.0 if w is None else float(w[t, k])) * Ys[slot[t, k]]
    return out


def moe_combine_bwd(dOut, Ys, slot, routed, w):
    T, K = slot.shape
    dYs, dw = np.zeros((T * K, Ys.shape[1])), np.zeros((T, K))
    for t in range(T):
        for k in range(K):
            if slot[t, k] < routed:
                dYs[slot[t, k]] = float(w[t, k]) * dOut[t]
                dw[t, k] = dOut[t] @ Ys[slot[t, k]]
    return dYs, dw


# ---------------------------------------------------------------- 8-bit activations
_E4M3 = np.array([codec.e4m3_value(b) for b in range(127)])        # 0 .. 448, increasing


def _e4m3_nearest(v):
    """E4M3 bytes of |v| <= 448, ties to the even byte."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_E4M3, a), 1, 126)
    lo = hi - 1
    d_lo, d_hi = a - _E4M3[lo], _E4M3[hi] - a
    up = (d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0))
    return (np.where(up, hi, lo) | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def act_pack(act, X):
    """codes uint8 [T, I], scale bytes uint8 [T, I/32]."""
    T, I = X.shape
    x = np.asarray(X, np.float64).reshape(T, I // ACT_BLOCK, ACT_BLOCK)
    codes = np.zeros(x.shape, np.uint8)
    scales = np.zeros(x.shape[:2], np.uint8)
    for t in range(T):
        for b in range(x.shape[1]):
            v = x[t, b]
            if not np.isfinite(v).all():
                scales[t, b] = 255
                continue
            amax = np.abs(v).max()
            if amax == 0:
                k = -126
            elif act == "int8":
                k = int(np.frexp(amax)[1]) - 1 - 6
            else:
                m, e = np.frexp(amax / 448.0)           # amax has 8 bits: the quotient's log is exact enough to ceil
                k = int(e) - 1 if amax == np.ldexp(448.0, int(e) - 1) else int(e)
            k = min(max(k, -126), 127)
            q = np.ldexp(v, -k)
            if act == "int8":
                codes[t, b] = np.clip(np.rint(q), -127, 127).astype(np.int8).view(np.uint8)
            else:
                codes[t, b] = _e4m3_nearest(q)
            scales[t, b] = k + 127
    return codes.reshape(T, I), scales


def act_unpack(act, codes, scales):
    T, I = codes.shape
    if act == "int8":
        v = codes.view(np.int8).astype(np.float64)
    else:
        v = np.array([codec.e4m3_value(b) for b in range(256)])[codes]
    f = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(f, ACT_BLOCK, axis=1)


# ---------------------------------------------------------------- cross entropy
def ce_fwd(X, W, targets):
    """(loss, lse), zeros for rows whose target is outside the vocabulary."""
    X, W = np.asarray(X, np.float64), np.asarray(W, np.float64)
    l = X @ W.T
    top = l.max(axis=1, keepdims=True)
    lse = (top + np.log(np.exp(l - top).sum(axis=1, keepdims=True)))[:, 0]
    valid = (targets >= 0) & (targets < W.shape[0])
    at = np.where(valid, targets, 0)
    loss = lse - l[np.arange(len(l)), at]
    return np.where(valid, loss, 0.0), np.where(valid, lse, 0.0)


def ce_bwd(X, W, targets, dloss):
    X, W = np.asarray(X, np.float64), np.asarray(W, np.float64)
    l = X @ W.T
    p = np.exp(l - l.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    valid = (targets >= 0) & (targets < W.shape[0])
    for t in np.flatnonzero(valid):
        p[t, targets[t]] -= 1.0
    return np.where(valid[:, None], np.asarray(dloss, np.float64)[:, None] * (p @ W), 0.0)
