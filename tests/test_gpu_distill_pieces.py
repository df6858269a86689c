"""Distillation over a vocabulary of several pieces, in each form that takes
pieces: the gradient from bf16 rows and from MXFP4 codes, both directions of a
4-bit head written out in bf16, the logits of the layer's own products.  Entries
lie on both sides of every multiple of 256, so on both sides of every piece's
ends and in pieces behind the first, with which what their rounding loses is kept;
some come twice, some are left out, some tokens have none.

Bounds as for one piece: a logit is an fp32 sum of I exact products over tau, off by
a = 2 gamma_I sum |x w| / tau at most; lse moves by the largest a and its own steps,
own = (|s| + 64) 2^-22; the teacher's q are off by b = (d + 16 + log K) 2^-22 of
themselves, d = |z - top| / tau; the loss is tau^2 times a q-weighted sum of those; a
logit's gradient is off by p (2 a + 2 own) + q b and rounded to bf16, dX by its fp32
sum over V and its last rounding."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import student
from paper_2609_04526_amd import inputs
from parity_check import gamma
from test_gpu_ce_pieces import WS2, _head

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

F64 = torch.float64
K, TAU = 12, 1.5


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    yield _sq
    torch.cuda.empty_cache()


def _entries(T, V):
    """ids int64 and logits fp32 [T, K]."""
    g = inputs.rng(T + V)
    edges = np.arange(0, V + 256, 256)
    edges = np.unique(np.clip(np.concatenate([edges - 1, edges]), 0, V - 1))
    ids = np.where(g.random((T, K)) < 0.6, g.choice(edges, (T, K)), g.integers(0, V, (T, K)))
    ids[::3, 5] = ids[::3, 4]
    ids[::4, 9:] = -1
    ids[::7] = V
    z = -np.sort(-3.0 * g.standard_normal((T, K)), axis=1)
    return ids, z.astype(np.float32)


@pytest.mark.parametrize("head,T,V,I,offset", [
    ("bf16", 5000, 60001, 256, 0),        # gradient: 26624 rows a piece
    ("mx", 4000, 70001, 512, 0),          # gradient from codes
    ("mx", 4000, 70001, 512, 4),          # the same written out in bf16
    ("mx", 600, 300001, 1056, 0),         # both directions written out
    ("nv", 600, 300001, 1024, 0),
    ("nv", 256, 200001, 64, 0),           # the layer's products, logits in pieces
    ("mx", 200, 300003, 96, 0),
])
def test_pieces(sq, head, T, V, I, offset):
    W, scales, w = _head(head, V, I, offset)
    if T > 256:
        assert T * V * 2 > 256 << 20                           # the logits' gradients of more than one piece
    X = inputs.device_bf16_normal(T, (T, I))
    ids, z = _entries(T, V)
    idd, zd = torch.from_numpy(ids).cuda(), torch.from_numpy(z).cuda()
    dloss = torch.randn(T, generator=inputs.device_generator(T + 1), device="cuda")
    more = dict(temperature=TAU, scales=scales, ws2=WS2)
    loss, lse = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    _, _, picked = sq.sq_distill_fwd(head, X, W, idd, zd, loss=loss, lse=lse, **more)
    dX = torch.full((T, I), float("nan"), device="cuda")
    sq.sq_distill_bwd(head, X, W, idd, zd, lse, picked, dloss, dX=dX, **more)

    counts, q = (torch.from_numpy(v).cuda() for v in student.teacher(ids, z, TAU, V))
    live = counts.any(1)
    assert (loss[~live] == 0).all() and (lse[~live] == 0).all() and (dX[~live] == 0).all() and not picked[~counts].any()
    assert torch.isfinite(dX).all()
    at = torch.where(counts, idd, torch.zeros_like(idd))
    zc = zd.to(F64) / TAU
    d = torch.where(counts, zc, -1e30).amax(1) - torch.where(counts, zc, 1e30).amin(1)
    b = (d + 16 + np.log(K)) * 2.0 ** -22
    pick = torch.arange(0, T, max(1, T // 400), device="cuda")
    pick = pick[live[pick]]
    rows = [w[a:a + 65536].to(F64) for a in range(0, V, 65536)]
    for p in pick.split(64):
        x = X[p].to(F64)
        s = torch.zeros((len(p), V), dtype=F64, device="cuda")
        mag = torch.zeros(len(p), dtype=F64, device="cuda")
        for a, r in zip(range(0, V, 65536), rows):
            s[:, a:a + 65536] = x @ r.t().contiguous() / TAU
            mag = torch.maximum(mag, (x.abs() @ r.abs().t().contiguous()).amax(1) / TAU)
        norm, mine = torch.logsumexp(s, 1), torch.where(counts[p], s.gather(1, at[p]), 0.0)
        err, own = 2 * gamma(I + 4) * mag, (s.abs().amax(1) + 64) * 2.0 ** -22
        assert ((picked[p] - mine).abs() <= err[:, None] + 2.0 ** -22 * mine.abs()).all()
        assert ((lse[p] - norm).abs() <= err + own).all()
        log_q = torch.log(torch.where(q[p] > 0, q[p], 1.0))
        want = TAU ** 2 * (q[p] * (log_q - mine + norm[:, None])).sum(1)
        size = (q[p] * (log_q.abs() + (mine - norm[:, None]).abs())).sum(1)
        assert ((loss[p] - want).abs() <= TAU ** 2 * (2 * err + 2 * own + b[p] * (size + 1))).all()
        prob = torch.exp(s - norm[:, None])
        hot = torch.zeros_like(prob).scatter_add_(1, at[p], torch.where(counts[p], q[p], 0.0))
        c = (dloss[p].to(F64) * TAU)[:, None]
        d_err = c.abs() * (prob * (2 * err + 2 * own)[:, None] + hot * b[p][:, None] + (2.0 ** -8 + 2.0 ** -20) * (prob - hot).abs()
                           + 2 * gamma(V + 100) * (prob + hot))
        want, bound = torch.zeros_like(x), torch.zeros_like(x)
        for a, r in zip(range(0, V, 65536), rows):
            want += (c * (prob - hot))[:, a:a + 65536].contiguous() @ r
            bound += d_err[:, a:a + 65536].contiguous() @ r.abs()
        assert ((dX[p] - want).abs() <= bound + 2.0 ** -22 * want.abs() + 1e-30).all()


def test_gradient_of_codes_in_pieces_equals_that_of_bf16_values(sq):
    T, V, I = 4000, 70001, 512
    codes, scales, w = _head("mx", V, I, 0)
    X = inputs.device_bf16_normal(3, (T, I))
    idd, zd = (torch.from_numpy(v).cuda() for v in _entries(T, V))
    W = w.to(torch.bfloat16)
    assert torch.equal(W.to(F64), w)
    _, lse, picked = sq.sq_distill_fwd("bf16", X, W, idd, zd, temperature=TAU)
    dloss = torch.randn(T, generator=inputs.device_generator(4), device="cuda")
    a = sq.sq_distill_bwd("mx", X, codes, idd, zd, lse, picked, dloss, temperature=TAU, scales=scales)
    assert torch.equal(a, sq.sq_distill_bwd("bf16", X, W, idd, zd, lse, picked, dloss, temperature=TAU))
