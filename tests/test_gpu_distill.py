"""Distillation from a teacher's top logits against the oracle: all head formats,
one token to several tiles of tokens, tokens whose entries are cut short, left
out, doubled or all missing, temperatures, both id widths and logit types.

Bounds.  A logit is an fp32 sum of I exact products and a factor: s is off by at
most a = 2 gamma_{I+2} sum |x w| / tau.  lse moves by a, and its own steps add at
most own = (|s| + 64) 2^-22.  The teacher's q[k] are off by b = (d + 16) 2^-22 of
themselves, d = |z - top| / tau: the scaled difference, exponential, sum and
quotient, each a few fp32 roundings.  The loss is tau^2 times a q-weighted sum of
those.  A logit's gradient is off by p (2 a + 2 own) + q b and rounded to bf16
(2^-8 of itself at most); dX sums these against |W| in fp32 (depth V) and is
rounded to its type."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import student
from paper_2609_04526_amd import inputs
from parity_check import gamma
from test_gpu_ce import WS2, _head

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _entries(g, T, V, K, kind):
    """ids [T, K] and logits [T, K]."""
    ids = (V * g.random((T, K)) ** 2).astype(np.int64)
    z = -np.sort(-3.0 * g.standard_normal((T, K)), axis=1) + 5.0
    if kind == "ragged":
        keep = g.integers(0, K + 1, (T, 1))
        ids = np.where(np.arange(K) < keep, ids, g.choice([-1, -100, V, 2 ** 31 - 1], (T, K)))
        z = np.where(g.random((T, K)) < 0.1, -np.inf, z)
    elif kind == "twice":
        ids = ids[:, :1] + np.zeros_like(ids)
        ids[:, K // 2:] = V - 1
    elif kind == "none":
        ids = np.full_like(ids, -1)
    elif kind == "ends":                                       # first and last rows of the head, and its tiles' edges
        ids = g.choice([v for v in (0, V - 1, 255, 256, V // 8 * 8, V // 8 * 8 - 1, 63, 64) if v < V], (T, K))
    return ids, z


def _check(sq, head, T, V, I, K, kind="even", tau=1.0, gain=1.0, id_dtype=torch.int64, z_dtype=F32, out_dtype=F32, ids=None, z=None):
    seed = T + V + K
    W, scales, w = _head(head, seed, V, I, gain)
    g = inputs.rng(seed + 2)
    if ids is None:
        ids, z = _entries(g, T, V, K, kind)
    zt = torch.from_numpy(z).to(z_dtype)
    z = zt.double().numpy()
    X = inputs.bf16_normal(seed + 3, (T, I))
    dloss = g.standard_normal(T).astype(np.float32)
    args = (head, X.cuda(), W, torch.from_numpy(ids).to(id_dtype).cuda(), zt.cuda())
    more = dict(temperature=tau, scales=scales, ws2=WS2)
    loss, lse = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    picked = torch.full((T, K), float("nan"), device="cuda")
    sq.sq_distill_fwd(*args, loss=loss, lse=lse, picked=picked, **more)
    dX = torch.full((T, I), float("nan"), dtype=out_dtype, device="cuda")
    sq.sq_distill_bwd(*args, lse, picked, torch.from_numpy(dloss).cuda(), dX=dX, **more)

    tau = float(np.float32(tau))
    x = X.double().numpy()
    s, mag = x @ w.T / tau, np.abs(x) @ np.abs(w).T / tau
    r_loss, r_lse, r_picked = student.distill_fwd(x, w, ids, z, tau)
    r_dX = student.distill_bwd(x, w, ids, z, tau, dloss)
    counts, q = student.teacher(ids, z, tau, V)
    live = counts.any(1)
    at = np.where(counts, ids, 0)
    a = 2 * gamma(I + 4) * mag.max(1)
    own = (np.abs(s).max(1) + 64) * 2.0 ** -22
    mine = 2 * gamma(I + 4) * np.take_along_axis(mag, at, 1)
    assert (np.abs(picked.double().cpu().numpy() - r_picked) <= np.where(counts, mine + 2.0 ** -22 * np.abs(r_picked), 0)).all()
    assert (np.abs(lse.double().cpu().numpy() - r_lse) <= np.where(live, a + own, 0)).all()
    zc = np.where(counts, z, np.nan) / tau
    d = np.where(live, np.nanmax(np.where(counts, zc, -1e30), 1) - np.nanmin(np.where(counts, zc, 1e30), 1), 0)
    b = (d + 16 + np.log(K)) * 2.0 ** -22
    size = (q * (np.abs(np.log(np.where(q > 0, q, 1))) + np.abs(r_picked - r_lse[:, None]))).sum(1)
    assert (np.abs(loss.double().cpu().numpy() - r_loss) <= np.where(live, tau ** 2 * (2 * a + 2 * own + b * (size + 1)), 0)).all()
    p = np.exp(s - s.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    hot = np.zeros_like(p)
    for t, k in zip(*np.nonzero(counts)):
        hot[t, ids[t, k]] += q[t, k]
    c = (np.abs(dloss.astype(np.float64)) * tau)[:, None]
    d_err = c * (p * (2 * a + 2 * own)[:, None] + hot * b[:, None] + (2.0 ** -8 + 2.0 ** -20) * np.abs(p - hot)) + 1e-38
    bound = d_err @ np.abs(w) + 2 * gamma(V + 70) * (c * (p + hot)) @ np.abs(w)
    bound = bound + (2.0 ** -8 if out_dtype == BF16 else 2.0 ** -22) * np.abs(r_dX) * 1.01
    err = np.abs(dX.double().cpu().numpy() - r_dX)
    assert (err <= np.where(live[:, None], bound, 0)).all(), (err - bound).max()
    return loss, lse, picked, dX


@pytest.mark.parametrize("T,V,I,K", [(1, 1, 32, 1), (1, 257, 64, 3), (5, 1000, 512, 16), (64, 255, 96, 65), (65, 513, 160, 8),
                                     (128, 256, 64, 256), (129, 300, 96, 20), (256, 1025, 128, 64), (257, 770, 96, 33),
                                     (700, 1300, 288, 128), (3, 5000, 1056, 200), (70, 2049, 512, 64), (300, 1500, 512, 10)])
@pytest.mark.parametrize("head", ["bf16", "mx", "nv"])
def test_shapes(sq, head, T, V, I, K):
    n = T + V
    _check(sq, head, T, V, I, K, tau=(1.0, 2.0, 0.7)[n % 3], id_dtype=(torch.int64, torch.int32)[n // 2 % 2],
           z_dtype=(F32, BF16)[n // 3 % 2], out_dtype=(F32, BF16)[n // 4 % 2])


@pytest.mark.parametrize("kind", ["ragged", "twice", "ends", "none"])
@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("head", ["bf16", "mx", "nv"])
def test_entries(sq, head, T, kind):
    loss, lse, picked, dX = _check(sq, head, T, 781, 128, 24, kind=kind, tau=1.5)
    if kind == "none":
        assert not loss.any() and not lse.any() and not picked.any() and not dX.any()


@pytest.mark.parametrize("T,V", [(1, 40961), (9, 33000), (64, 36001), (129, 40007)])
@pytest.mark.parametrize("head", ["mx", "nv"])
def test_groups_of_a_4_bit_head(sq, head, T, V):
    """Few tokens through the layer's own products, groups of the head's rows among them and rows past eights."""
    _check(sq, head, T, V, 64, 40, kind="ends" if T == 9 else "even", tau=2.0)


@pytest.mark.parametrize("tau", [2.0 ** -6, 0.25, 16.0, 1000.0])
@pytest.mark.parametrize("T", [20, 400])
def test_temperatures(sq, T, tau):
    _check(sq, "bf16", T, 600, 96, 12, tau=tau)


@pytest.mark.parametrize("head,T", [("bf16", 50), ("bf16", 300), ("mx", 50), ("nv", 300)])
def test_the_loss_is_zero_where_student_and_teacher_agree(sq, head, T):
    """The teacher's entries are the student's own logits over the whole vocabulary: loss and gradient vanish, up to what
    the logits' rounding leaves of them."""
    V, I, K = 250, 64, 250
    W, scales, w = _head(head, 5, V, I)
    X = inputs.bf16_normal(6, (T, I))
    z = torch.from_numpy(X.double().numpy() @ w.T).float()
    ids = torch.arange(V).repeat(T, 1)
    more = dict(scales=scales, ws2=WS2, temperature=2.0)
    loss, lse, picked = sq.sq_distill_fwd(head, X.cuda(), W, ids.cuda(), z.cuda(), **more)
    dX = sq.sq_distill_bwd(head, X.cuda(), W, ids.cuda(), z.cuda(), lse, picked, torch.ones(T, device="cuda"), **more)
    a = (np.abs(z.double().numpy()).max() + 64) * 2.0 ** -21 + 2 * gamma(I + 4) * (np.abs(X.double().numpy()) @ np.abs(w).T).max()
    assert loss.abs().max().item() <= 4 * a * 2
    # each gradient is off by at most 2 (p + q) a and its rounding
    assert dX.abs().max().item() <= 2 * 4 * a * np.abs(w).max() * 2


def test_nan_and_infinite_teachers(sq):
    T, V, I, K = 6, 300, 64, 8
    W = (inputs.bf16_normal(1, (V, I)) / 8).cuda()
    X = inputs.bf16_normal(2, (T, I)).cuda()
    ids = torch.arange(K).repeat(T, 1).cuda()
    z = torch.zeros((T, K), device="cuda")
    z[1, 3], z[2, 4], z[3, 5], z[4] = float("nan"), float("inf"), float("-inf"), float("-inf")
    ids[5], z[5, 0] = -1, float("nan")                         # a NaN that is left out
    loss, lse, picked = sq.sq_distill_fwd("bf16", X, W, ids, z)
    dX = sq.sq_distill_bwd("bf16", X, W, ids, z, lse, picked, torch.ones(T, device="cuda"))
    assert loss.isnan().tolist() == [False, True, True, False, False, False]
    assert loss[4] == 0 and loss[5] == 0 and not dX[4].any() and not dX[5].any() and dX[1].isnan().all() and dX[2].isnan().all()
    assert not dX[[0, 3]].isnan().any()


def test_gradient_against_differences(sq):
    """dX of the loss's sum, by central differences of the loss in 64 bits along random directions."""
    T, V, I, K, tau = 30, 400, 96, 12, 1.3
    W, scales, w = _head("mx", 4, V, I)
    g = inputs.rng(9)
    ids, z = _entries(g, T, V, K, "ragged")
    zt = torch.from_numpy(z).float()
    X = inputs.bf16_normal(7, (T, I))
    dloss = g.standard_normal(T).astype(np.float32)
    args = ("mx", X.cuda(), W, torch.from_numpy(ids).cuda(), zt.cuda())
    loss, lse, picked = sq.sq_distill_fwd(*args, temperature=tau, scales=scales)
    dX = sq.sq_distill_bwd(*args, lse, picked, torch.from_numpy(dloss).cuda(), temperature=tau, scales=scales).double().cpu().numpy()
    x, t32 = X.double().numpy(), float(np.float32(tau))

    def total(v):
        return (student.distill_fwd(v, w, ids, zt.double().numpy(), t32)[0] * dloss).sum()

    for k in range(5):
        u = g.standard_normal((T, I))
        h = 1e-5
        want = (total(x + h * u) - total(x - h * u)) / (2 * h)
        # differences are off by h^2; a gradient's entry by 2^-8 of its logit gradients' weight on W
        slack = 2.0 ** -7 * (np.abs(dloss)[:, None] * tau * 2 * np.abs(w).max() * np.abs(u)).sum()
        assert abs((dX * u).sum() - want) <= slack * 0.1 + 1e-6 * abs(want)


def test_same_bits_on_every_run(sq):
    for T in (20, 300):
        a = _check(sq, "mx", T, 700, 512, 30, kind="twice")
        b = _check(sq, "mx", T, 700, 512, 30, kind="twice")
        assert all(torch.equal(u, v) for u, v in zip(a, b))
