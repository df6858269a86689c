"""Cross entropy of a head against the oracle: one token to several tiles of
tokens, vocabularies of one entry, odd ones and several pieces' worth, all head
formats, ignored and invalid targets, both target widths, large and infinite
logits.

Bounds.  A logit is an fp32 sum of I exact products: off by at most a =
gamma_I sum |x w| (Higham's bound).  lse moves by at most max a, and its own
steps (exponentials, sums over tiles, logarithm: each a few fp32 roundings, the
exponential's argument rounded at |l - top| 2^-24) add at most (|top| + 64)
2^-22.  loss adds the target's logit.  A logit's gradient c (p - [target]) is
off by c p (2 a + the same) and rounded to bf16 (2^-8 of itself at most); dX sums these
against |W| in fp32 (depth V) and is rounded to its type."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import linear, step
from paper_2609_04526_amd import inputs
from parity_check import gamma

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16, F32 = torch.bfloat16, torch.float32
BLOCK = {"mx": 32, "nv": 16}
WS2 = float(np.float32(1.0 / 448.0))


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _head(head, seed, V, I, gain=1.0):
    """Device operands of a head whose logits have a standard deviation of about `gain` * 2, and its fp64 values."""
    if head == "bf16":
        W = (inputs.bf16_normal(seed, (V, I)).float() * (2 * gain / np.sqrt(I))).to(BF16)
        return W.cuda(), None, W.double().numpy()
    codes = inputs.codes_uniform(seed, V, I)
    if head == "mx":
        e = int(np.round(np.log2(gain / np.sqrt(I))))
        sc = inputs.e8m0_uniform_exponents(seed + 1, V, I // 32, e - 1, e + 1)
        w = linear.dequant("mx", codes, sc)
    else:
        sc = (torch.from_numpy(np.abs(inputs.rng(seed + 1).standard_normal((V, I // 16)))) * (448.0 * gain / np.sqrt(I)))
        sc = sc.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        w = linear.dequant("nv", codes, sc, WS2)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(sc).cuda(), w


def _check(sq, head, T, V, I, seed, y=None, gain=1.0, y_dtype=torch.int64, out_dtype=F32):
    W, scales, w = _head(head, seed, V, I, gain)
    g = inputs.rng(seed + 2)
    if y is None:
        y = g.integers(0, V, T)
    y = np.asarray(y, np.int64)
    X = inputs.bf16_normal(seed + 3, (T, I))
    dloss = g.standard_normal(T).astype(np.float32)
    yd, dl = torch.from_numpy(y).to(y_dtype).cuda(), torch.from_numpy(dloss).cuda()
    loss, lse = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    sq.sq_ce_fwd(head, X.cuda(), W, yd, scales=scales, ws2=WS2, loss=loss, lse=lse)
    dX = torch.full((T, I), float("nan"), dtype=out_dtype, device="cuda")
    sq.sq_ce_bwd(head, X.cuda(), W, yd, lse, dl, scales=scales, ws2=WS2, dX=dX)

    x = X.double().numpy()
    l, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    r_loss, r_lse = step.ce_fwd(x, w, y)
    r_dX = step.ce_bwd(x, w, y, dloss)
    valid = (y >= 0) & (y < V)
    a = 2 * gamma(I + 2) * mag.max(1)
    own = (np.abs(l).max(1) + 64) * 2.0 ** -22
    assert (np.abs(lse.double().cpu().numpy() - r_lse) <= np.where(valid, a + own, 0)).all()
    assert (np.abs(loss.double().cpu().numpy() - r_loss) <= np.where(valid, 2 * a + 2 * own, 0)).all()
    p = np.exp(l - l.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    hot = np.zeros_like(p)
    hot[np.flatnonzero(valid), y[valid]] = 1.0
    c = np.abs(dloss.astype(np.float64))[:, None]
    d_err = c * (p * (2 * a + 2 * own)[:, None] + (2.0 ** -8 + 2.0 ** -20) * np.abs(p - hot)) + 1e-38
    total = c * (p + hot) @ np.abs(w)
    bound = d_err @ np.abs(w) + 2 * gamma(V + 70) * total + (2.0 ** -8 if out_dtype == BF16 else 2.0 ** -22) * np.abs(r_dX) * 1.01
    err = np.abs(dX.double().cpu().numpy() - r_dX)
    assert (err <= np.where(valid[:, None], bound, 0)).all(), (err - bound).max()
    return loss, lse, dX


# few tokens (64-token tiles), 128- and 256-token tiles, ragged edges, rows beyond one tile, compact rows (T > 256)
@pytest.mark.parametrize("T,V,I", [(1, 1, 32), (1, 257, 64), (5, 1000, 512), (64, 255, 96), (65, 513, 160), (128, 256, 64),
                                   (129, 300, 96), (256, 1025, 128), (257, 770, 96), (700, 1300, 288), (3, 5000, 1056)])
@pytest.mark.parametrize("head", ["bf16", "mx", "nv"])
def test_shapes(sq, head, T, V, I):
    _check(sq, head, T, V, I, T + V)


@pytest.mark.parametrize("I", [8, 24, 72, 200, 264])
def test_bf16_head_of_odd_widths(sq, I):
    _check(sq, "bf16", 70, 301, I, I)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("y_dtype", [torch.int64, torch.int32])
@pytest.mark.parametrize("T", [40, 600])
def test_ignored_and_invalid_targets(sq, T, y_dtype, out_dtype):
    V = 777
    g = inputs.rng(T)
    y = np.where(g.random(T) < 0.5, g.integers(0, V, T), g.choice([-100, -1, V, V + 5, 2 ** 31 - 1], T))
    y[:3] = [0, V - 1, -1]
    _check(sq, "bf16", T, V, 128, T, y=y, y_dtype=y_dtype, out_dtype=out_dtype)


@pytest.mark.parametrize("T", [7, 300])
def test_all_tokens_ignored(sq, T):
    loss, lse, dX = _check(sq, "mx", T, 500, 64, 3, y=np.full(T, -100))
    assert not loss.any() and not lse.any() and not dX.any()


@pytest.mark.parametrize("head", ["bf16", "nv"])
def test_one_live_token_among_many(sq, head):
    y = np.full(1000, -100)
    y[777] = 12
    _check(sq, head, 1000, 600, 96, 5, y=y)


@pytest.mark.parametrize("gain", [1e-3, 30.0])
def test_flat_and_peaked_softmax(sq, gain):
    """Logits near 0 (every p about 1 / V) and of a few hundred (one p is 1)."""
    _check(sq, "bf16", 300, 900, 128, 8, gain=gain)


def test_several_pieces_of_the_vocabulary(sq):
    """Many tokens: a piece's logit gradients are bounded, so the vocabulary takes several; the sums carry over."""
    T, V, I = 66000, 5000, 8
    need = sq.sq_ce_bwd_workspace("bf16", T, V, I)
    assert need < T * V * 2                       # less than all of the logits' gradients at once
    W, _, w = _head("bf16", 1, V, I)
    X = inputs.bf16_normal(2, (T, I))
    y = inputs.rng(3).integers(0, V, T)
    yd, dl = torch.from_numpy(y).cuda(), torch.ones(T, device="cuda")
    loss, lse = sq.sq_ce_fwd("bf16", X.cuda(), W, yd)
    dX = sq.sq_ce_bwd("bf16", X.cuda(), W, yd, lse, dl)
    pick = np.r_[0:64, T // 2:T // 2 + 64, T - 64:T]
    x = X.double().numpy()[pick]
    r_loss, r_lse = step.ce_fwd(x, w, y[pick])
    r_dX = step.ce_bwd(x, w, y[pick], np.ones(len(pick)))
    assert np.abs(lse.cpu().numpy()[pick] - r_lse).max() < 1e-5
    assert np.abs(loss.cpu().numpy()[pick] - r_loss).max() < 2e-5
    # each p rounded to bf16: 2^-8 of sum (p + [target]) |W|
    bound = 2.0 ** -8 * (2 * np.abs(w).max(0))
    assert (np.abs(dX.cpu().numpy()[pick] - r_dX) <= bound).all()


@pytest.mark.parametrize("head", ["mx", "nv"])
def test_a_4_bit_head_equals_its_bf16_values(sq, head):
    """The same bits as the head written out in bf16 (MXFP4; NVFP4 with ws2 = 1)."""
    T, V, I = 300, 1000, 256
    codes = inputs.device_codes_uniform(4, V, I)
    if head == "mx":
        sc = inputs.device_e8m0_normal_exponents(5, V, I // 32, -5.0, 1.0)
        w = linear.dequant("mx", codes.cpu().numpy(), sc.cpu().numpy())
    else:
        sc = (torch.rand((V, I // 16), generator=inputs.device_generator(6), device="cuda") * 0.1).to(torch.float8_e4m3fn).view(torch.uint8)
        w = linear.dequant("nv", codes.cpu().numpy(), sc.cpu().numpy(), 1.0)
    W = torch.from_numpy(w).to(BF16).cuda()
    assert np.array_equal(W.double().cpu().numpy(), w)
    X = inputs.device_bf16_normal(7, (T, I))
    y = torch.arange(T, device="cuda") * 3 % V
    a, b = sq.sq_ce_fwd(head, X, codes, y, scales=sc), sq.sq_ce_fwd("bf16", X, W, y)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    dl = torch.rand(T, generator=inputs.device_generator(8), device="cuda")
    assert torch.equal(sq.sq_ce_bwd(head, X, codes, y, a[1], dl, scales=sc), sq.sq_ce_bwd("bf16", X, W, y, b[1], dl))


def test_logits_without_a_value(sq):
    """-inf beside finite logits is probability 0; +inf and NaN give NaN in their own row only."""
    V, I = 300, 32
    W = torch.zeros((V, I), dtype=BF16)
    W[:, 0] = torch.linspace(-1, 1, V).to(BF16)
    W[7, 1] = float("-inf")
    W[9, 2] = float("inf")
    W[11, 3] = float("nan")
    X = torch.zeros((5, I), dtype=BF16)
    X[:, 0] = 1
    X[0, 1], X[1, 2], X[2, 3], X[3, 1] = 1.0, 1.0, 1.0, 1.0
    # 0 * inf is NaN: rows that hold an infinity meet it in every token, so keep the others out of the columns
    Wd = torch.nan_to_num(W.float(), nan=0.0, posinf=0.0, neginf=0.0).to(BF16)
    y = torch.tensor([3, 4, 5, 6, 299])
    base, _ = sq.sq_ce_fwd("bf16", X.cuda(), Wd.cuda(), y.cuda())
    assert torch.isfinite(base).all()
    big = Wd.clone()
    big[7, 1] = -3e38
    Xb = X.clone()
    Xb[0, 1] = 3e38                                # the product overflows to -inf for token 0 alone
    loss, lse = sq.sq_ce_fwd("bf16", Xb.cuda(), big.cuda(), y.cuda())
    ref = torch.logsumexp(torch.cat((Wd.float()[:7, 0], Wd.float()[8:, 0])), 0)
    assert abs(lse[0].item() - ref.item()) < 1e-5
    big[7, 1] = 3e38
    loss, lse = sq.sq_ce_fwd("bf16", Xb.cuda(), big.cuda(), y.cuda())
    assert torch.isnan(lse[0]) and torch.isnan(loss[0]) and torch.isfinite(lse[1:3]).all() and torch.isfinite(lse[4])


def test_deterministic_and_on_another_stream(sq):
    T, V, I = 500, 3000, 512
    W, _, _ = _head("bf16", 1, V, I)
    X, y = inputs.device_bf16_normal(2, (T, I)), torch.arange(T, device="cuda") * 5 % V
    dl = torch.ones(T, device="cuda")
    loss, lse = sq.sq_ce_fwd("bf16", X, W, y)
    dX = sq.sq_ce_bwd("bf16", X, W, y, lse, dl)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        loss2, lse2 = sq.sq_ce_fwd("bf16", X, W, y)
        dX2 = sq.sq_ce_bwd("bf16", X, W, y, lse2, dl)
    s.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2) and torch.equal(dX, dX2)


def test_no_tokens(sq):
    W, _, _ = _head("bf16", 1, 100, 64)
    X, y = torch.empty((0, 64), dtype=BF16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = sq.sq_ce_fwd("bf16", X, W, y)
    assert loss.shape == lse.shape == (0,)
    assert sq.sq_ce_bwd("bf16", X, W, y, lse, loss).shape == (0, 64)


# few tiles and long rows: the logits' sums over I split into planes, with and without compact rows, and ignored tokens
@pytest.mark.parametrize("T,V,I", [(1, 1, 1024), (4, 1136, 7296), (200, 700, 2080), (300, 513, 1088), (1000, 260, 4096)])
@pytest.mark.parametrize("head", ["bf16", "nv"])
def test_few_tiles_of_long_rows(sq, head, T, V, I):
    y = inputs.rng(T + 1).integers(0, V, T)
    y[1::5] = -1
    _check(sq, head, T, V, I, T + I, y, out_dtype=BF16 if T > 200 else F32)


# tiles of dX that would leave the last round of the compute units poorly filled, in splits of the vocabulary, with live rows
# that need more groups than all of the rows would
@pytest.mark.parametrize("T,V,I,ignored", [(2200, 1300, 2560, 0), (1100, 1700, 4600, 3), (1900, 1100, 1096, 2)])
def test_splits_of_many_tiles(sq, T, V, I, ignored):
    y = inputs.rng(T + 1).integers(0, V, T)
    if ignored:
        y[::ignored] = V
    _check(sq, "bf16", T, V, I, T + I, y, out_dtype=BF16)


# a 4-bit head's rows in groups: the last one of the gradient overlaps the one before it, the logits' in groups of 4096 with a
# narrower last one, rows past a multiple of 8, and the target in each of these places
@pytest.mark.parametrize("T,V,I", [(6, 2665, 704), (3, 33003, 64), (130, 33003, 64), (2, 40961, 96)])
@pytest.mark.parametrize("head", ["mx", "nv"])
def test_groups_of_a_4_bit_head(sq, head, T, V, I):
    g = inputs.rng(T + 2)
    edges = np.array([V - 1, V // 8 * 8 - 1, 0, V // 8 * 8, V // 8 * 8 - 300, -1, V])
    y = np.where(g.random(T) < 0.5, g.choice(edges, T), g.integers(0, V, T))
    _check(sq, head, T, V, I, T + I, y)


@pytest.mark.parametrize("T,V,I", [(3, 37, 64), (70, 300, 160), (290, 1001, 96)])
@pytest.mark.parametrize("head", ["bf16", "mx", "nv"])
def test_gradient_by_differences(sq, head, T, V, I):
    """loss(X + U) - loss(X - U) against 2 <dX, U>, X and U on a grid of bf16 that holds X +- U.

    Per token the third derivative along U is a third central moment of the logits' changes, (2 m)^3 at most for changes up to m,
    so the difference is off by (2 m)^3 / 3; each loss by its own bound, dX by the rounding of the logits' gradients, 2^-8 of
    sum |p - hot| <= 2 against changes up to m, and its fp32 sums."""
    W, scales, w = _head(head, T, V, I, 0.2)
    g = inputs.rng(T + 5)
    x, u = g.integers(-16, 17, (T, I)) / 8.0, g.integers(-1, 2, (T, I)) / 64.0
    y = torch.from_numpy(g.integers(0, V, T)).cuda()
    dev = lambda a: torch.from_numpy(a).to(BF16).cuda()
    assert torch.equal(dev(x + u).double().cpu(), torch.from_numpy(x + u))
    up, down = (sq.sq_ce_fwd(head, dev(a), W, y, scales=scales, ws2=WS2)[0].double().cpu().numpy() for a in (x + u, x - u))
    lse = sq.sq_ce_fwd(head, dev(x), W, y, scales=scales, ws2=WS2)[1]
    dX = sq.sq_ce_bwd(head, dev(x), W, y, lse, torch.ones(T, device="cuda"), scales=scales, ws2=WS2).double().cpu().numpy()
    change = np.abs(u @ w.T).max(1)
    mag = (np.abs(x) + np.abs(u)) @ np.abs(w).T
    one = 4 * gamma(I + 2) * mag.max(1) + 2 * (mag.max(1) + 64) * 2.0 ** -22
    sums = 2 * gamma(V + 70) * 2 * (np.abs(u) @ np.abs(w).T).max(1)
    bound = (2 * change) ** 3 / 3 + 2 * one + 2 * (2.0 ** -8 + 2.0 ** -18) * 2 * change + 2 * sums
    assert (np.abs((up - down) - 2 * (dX * u).sum(1)) <= bound).all()
    assert (bound < 0.2 * np.abs(up - down).max()).all()        # the bound says something


# statistics straight from MXFP4 codes: 64-, 128- and 256-token tiles, groups of scales that end inside and with the row,
# ragged vocabularies, and codes that are not aligned for it
@pytest.mark.parametrize("T,V,I", [(300, 3003, 512), (257, 17000, 1024), (700, 9001, 1536), (1030, 16399, 2048), (2100, 66, 4608)])
@pytest.mark.parametrize("offset", [0, 4])
def test_statistics_of_codes_equal_those_of_bf16_values(sq, T, V, I, offset):
    codes, scales, w = _head("mx", V, V, I)
    base = torch.zeros(codes.numel() + 16, dtype=torch.uint8, device="cuda")
    base[offset:offset + codes.numel()] = codes.reshape(-1)
    codes = base[offset:offset + codes.numel()].view(V, I // 2)
    y = torch.from_numpy(inputs.rng(T).integers(0, V, T)).cuda()
    y[::5] = -1
    X = inputs.device_bf16_normal(T, (T, I))
    got = sq.sq_ce_fwd("mx", X, codes, y, scales=scales)
    want = sq.sq_ce_fwd("bf16", X, torch.from_numpy(w).to(BF16).cuda(), y)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# and of few tokens, where there are tiles enough
@pytest.mark.parametrize("T,V,I", [(3, 34001, 512), (130, 33333, 512)])
def test_statistics_of_codes_of_few_tokens(sq, T, V, I):
    codes, scales, w = _head("mx", V, V, I)
    y = torch.from_numpy(inputs.rng(T).integers(0, V, T)).cuda()
    X = inputs.device_bf16_normal(T, (T, I))
    got = sq.sq_ce_fwd("mx", X, codes, y, scales=scales)
    want = sq.sq_ce_fwd("bf16", X, torch.from_numpy(w).to(BF16).cuda(), y)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# the gradient straight from MXFP4 codes: dX tiles of 64, 128 and 256 tokens, splits of the vocabulary, ragged edges, and codes
# that are not aligned for it, which go through bf16 in memory
@pytest.mark.parametrize("T,V,I", [(300, 3003, 512), (257, 17000, 1024), (700, 9001, 1536), (1030, 16399, 2048), (2100, 9000, 1024)])
@pytest.mark.parametrize("offset", [0, 4])
def test_gradient_of_codes_equals_that_of_bf16_values(sq, T, V, I, offset):
    codes, scales, w = _head("mx", V, V, I)
    base = torch.zeros(codes.numel() + 16, dtype=torch.uint8, device="cuda")
    base[offset:offset + codes.numel()] = codes.reshape(-1)
    codes = base[offset:offset + codes.numel()].view(V, I // 2)
    g = inputs.rng(T)
    y = torch.from_numpy(g.integers(0, V, T)).cuda()
    y[::5] = -1
    dloss = torch.from_numpy(g.standard_normal(T).astype(np.float32)).cuda()
    X, W = inputs.device_bf16_normal(T, (T, I)), torch.from_numpy(w).to(BF16).cuda()
    _, lse = sq.sq_ce_fwd("bf16", X, W, y)
    got = sq.sq_ce_bwd("mx", X, codes, y, lse, dloss, scales=scales)
    assert torch.equal(got, sq.sq_ce_bwd("bf16", X, W, y, lse, dloss))


@pytest.mark.parametrize("T,V,I", [(100, 34001, 512), (256, 33333, 512), (65, 40008, 1024)])
def test_gradient_of_codes_of_few_tokens(sq, T, V, I):
    codes, scales, w = _head("mx", V, V, I)
    g = inputs.rng(T)
    y = torch.from_numpy(g.integers(0, V, T)).cuda()
    y[::7] = V
    dloss = torch.from_numpy(g.standard_normal(T).astype(np.float32)).cuda()
    X, W = inputs.device_bf16_normal(T, (T, I)), torch.from_numpy(w).to(BF16).cuda()
    _, lse = sq.sq_ce_fwd("bf16", X, W, y)
    got = sq.sq_ce_bwd("mx", X, codes, y, lse, dloss, scales=scales)
    assert torch.equal(got, sq.sq_ce_bwd("bf16", X, W, y, lse, dloss))
