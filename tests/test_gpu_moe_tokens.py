"""Tokens to experts and back (sq_moe_sort, sq_moe_gather, sq_moe_combine and
its gradients) against the oracle: few and many pairs (both forms of the sort),
ids of both widths, dropped pairs, experts and tokens without any pair, odd row
widths, fp32 and bf16 rows, and non-finite values in rows that are not routed."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import step
from parity_check import gamma

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _ids(seed, T, K, E, drop, dtype=np.int64):
    g = np.random.default_rng(seed)
    ids = g.integers(0, E, (T, K))
    return np.where(g.random((T, K)) < drop, g.choice([-1, -7, E, E + 3], (T, K)), ids).astype(dtype)


def _check_sort(sq, ids, E):
    got = sq.sq_moe_sort(torch.from_numpy(ids).cuda(), E)
    for a, b in zip(got, step.moe_sort(ids, E)):
        assert np.array_equal(a.cpu().numpy(), b)
    return got


@pytest.mark.parametrize("T,K,E,drop", [
    (0, 2, 4, 0.0), (1, 1, 1, 0.0), (1, 8, 128, 0.0), (3, 2, 2, 1.0), (63, 1, 7, 0.1), (257, 5, 255, 0.2),
    (1000, 8, 128, 0.05), (513, 3, 2048, 0.0),
])
@pytest.mark.parametrize("dtype", [np.int64, np.int32])
def test_sort(sq, T, K, E, drop, dtype):
    _check_sort(sq, _ids(T + E, T, K, E, drop, dtype), E)


@pytest.mark.parametrize("T,K,E,drop", [(8193, 8, 128, 0.05), (70001, 1, 1, 0.3), (16385, 5, 2048, 0.0), (65537, 2, 3, 0.0)])
@pytest.mark.parametrize("dtype", [np.int64, np.int32])
def test_sort_of_many_pairs(sq, T, K, E, drop, dtype):
    """Above the pairs that one launch takes: chunks of 4096 pairs, the last one short."""
    assert sq.sq_moe_sort_workspace(T, K, E) > 0
    _check_sort(sq, _ids(T + E, T, K, E, drop, dtype), E)


@pytest.mark.parametrize("T", [40, 9000])
def test_sort_with_one_expert_taking_all(sq, T):
    ids = np.full((T, 8), 5, np.int64)
    _check_sort(sq, ids, 9)
    _check_sort(sq, np.full((T, 8), -1, np.int64), 9)


def _case(seed, T, K, E, H, drop, y_dtype, d_dtype=None):
    g = np.random.default_rng(seed)
    ids = _ids(seed, T, K, E, drop)
    offsets, token, slot = (torch.from_numpy(a).cuda() for a in step.moe_sort(ids, E))
    mk = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32))  # noqa: E731
    Ys, d = mk(T * K, H).to(y_dtype), mk(T, H).to(d_dtype or y_dtype)
    w = torch.from_numpy(g.random((T, K)).astype(np.float32))
    return offsets, slot, Ys, d, w


def _np(t):
    return t.double().cpu().numpy()


def _close(got, ref, absref, terms):
    """fp32 sums of `terms` rounded steps, and the output's own rounding."""
    u = 2.0 ** -8 if got.dtype == BF16 else 0.0
    bad = ~(np.abs(_np(got) - ref) <= 2 * gamma(terms) * absref + u * (np.abs(ref) + 2 * gamma(terms) * absref) + 1e-38)
    assert not bad.any(), np.argwhere(bad)[:3]


SHAPES = [(1, 1, 1, 8, 0.0), (1, 8, 128, 2048, 0.0), (5, 3, 4, 1000, 0.3), (77, 9, 16, 4104, 0.1), (130, 2, 8, 520, 1.0),
          (300, 17, 32, 264, 0.2), (2100, 4, 16, 512, 0.05)]


@pytest.mark.parametrize("T,K,E,H,drop", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gather(sq, T, K, E, H, drop, dtype):
    offsets, slot, _, X, _ = _case(T + H, T, K, E, H, drop, dtype)
    if T > 1:
        X[1, :3] = torch.tensor([float("nan"), float("inf"), -0.0])
    Xs = torch.full((T * K, H), 7.0, dtype=dtype, device="cuda")
    sq.sq_moe_gather(X.cuda(), slot, offsets, Xs=Xs)
    ref = step.moe_gather(_np(X), slot.cpu().numpy(), int(offsets[-1]))
    assert np.array_equal(_np(Xs), ref, equal_nan=True)


@pytest.mark.parametrize("T,K,E,H,drop", SHAPES)
@pytest.mark.parametrize("y_dtype,out_dtype", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("weighted", [True, False])
def test_combine(sq, T, K, E, H, drop, y_dtype, out_dtype, weighted):
    offsets, slot, Ys, _, w = _case(T + H + 1, T, K, E, H, drop, y_dtype)
    R = int(offsets[-1])
    Ys[R:] = float("nan")                        # rows of dropped pairs reach nothing
    if R == 0:
        Ys[:] = float("inf")
    out = sq.sq_moe_combine(Ys.cuda(), slot, offsets, w.cuda() if weighted else None, out_dtype=out_dtype)
    assert out.dtype == out_dtype
    y, s, v = _np(Ys), slot.cpu().numpy(), _np(w) if weighted else None
    with np.errstate(invalid="ignore"):
        ref, mag = step.moe_combine(y, s, R, v), step.moe_combine(np.abs(y), s, R, v)
    _close(out, ref, mag, K + 1)


@pytest.mark.parametrize("T,K,E,H,drop", SHAPES)
@pytest.mark.parametrize("d_dtype,y_dtype,g_dtype", [(BF16, BF16, BF16), (F32, BF16, BF16), (BF16, F32, F32), (F32, F32, F32),
                                                     (F32, F32, BF16), (BF16, F32, BF16), (F32, BF16, F32), (BF16, BF16, F32)])
def test_combine_bwd(sq, T, K, E, H, drop, d_dtype, y_dtype, g_dtype):
    offsets, slot, Ys, d, w = _case(T + H + 2, T, K, E, H, drop, y_dtype, d_dtype)
    R = int(offsets[-1])
    Ys[R:] = float("nan")
    dYs = torch.full((T * K, H), 7.0, dtype=g_dtype, device="cuda")
    dw = torch.full((T, K), 7.0, device="cuda")
    sq.sq_moe_combine_bwd(d.cuda(), Ys.cuda(), slot, offsets, w.cuda(), dYs=dYs, dweights=dw)
    y, s = _np(Ys), slot.cpu().numpy()
    rY, rw = step.moe_combine_bwd(_np(d), y, s, R, _np(w))
    _, mag = step.moe_combine_bwd(np.abs(_np(d)), np.abs(y), s, R, _np(w))
    _close(dYs, rY, np.abs(rY), 2)
    _close(dw, rw, mag, H + 8)


def test_combine_bwd_of_a_dropped_pair_ignores_the_token(sq):
    """A dropped pair's gradients are zeros also where dOut is not finite."""
    slot = torch.tensor([[1, 2], [0, 3]], dtype=torch.int32, device="cuda")      # routed: 0 and 1
    offsets = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    d = torch.full((2, 8), float("inf"), device="cuda")
    Ys, w = torch.ones((4, 8), device="cuda"), torch.ones((2, 2), device="cuda")
    dYs, dw = sq.sq_moe_combine_bwd(d, Ys, slot, offsets, w)
    assert torch.isinf(dYs[:2]).all() and (dYs[2:] == 0).all()
    assert torch.isinf(dw[:, 0]).all() and (dw[:, 1] == 0).all()


def test_slots_outside_the_pairs_count_as_dropped(sq):
    slot = torch.tensor([[0, 2 ** 31 - 1], [-1, 4]], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    X = torch.ones((2, 16), device="cuda")
    Xs = torch.zeros((4, 16), device="cuda")
    sq.sq_moe_gather(X, slot, offsets, Xs=Xs)
    assert (Xs[0] == 1).all() and (Xs[1:] == 0).all()
    out = sq.sq_moe_combine(X.new_full((4, 16), 3.0), slot, offsets)
    assert (out[0] == 3).all() and (out[1] == 0).all()
    dYs, dw = torch.zeros((4, 16), device="cuda"), torch.ones((2, 2), device="cuda")
    sq.sq_moe_combine_bwd(X, X.new_full((4, 16), 3.0), slot, offsets, torch.ones((2, 2), device="cuda"), dYs=dYs, dweights=dw)
    assert (dYs[0] == 1).all() and (dYs[1:] == 0).all() and dw.cpu().tolist() == [[48.0, 0.0], [0.0, 0.0]]


def test_no_tokens(sq):
    ids = torch.empty((0, 4), dtype=torch.int64, device="cuda")
    offsets, token, slot = sq.sq_moe_sort(ids, 6)
    assert offsets.cpu().tolist() == [0] * 7 and token.numel() == 0
    X = torch.empty((0, 64), device="cuda")
    assert sq.sq_moe_gather(X, slot, offsets).shape == (0, 64)
    assert sq.sq_moe_combine(X, slot, offsets).shape == (0, 64)


def test_rows_past_32_bit_offsets(sq):
    """N*H above 2^31 elements: the last expert's rows are where they belong."""
    T, K, H = 66000, 8, 4096
    slot = torch.arange(T * K, dtype=torch.int32, device="cuda").view(T, K)
    offsets = torch.tensor([0, T * K], dtype=torch.int32, device="cuda")
    X = torch.zeros((T, H), dtype=BF16, device="cuda")
    X[-1] = 3.0
    Xs = sq.sq_moe_gather(X, slot, offsets)
    assert Xs.numel() > 2 ** 31
    assert (Xs[-K:] == 3).all() and (Xs[-2 * K:-K] == 0).all() and (Xs[:K] == 0).all()
    out = sq.sq_moe_combine(Xs, slot, offsets, out_dtype=BF16)
    assert (out[-1] == 24).all() and (out[:-1] == 0).all()
    w = torch.full((T, K), 0.5, device="cuda")
    dYs, dw = sq.sq_moe_combine_bwd(X, Xs, slot, offsets, w)
    assert (dYs[-K:] == 1.5).all() and (dYs[:-K] == 0).all()
    assert (dw[-1] == 9.0 * H).all() and (dw[:-1] == 0).all()


def test_same_results_on_another_stream(sq):
    offsets, slot, Ys, d, w = _case(5, 200, 4, 16, 512, 0.1, BF16)
    Ys, d, w = Ys.cuda(), d.cuda(), w.cuda()
    want = [sq.sq_moe_combine(Ys, slot, offsets, w)] + list(sq.sq_moe_combine_bwd(d, Ys, slot, offsets, w))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [sq.sq_moe_combine(Ys, slot, offsets, w)] + list(sq.sq_moe_combine_bwd(d, Ys, slot, offsets, w))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


# ids that begin inside an aligned group of four, the longest sort of one launch, and lengths around a wave's step
@pytest.mark.parametrize("T,K,E", [(65536, 1, 300), (8191, 8, 64), (4097, 1, 5), (1023, 3, 17), (255, 1, 2), (1, 3, 4)])
@pytest.mark.parametrize("skip", [1, 2, 3])
@pytest.mark.parametrize("dtype", [np.int64, np.int32])
def test_sort_of_unaligned_ids(sq, T, K, E, skip, dtype):
    ids = _ids(T + skip, T, K, E, 0.1, dtype)
    base = torch.full((T * K + skip,), -1, dtype=torch.from_numpy(ids).dtype, device="cuda")
    base[skip:] = torch.from_numpy(ids).cuda().reshape(-1)
    got = sq.sq_moe_sort(base[skip:].view(T, K), E)
    for a, b in zip(got, step.moe_sort(ids, E)):
        assert np.array_equal(a.cpu().numpy(), b)


# rows beyond what the caches hold are read past them
@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("y_dtype,out_dtype", [(BF16, BF16), (F32, F32)])
def test_combine_of_many_bytes(sq, weighted, y_dtype, out_dtype):
    T, K, E, H = 5003, 4, 37, 2056
    offsets, _, slot = sq.sq_moe_sort(torch.from_numpy(_ids(5, T, K, E, 0.2)).cuda(), E)
    Ys = torch.randn((T * K, H), generator=torch.Generator("cuda").manual_seed(6), device="cuda").to(y_dtype)
    w = torch.rand((T, K), generator=torch.Generator("cuda").manual_seed(7), device="cuda") - 0.5 if weighted else None
    out = torch.full((T, H), float("nan"), dtype=out_dtype, device="cuda")
    sq.sq_moe_combine(Ys, slot, offsets, w, out=out)
    live = (slot < offsets[-1]).double()
    f = live * w.double() if weighted else live
    ref, mag = torch.zeros((2, T, H), dtype=torch.float64, device="cuda")
    for k in range(K):
        rows = Ys[slot[:, k].long()].double() * f[:, k, None]
        ref += rows
        mag += rows.abs()
    # K fused steps in fp32, and the rounding of the result
    bound = K * 2.0 ** -24 * 1.01 * mag + (2.0 ** -8 if out_dtype == BF16 else 0.0) * (ref.abs() + K * 2.0 ** -23 * mag)
    assert ((out.double() - ref).abs() <= bound).all()
