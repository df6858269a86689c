"""The oracle of the step's operators against hand-worked values and against
differences of the functions whose gradients it states."""

import numpy as np
import pytest

from oracle import codec, step


def test_sort_by_hand():
    ids = np.array([[2, 0], [0, -1], [2, 7], [1, 0]])
    offsets, token, slot = step.moe_sort(ids, 3)
    # pairs in order: expert 0: 1, 2, 7; expert 1: 6; expert 2: 0, 4; dropped: 3, 5
    assert offsets.tolist() == [0, 3, 4, 6]
    assert token.tolist() == [0, 1, 3, 3, 0, 2, 1, 2]
    assert slot.reshape(-1).tolist() == [4, 0, 1, 6, 5, 7, 3, 2]


def test_combine_gradients_by_differences():
    g = np.random.default_rng(3)
    T, K, E, H = 5, 3, 4, 8
    ids = g.integers(-1, E, (T, K))
    offsets, _, slot = step.moe_sort(ids, E)
    R = int(offsets[-1])
    Ys, w, dOut = g.standard_normal((T * K, H)), g.random((T, K)), g.standard_normal((T, H))
    dYs, dw = step.moe_combine_bwd(dOut, Ys, slot, R, w)
    f = lambda y, v: float((dOut * step.moe_combine(y, slot, R, v)).sum())  # noqa: E731
    h = 1e-6
    for _ in range(40):
        i, j = g.integers(T * K), g.integers(H)
        a, b = Ys.copy(), Ys.copy()
        a[i, j] += h
        b[i, j] -= h
        assert abs((f(a, w) - f(b, w)) / (2 * h) - dYs[i, j]) < 1e-7
        t, k = g.integers(T), g.integers(K)
        a, b = w.copy(), w.copy()
        a[t, k] += h
        b[t, k] -= h
        assert abs((f(Ys, a) - f(Ys, b)) / (2 * h) - dw[t, k]) < 1e-7
    # the gather's gradient is the sum over a token's routed rows
    X, dXs = g.standard_normal((T, H)), g.standard_normal((T * K, H))
    lhs = float((step.moe_gather(X, slot, R) * dXs).sum())
    assert abs(lhs - float((X * step.moe_combine(dXs, slot, R)).sum())) < 1e-10


def test_int8_blocks_by_hand():
    x = np.zeros((1, 32))
    x[0, :4] = [127.5, -1.0, 0.5, 1.5]         # amax in [64, 128): k = 0, 127.5 rounds to 128 and saturates
    q, s = step.act_pack("int8", x)
    assert s[0, 0] == 127 and q.view(np.int8)[0, :4].tolist() == [127, -1, 0, 2]
    assert step.act_unpack("int8", q, s)[0, :4].tolist() == [127.0, -1.0, 0.0, 2.0]


def test_e4m3_blocks_by_hand():
    x = np.zeros((1, 96))
    x[0, 0], x[0, 1] = 448.0, 17.0             # exactly the largest value: k = 0; 17 lies between 16 and 18: even
    x[0, 32], x[0, 33] = 450.0, -3.0           # above it: k = 1; 225 between 224 and 240
    x[0, 64], x[0, 65] = 1.0, 1.0 / 512        # k = ceil(log2(1 / 448)) = -8
    q, s = step.act_pack("e4m3", x)
    assert s[0].tolist() == [127, 128, 119]
    v = step.act_unpack("e4m3", q, s)[0]
    assert v[:2].tolist() == [448.0, 16.0]
    assert v[32:34].tolist() == [448.0, -3.0]
    assert v[64:66].tolist() == [1.0, 1.0 / 512]


@pytest.mark.parametrize("act", ["int8", "e4m3"])
def test_blocks_without_a_value(act):
    x = np.zeros((2, 96))
    x[0, 5], x[0, 40], x[1, 70] = np.inf, np.nan, 2.0 ** -133
    q, s = step.act_pack(act, x)
    assert s[0].tolist() == [255, 255, 1] and s[1].tolist() == [1, 1, 1]
    v = step.act_unpack(act, q, s)
    assert np.isnan(v[0, :64]).all() and (v[0, 64:] == 0).all()
    # 2^-133 at the smallest scale 2^-126: 2^-7 rounds to 0 as a whole number and is a subnormal E4M3 value
    assert v[1, 70] == (0.0 if act == "int8" else 2.0 ** -133) and np.count_nonzero(v[1]) == (act == "e4m3")


@pytest.mark.parametrize("act,share", [("int8", 1 / 128), ("e4m3", 1 / 16)])
def test_rounding_error_of_a_block(act, share):
    """int8: half a step, amax / 128 at most; E4M3: half of 2^-3 of each value above its subnormals."""
    g = np.random.default_rng(11)
    x = g.standard_normal((64, 128)) * np.exp(g.standard_normal((64, 1)))
    v = step.act_unpack(act, *step.act_pack(act, x))
    amax = np.abs(x).reshape(64, 4, 32).max(-1).repeat(32, axis=1)
    bound = amax * share if act == "int8" else np.maximum(np.abs(x), amax * 2.0 ** -14) * share
    assert (np.abs(v - x) <= bound).all()


def test_e4m3_nearest_takes_the_even_byte():
    grid = step._E4M3
    mid = (grid[1:] + grid[:-1]) / 2
    got = step._e4m3_nearest(mid)
    assert (got % 2 == 0).all()
    assert [codec.e4m3_value(int(b)) for b in step._e4m3_nearest(-grid)][1:] == (-grid[1:]).tolist()


def test_cross_entropy_gradient_by_differences():
    g = np.random.default_rng(5)
    T, V, H = 6, 11, 7
    X, W, dl = g.standard_normal((T, H)), g.standard_normal((V, H)), g.standard_normal(T)
    y = np.array([0, 10, -100, 3, 11, 3])
    loss, lse = step.ce_fwd(X, W, y)
    assert loss[2] == lse[2] == loss[4] == lse[4] == 0.0
    assert abs(loss[0] + np.log(np.exp(X[0] @ W[0]) / np.exp(X[0] @ W.T).sum())) < 1e-12
    dX = step.ce_bwd(X, W, y, dl)
    assert (dX[2] == 0).all() and (dX[4] == 0).all()
    h = 1e-6
    for t in range(T):
        for j in range(H):
            a, b = X.copy(), X.copy()
            a[t, j] += h
            b[t, j] -= h
            d = (step.ce_fwd(a, W, y)[0][t] - step.ce_fwd(b, W, y)[0][t]) / (2 * h) * dl[t]
            assert abs(d - dX[t, j]) < 1e-7
