"""Activations in the layer's 4-bit storage against the oracle: every bf16 value
through both formats bit for bit, and the products of two 4-bit operands, single
and over experts, every element within the bound of its fp32 sum: the products
are exact, so a sum of I terms is off by 2 gamma_I sum |x w| at most, and a bf16
output by half a step (2^-8 of itself) more."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import linear, rtn, student
from paper_2609_04526_amd import inputs
from parity_check import elementwise_bound

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16, F32 = torch.bfloat16, torch.float32
BLOCK = {"mx": 32, "nv": 16}
XWS2, WS2 = 2.0 ** -9, float(np.float32(1.0 / 448.0))


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _all_bf16():
    return torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(BF16)


def _same(a, b):
    """Equal bits, any NaN for any other."""
    a, b = a.float(), b.float()
    return torch.equal(torch.nan_to_num(a, nan=777.0), torch.nan_to_num(b, nan=777.0)) and torch.equal(a.isnan(), b.isnan())


def _check_pack(sq, fmt, X, ws2):
    codes, scales = sq.sq_act4_pack(fmt, X.cuda(), ws2=ws2)
    rc, rs = student.act4_pack(fmt, X.float().numpy(), ws2)
    assert np.array_equal(scales.cpu().numpy(), rs)
    assert np.array_equal(codes.cpu().numpy(), rc)
    v = sq.sq_act4_unpack(fmt, codes, scales, ws2=ws2)
    # code times scale is exact in fp32, the scalar's product rounded once, then to bf16; a sum of magnitudes from
    # 2^128 on is an infinity in fp32 as it is in bf16
    with np.errstate(over="ignore"):
        want = student.act4_values(fmt, rc, rs).astype(np.float32) * np.float32(ws2 if fmt == "nv" else 1.0)
    assert v.dtype == BF16 and _same(v.cpu(), torch.from_numpy(want).to(BF16))


@pytest.mark.parametrize("fmt,ws2", [("mx", 1.0), ("nv", XWS2), ("nv", 0.013)])
def test_every_bf16_as_a_block_of_its_own(sq, fmt, ws2):
    X = torch.zeros((2048, 1024), dtype=BF16)
    X.view(-1, 32)[:, 5] = _all_bf16()
    _check_pack(sq, fmt, X, ws2)


@pytest.mark.parametrize("fmt,ws2", [("mx", 1.0), ("nv", XWS2), ("nv", 0.013)])
@pytest.mark.parametrize("top", [1.0, 6.0, 5.96875, 448.0, 2.0 ** -120, 2.0 ** -126, 2.0 ** 127])
def test_every_smaller_bf16_under_one_scale(sq, fmt, ws2, top):
    v = _all_bf16()
    v = v[v.float().abs() <= top]
    B = BLOCK[fmt]
    v = torch.cat((v, v.new_zeros((-len(v)) % (B - 1))))
    X = torch.cat((v.view(-1, B - 1), torch.full((len(v) // (B - 1), 1), top, dtype=BF16)), 1)
    X = torch.cat((X, X.new_zeros(((-len(X)) % 32, B)))).view(-1, 32 * B)
    _check_pack(sq, fmt, X, ws2)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("T,I", [(1, 32), (3, 96), (17, 544), (65, 4096)])
def test_as_the_requantiser(sq, fmt, T, I):
    """Codes and scales of finite values are rtn_quantize's (whose rows come in eights)."""
    X = inputs.bf16_normal(T, (T, I)) * 3
    X[T // 2, 7] = float("inf")
    X[0, 20] = float("nan")
    _check_pack(sq, fmt, X, XWS2)
    X = inputs.bf16_normal(T + 1, (8 * T, I)).cuda()
    codes, scales = sq.sq_act4_pack(fmt, X, ws2=XWS2)
    rc, rs, _ = sq.rtn_quantize(fmt, X, sq.TIE_EVEN, ws2_in=XWS2)
    assert torch.equal(codes, rc) and torch.equal(scales, rs)


def _layer(fmt, seed, O, I):
    codes = inputs.codes_uniform(seed, O, I)
    if fmt == "mx":
        scales = inputs.e8m0_uniform_exponents(seed + 1, O, I // 32, -9, -2)
    else:
        scales = inputs.e4m3_abs_normal(seed + 1, O, I // 16)
    return codes, scales


def _rows(fmt, seed, T, I):
    """An activation with uneven blocks, kept: (codes, scales, values without the scalar)."""
    g = inputs.rng(seed)
    X = g.standard_normal((T, I)) * np.exp2(np.repeat(g.integers(-6, 3, (T, I // 32)), 32, axis=1))
    X = torch.from_numpy(X).to(BF16)
    codes, scales = student.act4_pack(fmt, X.float().numpy(), XWS2)
    return codes, scales, student.act4_values(fmt, codes, scales)


def _check(Y, ref, mag, I, extra=0):
    Y = Y.cpu()
    bound = elementwise_bound(mag, I + extra)
    if Y.dtype == BF16:
        bound = bound * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(ref) + 1e-38
    bad = ~(np.abs(Y.double().numpy() - ref) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], bad.mean())


def _dev(*a):
    return [torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in a]


# one token to several tiles, around every tile's edge; inputs that end inside a step of 128 and of 256
@pytest.mark.parametrize("T,O,I", [(1, 8, 32), (1, 264, 4096), (2, 24, 96), (15, 520, 160), (16, 136, 128), (17, 256, 1056),
                                   (33, 264, 544), (64, 512, 256), (65, 264, 320), (100, 1032, 2048), (127, 8, 64),
                                   (128, 776, 512), (129, 256, 288), (255, 520, 1024), (257, 264, 96), (300, 1544, 640),
                                   (513, 512, 384), (700, 2056, 1152)])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_products(sq, fmt, T, O, I, out_dtype):
    codes, scales = _layer(fmt, T + O, O, I)
    xc, xs, x = _rows(fmt, T, T, I)
    w = linear.dequant(fmt, codes, scales, WS2 if fmt == "nv" else 1.0)
    x = x * (XWS2 if fmt == "nv" else 1.0)
    Y = torch.full((T, O), float("nan"), dtype=out_dtype, device="cuda")
    sq.sq_fwd_act4(fmt, *_dev(xc, xs, codes, scales), x_ws2=XWS2, ws2=WS2, Y=Y)
    _check(Y, x @ w.T, np.abs(x) @ np.abs(w).T, I, 4)


def _dequant(codes, scales):
    """MXFP4 values in 64 bits on the device."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    v = table[torch.stack((codes & 15, codes >> 4), -1).long()].view(scales.shape + (32,))
    return (v * torch.exp2(scales.double() - 127)[..., None]).view(codes.shape[:-1] + (-1,))


def _check_device(Y, ref, mag, depth):
    bound = 2 * depth * 2.0 ** -24 / (1 - depth * 2.0 ** -24) * mag + 1e-38
    if Y.dtype == BF16:
        bound = bound * (1 + 2.0 ** -7) + 2.0 ** -8 * ref.abs()
    bad = ~((Y.double() - ref).abs() <= bound)
    assert not bad.any(), (bad.nonzero()[:5].tolist(), bad.double().mean().item())


# several rounds of the largest tiles; one round of each other kind; sums split over workgroups, of whole and of odd inputs
@pytest.mark.parametrize("T,O,I", [(4100, 4104, 544), (8200, 2056, 160), (2000, 4096, 288), (1030, 4096, 512), (600, 14336, 96),
                                   (70, 264, 6176), (100, 256, 8192), (65, 1032, 14336), (300, 136, 7200), (63, 4104, 6144)])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_larger_products(sq, T, O, I, out_dtype):
    codes, scales = _dev(*_layer("mx", T + O, O, I))
    xc, xs, _ = _rows("mx", T % 97, min(T, 500), I)
    xc, xs = (torch.from_numpy(v).cuda().repeat((T + len(v) - 1) // len(v), 1)[:T].contiguous() for v in (xc, xs))
    xs = (xs.int() + torch.arange(T, device="cuda", dtype=torch.int32)[:, None] % 5).to(torch.uint8)   # no two parts alike
    Y = torch.full((T, O), float("nan"), dtype=out_dtype, device="cuda")
    sq.sq_fwd_act4("mx", xc, xs, codes, scales, Y=Y)
    x, w = _dequant(xc, xs), _dequant(codes, scales)
    _check_device(Y, x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous(), I + 8)


@pytest.mark.parametrize("E,T,K,O,I", [(8, 4096, 2, 776, 160), (16, 2000, 3, 520, 288), (40, 700, 4, 264, 96), (8, 512, 2, 1536, 256),
                                       (128, 16, 8, 768, 128), (4, 333, 1, 4104, 544)])
def test_larger_experts(sq, E, T, K, O, I):
    """Uneven ranges under every kind of tile, their offsets from the sort, some pairs dropped."""
    g = inputs.rng(E + T)
    ids = np.minimum((E * g.random((T, K)) ** 1.7).astype(np.int64), E - 1)
    ids[g.random((T, K)) < 0.03] = -1
    offsets, rows, _ = sq.sq_moe_sort(torch.from_numpy(ids).cuda(), E)
    codes, scales = (v.view(E, O, -1) for v in _dev(*_layer("mx", E, E * O, I)))
    xc, xs, _ = _rows("mx", T, T, I)
    xc, xs = _dev(xc, xs)
    Y = torch.full((T * K, O), float("nan"), dtype=BF16, device="cuda")
    sq.sq_fwd_act4_batched("mx", xc, xs, rows, offsets, codes, scales, Y=Y)
    x, o = _dequant(xc, xs)[rows.long()], offsets.tolist()
    for e in range(E):
        w, r = _dequant(codes[e], scales[e]), x[o[e]:o[e + 1]]
        _check_device(Y[o[e]:o[e + 1]], r @ w.t().contiguous(), r.abs() @ w.abs().t().contiguous(), I)
    assert not Y[o[E]:].any()


@pytest.mark.parametrize("T", [5, 300])
def test_every_scale_byte(sq, T):
    """All pairs of E8M0 bytes whose product stays in fp32, and NaN scales of either operand."""
    g = inputs.rng(T)
    I, O = 256, 264
    codes, xc = inputs.codes_uniform(1, O, I), inputs.codes_uniform(2, T, I)
    xs = np.repeat(g.integers(0, 255, (T, 1)), I // 32, axis=1).astype(np.uint8)
    ws = np.repeat(g.integers(0, 255, (O, 1)), I // 32, axis=1).astype(np.uint8)
    xs[0], xs[1], ws[0], ws[1] = 0, 254, 0, 254
    Y = sq.sq_fwd_act4("mx", *_dev(xc, xs, codes, ws)).cpu().double().numpy()
    x, w = linear.dequant("mx", xc, xs), linear.dequant("mx", codes, ws)
    ref, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    inside = (mag < 2.0 ** 126) & (mag > 2.0 ** -90)
    assert inside.any()
    assert (np.abs(Y - ref) <= elementwise_bound(mag, I))[inside].all()
    # partial sums from 2^128 on are infinite; where they have both signs, as the terms' signs do, their sum is NaN
    assert not np.isfinite(Y[np.abs(ref) >= 2.0 ** 129]).any()
    # what lies below fp32's normal numbers may be flushed
    assert (np.abs(Y - ref) <= 2.0 ** -90 * 2 * 2.0 ** -20 + 2.0 ** -120)[mag <= 2.0 ** -90].all()
    xs[3, 5] = 255
    ws[7, 2] = 255
    Z = sq.sq_fwd_act4("mx", *_dev(xc, xs, codes, ws)).cpu().double().numpy()
    assert np.isnan(Z[3]).all() and np.isnan(Z[:, 7]).all()
    # nothing else is touched
    assert np.array_equal(*(np.delete(np.delete(v, 3, 0), 7, 1) for v in (Y, Z)), equal_nan=True)


def _split(g, E, N, kind):
    """Offsets of E ranges that fill N rows, or leave some at the end."""
    if kind == "even":
        cut = np.sort(g.integers(0, N + 1, E))
        cut[-1] = N
    elif kind == "one":
        cut = np.where(np.arange(E) >= E // 2, N, 0)
    elif kind == "dropped":
        cut = np.sort(g.integers(0, N - N // 4 + 1, E))
    else:
        cut = np.zeros(E, np.int64)
    return np.concatenate([[0], cut]).astype(np.int32)


@pytest.mark.parametrize("kind", ["even", "one", "dropped", "empty"])
@pytest.mark.parametrize("E,T,N,O,I", [(1, 4, 7, 24, 32), (3, 9, 40, 264, 160), (7, 30, 130, 136, 256), (130, 16, 128, 40, 96), (700, 16, 300, 24, 64), (8192, 50, 400, 16, 32),
                                       (5, 200, 1200, 520, 288), (2, 300, 900, 256, 512), (70, 64, 700, 72, 128)])
def test_experts(sq, E, T, N, O, I, kind):
    g = inputs.rng(E * N)
    codes, scales = _layer("mx", N, E * O, I)
    xc, xs, x = _rows("mx", T, T, I)
    offsets, rows = _split(g, E, N, kind), g.integers(0, T, N).astype(np.int32)
    rows[:2] = [-1, T]                                      # read as rows of zeros
    w = linear.dequant("mx", codes, scales).reshape(E, O, I)
    c3, s3 = codes.reshape(E, O, -1), scales.reshape(E, O, -1)
    for out_dtype in (F32, BF16):
        Y = torch.full((N, O), float("nan"), dtype=out_dtype, device="cuda")
        sq.sq_fwd_act4_batched("mx", *_dev(xc, xs, rows, offsets, c3, s3), Y=Y)
        _check(Y, student.experts(x, rows, offsets, w), student.experts(np.abs(x), rows, offsets, np.abs(w)), I)


@pytest.mark.parametrize("kind", ["even", "one", "dropped", "empty"])
@pytest.mark.parametrize("E,T,N,O,I", [(200, 64, 512, 1288, 64), (1500, 40, 1600, 264, 96), (30, 200, 3300, 2056, 288),
                                       (12, 300, 3000, 4104, 544)])
def test_experts_of_several_rounds(sq, E, T, N, O, I, kind):
    """So many tiles that the chunks come from a table, and last ones take smaller tiles; rows before the first range as well."""
    g = inputs.rng(E + N)
    codes, scales = (v.view(E, O, -1) for v in _dev(*_layer("mx", N, E * O, I)))
    xc, xs, _ = _rows("mx", T, T, I)
    xc, xs = _dev(xc, xs)
    offsets, rows = _split(g, E, N, kind), g.integers(0, T, N).astype(np.int32)
    if kind == "dropped":
        offsets = np.maximum(offsets, 3)
    Y = torch.full((N, O), float("nan"), dtype=BF16, device="cuda")
    sq.sq_fwd_act4_batched("mx", xc, xs, *_dev(rows, offsets), codes, scales, Y=Y)
    x = _dequant(xc, xs)[torch.from_numpy(rows).long().cuda()]
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        w, r = _dequant(codes[e], scales[e]), x[lo:hi]
        _check_device(Y[lo:hi], r @ w.t().contiguous(), r.abs() @ w.abs().t().contiguous(), I)
    assert not Y[:offsets[0]].any() and not Y[offsets[E]:].any()


@pytest.mark.parametrize("E,T,N,O,I", [(200, 64, 512, 1288, 64), (12, 300, 3000, 4104, 96), (8, 60, 200, 264, 160), (4, 5, 10, 40, 64)])
def test_experts_captured_with_other_offsets(sq, E, T, N, O, I):
    """A graph of the product follows the offsets and rows that lie in its buffers at each replay."""
    g = inputs.rng(E + T)
    codes, scales = (v.view(E, O, -1) for v in _dev(*_layer("mx", N, E * O, I)))
    xc, xs, _ = _rows("mx", T, T, I)
    xc, xs = _dev(xc, xs)
    offsets, rows = _dev(_split(g, E, N, "even"), g.integers(0, T, N).astype(np.int32))
    ws = torch.empty(max(sq.sq_fwd_act4_batched_workspace("mx", E, T, N, O, I), 1), dtype=torch.uint8, device="cuda")
    Y = torch.empty((N, O), dtype=BF16, device="cuda")
    run = lambda out: sq.sq_fwd_act4_batched("mx", xc, xs, rows, offsets, codes, scales, Y=out, workspace=ws)
    run(Y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(Y)
    for kind in ("one", "dropped", "empty", "even", "even"):
        offsets.copy_(torch.from_numpy(_split(g, E, N, kind)))
        rows.copy_(torch.from_numpy(g.integers(0, T, N).astype(np.int32)))
        want = run(torch.full((N, O), float("nan"), dtype=BF16, device="cuda"))
        Y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want)


def test_experts_rows_in_place(sq):
    """Without row numbers, row s is row s; rows before the first range are zeros too; offsets past the rows are held."""
    E, N, O, I = 4, 90, 72, 128
    codes, scales = _layer("mx", 3, E * O, I)
    xc, xs, x = _rows("mx", 4, N, I)
    w = linear.dequant("mx", codes, scales).reshape(E, O, I)
    d = _dev(xc, xs, codes.reshape(E, O, -1), scales.reshape(E, O, -1))
    for offsets in ([5, 20, 20, 61, 80], [0, 30, 60, 90, 900], [-7, 1, 2, 3, 4]):
        o = np.array(offsets, np.int32)
        Y = torch.full((N, O), float("nan"), device="cuda")
        sq.sq_fwd_act4_batched("mx", d[0], d[1], None, torch.from_numpy(o).cuda(), d[2], d[3], Y=Y)
        held = np.clip(o, 0, N)
        _check(Y, student.experts(x, np.arange(N), held, w), student.experts(np.abs(x), np.arange(N), held, np.abs(w)), I)


@pytest.mark.parametrize("T", [3, 700])
def test_nan_blocks_of_either_nvfp4_operand(sq, T):
    """A kept block that held a NaN or Inf makes its row NaN, and a NaN scale of the layer its output; no other."""
    O, I = 72, 160
    codes, scales = _layer("nv", 5, O, I)
    X = torch.randn(T, I, generator=torch.Generator().manual_seed(T)).to(BF16)
    X[1, 37], X[2, 159] = float("nan"), float("-inf")
    xc, xs = sq.sq_act4_pack("nv", X.cuda(), XWS2)
    c, s = _dev(codes, scales)
    s[5, 3] = 0x7F
    Y = sq.sq_fwd_act4("nv", xc, xs, c, s, x_ws2=XWS2, ws2=WS2)
    bad = torch.zeros((T, O), dtype=torch.bool)
    bad[1:3], bad[:, 5] = True, True
    assert torch.equal(Y.cpu().isnan(), bad)


@pytest.mark.parametrize("G", [1, 4])
def test_experts_of_no_kept_row(sq, G):
    """Without a kept row every row number lies outside, and all of Y is zeros."""
    E, N, O, I = 3, 90, 264, 32 * G
    codes, scales = (v.view(E, O, -1) for v in _dev(*_layer("mx", 8, E * O, I)))
    offsets, rows = _dev(np.array([0, 10, 60, 90], np.int32), np.arange(N, dtype=np.int32))
    x, xs = torch.empty((0, I // 2), dtype=torch.uint8, device="cuda"), torch.empty((0, G), dtype=torch.uint8, device="cuda")
    Y = torch.full((N, O), float("nan"), device="cuda")
    sq.sq_fwd_act4_batched("mx", x, xs, rows, offsets, codes, scales, Y=Y)
    assert not Y.any()


def test_empty_calls(sq):
    c, s = _dev(*_layer("mx", 1, 64, 128))
    e = torch.empty((0, 64), dtype=torch.uint8, device="cuda")
    es = torch.empty((0, 4), dtype=torch.uint8, device="cuda")
    assert sq.sq_fwd_act4("mx", e, es, c, s).shape == (0, 64)
    rows, offsets = torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    assert sq.sq_fwd_act4_batched("mx", e, es, rows, offsets, c[None], s[None]).shape == (0, 64)
    codes, scales = sq.sq_act4_pack("mx", torch.empty((0, 128), dtype=BF16, device="cuda"))
    assert codes.shape == (0, 64) and sq.sq_act4_unpack("mx", codes, scales).shape == (0, 128)


def test_same_bits_on_every_run(sq):
    for T in (3, 40, 300):
        xc, xs, _ = _rows("mx", T, T, 1024)
        d = _dev(xc, xs, *_layer("mx", 5, 520, 1024))
        assert torch.equal(sq.sq_fwd_act4("mx", *d), sq.sq_fwd_act4("mx", *d))


# inputs that end within a stage of 256, with scale rows of whole words (whose next row's bytes lie in the same copy) and
# of others, through tiles of every extent and split sums
@pytest.mark.parametrize("T,O,I", [(300, 264, 128), (300, 264, 384), (65, 264, 640), (129, 520, 160), (700, 2056, 384), (2000, 4096, 128),
                                   (4100, 4104, 384), (100, 264, 6272), (100, 264, 6304), (5, 264, 384), (5, 264, 96), (40, 520, 640)])
def test_nan_scales_beside_the_inputs_end(sq, T, O, I):
    """A NaN scale in a row's first block reaches that row of Y, or column, and not the row before it, whose stage ends there."""
    g = inputs.rng(T + I)
    xc, codes = inputs.codes_uniform(1, T, I), inputs.codes_uniform(2, O, I)
    xs, ws = g.integers(118, 128, (T, I // 32)).astype(np.uint8), g.integers(118, 128, (O, I // 32)).astype(np.uint8)
    d = _dev(xc, xs, codes, ws)
    for out_dtype in (F32, BF16):
        want = sq.sq_fwd_act4("mx", *d, out_dtype=out_dtype)
        assert torch.isfinite(want).all()
        r, c = [v for v in (1, 3, 32, 64, T - 1) if v < T], [0, 7, 63, 64, 128, O - 1]
        nx, nw = d[1].clone(), d[3].clone()
        nx[r, 0], nw[c, 0] = 0xFF, 0xFF
        Y = sq.sq_fwd_act4("mx", d[0], nx, d[2], nw, out_dtype=out_dtype)
        bad = torch.zeros((T, O), dtype=torch.bool, device="cuda")
        bad[r], bad[:, c] = True, True
        assert torch.equal(Y.isnan(), bad)
        assert torch.equal(torch.where(bad, torch.zeros_like(Y), Y), torch.where(bad, torch.zeros_like(Y), want))


@pytest.mark.parametrize("E,T,N,O,I", [(200, 64, 512, 1288, 128), (30, 200, 3300, 2056, 384), (12, 300, 3000, 4104, 640), (8, 60, 200, 264, 384)])
def test_nan_scales_beside_the_inputs_end_of_experts(sq, E, T, N, O, I):
    """The same over experts, the last row of one and the first of the next among them."""
    g = inputs.rng(E + I)
    xc, codes = inputs.codes_uniform(1, T, I), inputs.codes_uniform(2, E * O, I).reshape(E, O, -1)
    xs, ws = g.integers(118, 128, (T, I // 32)).astype(np.uint8), g.integers(118, 128, (E, O, I // 32)).astype(np.uint8)
    offsets, rows = _split(g, E, N, "even"), g.integers(0, T, N).astype(np.int32)
    xc, xs, rows, offsets, codes, ws = _dev(xc, xs, rows, offsets, codes, ws)
    want = sq.sq_fwd_act4_batched("mx", xc, xs, rows, offsets, codes, ws)
    assert torch.isfinite(want).all()
    nx, nw = xs.clone(), ws.clone()
    r, e, c = [1, 7, T - 1], [0, E // 2, E - 1], [0, 64, O - 1]
    nx[r, 0] = 0xFF
    for k in e:
        nw[k, c, 0] = 0xFF
    Y = sq.sq_fwd_act4_batched("mx", xc, nx, rows, offsets, codes, nw)
    bad = torch.isin(rows, torch.tensor(r, dtype=torch.int32, device="cuda"))[:, None].repeat(1, O)
    o = offsets.tolist()
    for k in e:
        bad[o[k]:o[k + 1], c] = True
    bad[:o[0]], bad[o[E]:] = False, False
    assert torch.equal(Y.isnan(), bad)
    assert torch.equal(torch.where(bad, torch.zeros_like(Y), Y), torch.where(bad, torch.zeros_like(Y), want))


@pytest.mark.parametrize("kind", ["even", "one", "dropped", "empty"])
@pytest.mark.parametrize("E,T,N,O,I", [(200, 64, 512, 1288, 64), (30, 200, 3300, 2056, 288), (12, 300, 3000, 4104, 544)])
def test_experts_of_several_rounds_to_fp32(sq, E, T, N, O, I, kind):
    """Chunks from a table with tiles of 64, 128 and 256 rows, whose fp32 outputs leave 32 rows at a time."""
    g = inputs.rng(E + N)
    codes, scales = (v.view(E, O, -1) for v in _dev(*_layer("mx", N, E * O, I)))
    xc, xs, _ = _rows("mx", T, T, I)
    xc, xs = _dev(xc, xs)
    offsets, rows = _split(g, E, N, kind), g.integers(0, T, N).astype(np.int32)
    if kind == "dropped":
        offsets = np.maximum(offsets, 3)
    Y = torch.full((N, O), float("nan"), device="cuda")
    sq.sq_fwd_act4_batched("mx", xc, xs, *_dev(rows, offsets), codes, scales, Y=Y)
    x = _dequant(xc, xs)[torch.from_numpy(rows).long().cuda()]
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        w, r = _dequant(codes[e], scales[e]), x[lo:hi]
        _check_device(Y[lo:hi], r @ w.t().contiguous(), r.abs() @ w.abs().t().contiguous(), I)
    assert not Y[:offsets[0]].any() and not Y[offsets[E]:].any()
