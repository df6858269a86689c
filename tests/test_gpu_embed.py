"""Embedding lookup and its gradients against the oracle.

Bounds.  A looked-up value takes at most three fp32 roundings (the NVFP4 scale,
its product with the code, the factor) and the output's.  A gradient is an fp32
sum of n tokens (times 32 or 16 columns for the scales), off by 2 gamma_n of the
sum of magnitudes, and the factor's and the output's rounding."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import linear, student
from paper_2609_04526_amd import inputs
from parity_check import elementwise_bound

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16, F32 = torch.bfloat16, torch.float32
WS2 = float(np.float32(1.0 / 448.0))
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _table(head, seed, V, I):
    if head == "bf16":
        W = inputs.bf16_normal(seed, (V, I))
        return W.cuda(), None, W.double().numpy()
    codes = inputs.codes_uniform(seed, V, I)
    scales = inputs.e8m0_uniform_exponents(seed + 1, V, I // 32, -9, 3) if head == "mx" else inputs.e4m3_abs_normal(seed + 1, V, I // 16)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), linear.dequant(head, codes, scales, WS2)


def _ids(g, kind, T, V):
    if kind == "one":
        return np.full(T, V // 2)
    if kind == "few":
        return g.integers(0, min(V, 3), T)
    if kind == "ragged":                                       # runs of many lengths, and ids outside the table
        ids = (V * g.random(T) ** 4).astype(np.int64)
        return np.where(g.random(T) < 0.2, g.choice([-100, -1, V, V + 3, 2 ** 31 - 1], T), ids)
    if kind == "none":
        return np.full(T, -1)
    return g.integers(0, V, T)


SHAPES = [(1, 1, 32), (2, 5, 64), (63, 40, 96), (64, 1000, 32), (65, 300, 2080), (200, 37, 256), (1000, 513, 544), (2500, 700, 64)]


@pytest.mark.parametrize("head", ["bf16", "mx", "nv"])
@pytest.mark.parametrize("T,V,I", SHAPES)
def test_lookup(sq, head, T, V, I):
    W, scales, w = _table(head, T, V, I)
    for n, (id_dtype, out_dtype) in enumerate([(torch.int64, F32), (torch.int32, BF16)]):
        ids = _ids(inputs.rng(T + n), "ragged", T, V)
        factor = float(np.float32(np.sqrt(I)))
        out = torch.full((T, I), float("nan"), dtype=out_dtype, device="cuda")
        sq.sq_embed_fwd(head, torch.from_numpy(ids).to(id_dtype).cuda(), W, scales=scales, ws2=WS2, factor=factor, out=out)
        ref = student.embed_fwd(ids, w, factor)
        err = np.abs(out.double().cpu().numpy() - ref)
        assert (err <= np.abs(ref) * (HALF[out_dtype] * (1 + 2.0 ** -10) + 4 * 2.0 ** -24)).all()


def _check_grad(sq, head, T, V, I, kind, id_dtype, d_dtype, out_dtype):
    g = inputs.rng(T + V)
    ids = _ids(g, kind, T, V)
    dOut = torch.from_numpy(g.standard_normal((T, I))).to(d_dtype)
    d = dOut.double().numpy()
    factor = 1.7
    idd, dd = torch.from_numpy(ids).to(id_dtype).cuda(), dOut.cuda()
    n = max(1, np.bincount(ids[(ids >= 0) & (ids < V)], minlength=1).max())
    if head == "bf16":
        got = torch.full((V, I), float("nan"), dtype=out_dtype, device="cuda")
        sq.sq_embed_bwd(idd, dd, V, factor=factor, dW=got)
        again = sq.sq_embed_bwd(idd, dd, V, factor=factor, out_dtype=out_dtype)
        ref, mag, depth = student.embed_bwd(ids, d, V, factor), student.embed_bwd(ids, np.abs(d), V, factor), n + 3
    else:
        codes = inputs.codes_uniform(T, V, I)
        cd = torch.from_numpy(codes).cuda()
        got = torch.full((V, I // (32 if head == "mx" else 16)), float("nan"), device="cuda")
        sq.sq_embed_bwd_dscale(head, idd, dd, cd, factor=factor, dS=got)
        again = sq.sq_embed_bwd_dscale(head, idd, dd, cd, factor=factor)
        ref = student.embed_bwd_dscale(head, ids, d, codes, factor)
        mag = np.abs(linear.code_values(codes)) * student.embed_bwd(ids, np.abs(d), V, factor)
        mag, depth = mag.reshape(got.shape + (-1,)).sum(-1), n + 36
    assert torch.equal(got, again)                             # the same bits on every run
    bound = elementwise_bound(mag, depth) + HALF[out_dtype if head == "bf16" else F32] * np.abs(ref) * 1.01
    bad = ~(np.abs(got.double().cpu().numpy() - ref) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:5], bad.mean())
    assert not np.where(mag == 0, got.float().cpu().numpy(), 0).any()


@pytest.mark.parametrize("kind", ["even", "ragged", "one", "few", "none"])
@pytest.mark.parametrize("head", ["bf16", "mx", "nv"])
@pytest.mark.parametrize("T,V,I", SHAPES)
def test_gradients(sq, head, T, V, I, kind):
    n = T + V + len(kind)
    _check_grad(sq, head, T, V, I, kind, (torch.int64, torch.int32)[n % 2], (F32, BF16)[n // 2 % 2], (F32, BF16)[n // 3 % 2])


@pytest.mark.parametrize("kind", ["ragged", "one"])
@pytest.mark.parametrize("T,V", [(1023, 511), (1024, 512), (1025, 5000), (16384, 50001), (20000, 300001), (70000, 1000), (131073, 600),
                                 (140000, 270001)])
def test_many_tokens(sq, T, V, kind):
    """The sort by 9 bits a pass: two passes, three from 2^18 ids on; more than 131072 tokens take the other sort."""
    _check_grad(sq, "mx", T, V, 32, kind, torch.int64, BF16, F32)


def test_no_tokens(sq):
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    d = torch.empty((0, 64), device="cuda")
    dW = torch.full((5, 64), 3.0, device="cuda")
    assert not sq.sq_embed_bwd(ids, d, 5, dW=dW).any()
    dS = torch.full((5, 2), 3.0, device="cuda")
    assert not sq.sq_embed_bwd_dscale("mx", ids, d, torch.zeros((5, 32), dtype=torch.uint8, device="cuda"), dS=dS).any()
    assert sq.sq_embed_fwd("bf16", ids, torch.zeros((5, 64), dtype=BF16, device="cuda")).shape == (0, 64)


def test_nan_stays_in_its_rows(sq):
    """A NaN of an ignored token reaches nothing, of another token its own row only."""
    ids = torch.tensor([3, -1, 3, 1], device="cuda")
    d = torch.ones((4, 64), device="cuda")
    d[1], d[3, 5] = float("nan"), float("inf")
    dW = sq.sq_embed_bwd(ids, d, 4)
    assert dW[0].eq(0).all() and dW[2].eq(0).all() and dW[3].eq(2).all() and torch.isinf(dW[1, 5]) and dW[1].isinf().sum() == 1
