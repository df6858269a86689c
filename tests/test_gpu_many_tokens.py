"""Calls of more tokens than one dimension of a launch holds (2^32 work-items),
with rows as narrow as they may be."""

import pytest
import torch

from conftest import ensure_library, gpu_ready

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16 = torch.bfloat16
T = (1 << 26) + 5


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


@pytest.fixture(scope="module")
def rows():
    """A row of 8 small whole numbers for every token, and its place: the tokens in reverse, the last two dropped."""
    X = (torch.arange(T, device="cuda")[:, None] % 251 + torch.arange(8, device="cuda")).to(BF16)
    slot = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")[:, None].contiguous()
    return X, slot, torch.tensor([0, T - 2], dtype=torch.int32, device="cuda")


def test_gather(sq, rows):
    X, slot, offsets = rows
    Xs = torch.full((T, 8), float("nan"), dtype=BF16, device="cuda")
    sq.sq_moe_gather(X, slot, offsets, Xs=Xs)
    want = X.flip(0)
    want[T - 2:] = 0
    assert torch.equal(Xs, want)


@pytest.mark.parametrize("weighted", [False, True])
def test_combine(sq, rows, weighted):
    X, slot, offsets = rows
    w = torch.full((T, 1), 2.0, device="cuda") if weighted else None
    out = sq.sq_moe_combine(X, slot, offsets, w, out_dtype=BF16)
    want = X.flip(0) * (2 if weighted else 1)
    want[:2] = 0                                               # the tokens of the last two places
    assert torch.equal(out, want)


def test_combine_bwd(sq, rows):
    X, slot, offsets = rows
    w = torch.full((T, 1), 2.0, device="cuda")
    dYs, dw = sq.sq_moe_combine_bwd(X, X, slot, offsets, w)
    want = X.flip(0) * 2
    want[T - 2:] = 0
    assert torch.equal(dYs, want)
    want = (X.float() * X.flip(0).float()).sum(1, keepdim=True)              # whole numbers below 2^24
    want[:2] = 0
    assert torch.equal(dw, want)
