"""Distillation of more tokens than one dimension of a launch holds by 16 in 1024
work-items (2^26 of them are 2^32), up to the most that are taken (2^27 - 1, whose
rows end 32-bit offsets), with rows as narrow as they may be.  Tokens
repeat after 1024, some of them ignored, so every run of 1024 has to come out as
the first; that one is compared with the oracle.

The runs' tiles may have other extents, so lse and loss differ by twice their own
steps, own = (max |s| + 64) 2^-22 each, and dX by the rounding of logit gradients
to bf16 (2^-8 of p + q against |W|, twice)."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import student
from paper_2609_04526_amd import inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

V, I, K = 60, 8, 2


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    yield _sq
    torch.cuda.empty_cache()


def _case(T):
    n = (T + 1023) // 1024
    X, W = inputs.bf16_normal(1, (1024, I)), inputs.bf16_normal(2, (V, I))
    g = inputs.rng(3)
    ids = g.integers(0, V, (1024, K)).astype(np.int32)
    ids[::5, 1] = -1
    ids[::7] = -1
    z = g.standard_normal((1024, K)).astype(np.float32)
    one = [X.cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(z).cuda()]
    return X, W, ids, z, one, [v.repeat(n, 1)[:T] for v in one]


@pytest.mark.parametrize("T", [1 << 26, (1 << 26) + 1024, (1 << 27) - 1])
def test_loss(sq, T):
    X, W, ids, z, one, many = _case(T)
    loss, lse = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    _, _, picked = sq.sq_distill_fwd("bf16", many[0], W.cuda(), many[1], many[2], loss=loss, lse=lse)
    x, w = X.double().numpy(), W.double().numpy()
    own = (np.abs(x @ w.T).max() + 64) * 2.0 ** -22
    r = student.distill_fwd(x, w, ids, z, 1.0)
    for got, want in zip((loss, lse), r):
        first = got[:1024]
        assert (np.abs(first.double().cpu().numpy() - want) <= 8 * own).all()
        # in parts, whose differences take no memory to speak of
        whole = T // 1024 * 1024
        for part in got[:whole].view(-1, 1024).split(4096):
            assert ((part - first).abs() <= 4 * own).all()
        assert ((got[whole:] - first[:T - whole]).abs() <= 4 * own).all()
    assert all((part == picked[:1024]).all() for part in picked[:whole].view(-1, 1024, K).split(4096))


def test_gradient(sq):
    T = (1 << 25) + 1024
    X, W, ids, z, one, many = _case(T)
    W = W.cuda()
    loss, lse, picked = sq.sq_distill_fwd("bf16", many[0], W, many[1], many[2])
    dX = sq.sq_distill_bwd("bf16", many[0], W, many[1], many[2], lse, picked, torch.ones(T, device="cuda"))
    l1 = sq.sq_distill_fwd("bf16", one[0], W, one[1], one[2])
    want = sq.sq_distill_bwd("bf16", one[0], W, one[1], one[2], l1[1], l1[2], torch.ones(1024, device="cuda"))
    counts, q = student.teacher(ids, z, 1.0, V)
    p = (X.cuda().float() @ W.float().t()).softmax(1)
    p.scatter_add_(1, torch.from_numpy(np.where(counts, ids, 0)).long().cuda(), torch.from_numpy(q).float().cuda())
    bound = 2.0 ** -7 * (p @ W.float().abs())
    assert all(((part - want).abs() <= bound).all() for part in dX.view(-1, 1024, I).split(4096))
    assert not dX.view(-1, 1024, I)[:, ::7].any()
