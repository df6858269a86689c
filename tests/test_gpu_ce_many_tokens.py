"""The loss of more tokens, or of more tiles of logits, than one dimension of a
launch holds (2^32 work-items), with rows as narrow as they may be.  Tokens repeat
after 1024, so every run of 1024 has to come out as the first; the first against
the oracle is what smaller calls are tested by."""

import pytest
import torch

from conftest import ensure_library, gpu_ready
from paper_2609_04526_amd import inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _case(T, V):
    n = T // 1024
    X, W = inputs.device_bf16_normal(1, (1024, 8)), inputs.device_bf16_normal(2, (V, 8))
    y = torch.arange(1024, device="cuda") * 37 % V
    return X, W, y, X.repeat(n, 1), y.repeat(n)


def test_loss_of_many_tiles(sq):
    T, V = 1 << 26, 8200
    X, W, y, Xn, yn = _case(T, V)
    got, one = sq.sq_ce_fwd("bf16", Xn, W, yn), sq.sq_ce_fwd("bf16", X, W, y)
    for a, b in zip(got, one):
        assert ((a.view(-1, 1024) - b).abs() <= 2.0 ** -18 * (1 + b.abs())).all()      # tiles of another extent


def test_gradient_of_many_tokens(sq):
    T, V = (1 << 25) + 1024, 60
    X, W, y, Xn, yn = _case(T, V)
    loss, lse = sq.sq_ce_fwd("bf16", Xn, W, yn)
    one, lse1 = sq.sq_ce_fwd("bf16", X, W, y)
    assert ((loss.view(-1, 1024) - one).abs() <= 2.0 ** -18 * (1 + one.abs())).all()
    dX = sq.sq_ce_bwd("bf16", Xn, W, yn, lse, torch.ones(T, device="cuda"))
    want = sq.sq_ce_bwd("bf16", X, W, y, lse1, torch.ones(1024, device="cuda"))
    p = (X.float() @ W.float().t()).softmax(1)
    bound = 2.0 ** -7 * ((p + torch.nn.functional.one_hot(y, V)) @ W.float().abs())
    assert ((dX.view(-1, 1024, 8) - want).abs() <= bound).all()
