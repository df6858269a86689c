"""The scale gradient from 8 bits under every scale byte, the largest ones among
them: one kept value reaches each output, so dS is half that value, exactly.

An int8 block whose largest value is 2^127 or more has scale byte 248, and its
values are finite; bytes from 249 on come from a caller only, and some of their
products leave bf16's range."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import step
from paper_2609_04526_amd import inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16 = torch.bfloat16
BLOCK = {"mx": 32, "nv": 16}


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _same(a, b):
    """Equal bits, any NaN equal to any other."""
    nan = torch.isnan(a)
    return torch.equal(nan, torch.isnan(b)) and torch.equal(a[~nan], b[~nan])


def _one_code_per_block(O, I):
    """Codes of 0.5 at column j = o (mod 32) of output o, zeros elsewhere: packed, low nibble first."""
    c = (np.arange(I)[None, :] % 32 == np.arange(O)[:, None] % 32).astype(np.uint8)
    return torch.from_numpy(c[:, 0::2] | c[:, 1::2] << 4).cuda()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("act", ["int8", "e4m3"])
def test_every_code_under_every_scale(sq, fmt, act):
    """Every byte as a code under every scale byte, one token: dS of its unpacked value, and half of it where it is normal."""
    O = I = 256
    q = torch.arange(256, dtype=torch.uint8, device="cuda").view(1, I)
    dY, codes = torch.ones((1, O), dtype=BF16, device="cuda"), _one_code_per_block(O, I)
    B = BLOCK[fmt]
    for byte in range(256):
        s = torch.full((1, I // 32), byte, dtype=torch.uint8, device="cuda")
        got = sq.sq_bwd_dscale_act8(fmt, act, q, s, dY, codes)
        x = sq.sq_act_unpack(act, q, s)
        assert _same(got, sq.sq_bwd_dscale(fmt, x, dY, codes)), byte
        x = step.act_unpack(act, q.cpu().numpy(), s.cpu().numpy())[0].reshape(-1, 32)
        normal = np.isfinite(x) & (np.abs(x) < 2.0 ** 127) & ((np.abs(x) >= 2.0 ** -125) | (x == 0))
        for b in np.flatnonzero(normal.all(1)):                # output o sees value o % 32 of the block
            want = np.zeros((32, 32 // B))
            want[np.arange(32), np.arange(32) // B] = 0.5 * x[b]
            have = got[:32, b * 32 // B:(b + 1) * 32 // B].double().cpu().numpy()
            assert np.array_equal(have, want), (byte, b)


# a tile cut at both edges, a split token sum, large tiles without a split, and a layer that goes through bf16 in memory
@pytest.mark.parametrize("T,O,I", [(70, 264, 288), (700, 264, 256), (333, 4096, 4096), (1025, 8192, 4096)])
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("act", ["int8", "e4m3"])
def test_blocks_of_the_largest_values(sq, fmt, act, T, O, I):
    """Blocks of values up to 3.2e38 (which E4M3 rounds below 2^128) among ordinary ones, dY small enough that every sum is finite."""
    X = inputs.device_bf16_normal(T, (T, I))
    big = torch.rand((T, I // 32, 1), generator=inputs.device_generator(T + 1), device="cuda") < 0.1
    X = torch.where(big, X.view(T, -1, 32).float() * 2.0 ** 126, X.view(T, -1, 32).float()).view(T, I)
    X = X.clamp(-3.2e38, 3.2e38).to(BF16).contiguous()
    q, s = sq.sq_act_pack(act, X)
    assert (s == (248 if act == "int8" else 246)).any()
    dY = (inputs.device_bf16_normal(T + 2, (T, O)).float() * 2.0 ** -60).to(BF16)
    codes = inputs.device_codes_uniform(T + 3, O, I)
    x = sq.sq_act_unpack(act, q, s)
    assert torch.isfinite(x).all()
    want = sq.sq_bwd_dscale(fmt, x, dY, codes)
    assert torch.isfinite(want).all()
    assert torch.equal(sq.sq_bwd_dscale_act8(fmt, act, q, s, dY, codes), want)


@pytest.mark.parametrize("act", ["int8", "e4m3"])
def test_the_largest_values_of_experts(sq, act):
    """The experts' form on the same blocks: each plane is its single product's."""
    T, O, I, counts = 300, 264, 288, [65, 0, 235]
    X = inputs.device_bf16_normal(4, (T, I))
    X[::7, 32:64] = (X[::7, 32:64].float() * 2.0 ** 126).clamp(-3.2e38, 3.2e38).to(BF16)
    q, s = sq.sq_act_pack(act, X)
    dY = (inputs.device_bf16_normal(5, (T, O)).float() * 2.0 ** -60).to(BF16)
    codes = inputs.device_codes_uniform(6, 3 * O, I).view(3, O, I // 2)
    at = np.concatenate([[0], np.cumsum(counts)])
    got = sq.sq_bwd_dscale_act8_batched("mx", act, q, s, None, torch.from_numpy(at.astype(np.int32)).cuda(), dY, codes)
    for e in range(3):
        a, b = at[e], at[e + 1]
        one = sq.sq_bwd_dscale_act8("mx", act, q[a:b].contiguous(), s[a:b].contiguous(), dY[a:b].contiguous(), codes[e])
        mag = sq.sq_bwd_dscale("mx", sq.sq_act_unpack(act, q[a:b].contiguous(), s[a:b].contiguous()).abs(), dY[a:b].abs().contiguous(),
                               (codes[e] & 0x77).contiguous())
        # the same exact products, fp32 sums in other orders
        assert torch.isfinite(one).all() and ((got[e] - one).abs() <= 2 * (counts[e] + 42) * 2.0 ** -23 * mag).all()
