"""Operators of a 4-bit student where offsets pass 32 bits: tables, gradients,
activations and experts of more than 2^31 elements or bytes, looked at where the
large offsets are."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import student
from paper_2609_04526_amd import inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    yield _sq
    torch.cuda.empty_cache()


def test_embedding_of_a_large_table(sq):
    V, H = 600011, 4096                                        # 2.46e9 elements
    ids = torch.tensor([0, V - 1, 5, V - 1, 600000, V], device="cuda")
    W = torch.zeros((V, H), dtype=BF16, device="cuda")
    for k, v in enumerate((0, 5, 600000, V - 1)):
        W[v] = k + 1
    out = sq.sq_embed_fwd("bf16", ids, W, factor=2.0)
    assert out.float().mean(1).tolist() == [2, 8, 4, 8, 6, 0] and out.float().std(1).max() == 0
    d = torch.arange(1, 7, device="cuda", dtype=torch.float32)[:, None].expand(6, H).contiguous()
    dW = sq.sq_embed_bwd(ids, d, V, out_dtype=BF16, dW=W)
    rows = {0: 1, V - 1: 6, 5: 3, 600000: 5}
    for v, want in rows.items():
        assert (dW[v] == want).all()
        dW[v] = 0
    # in parts: torch's own reductions over all of it would need a copy
    assert not any(part.any() for part in dW.split(50000))


@pytest.mark.parametrize("T", [3, 1500])
def test_gradient_of_more_units_than_a_launch_has(sq, T):
    V, H = (1 << 21) + 3, 8200                                 # 6.9e10 bytes: more than 2^32 of 16
    if torch.cuda.mem_get_info()[0] < V * H * 4 + (4 << 30):
        pytest.skip("needs 73 GB")
    ids = torch.full((T,), V - 2, device="cuda", dtype=torch.int32)
    ids[0] = 11
    dW = torch.ones((V, H), device="cuda")
    sq.sq_embed_bwd(ids, torch.ones((T, H), dtype=BF16, device="cuda"), V, dW=dW)
    assert (dW[11] == 1).all() and (dW[V - 2] == T - 1).all()
    dW[11] = dW[V - 2] = 0
    assert not any(part.any() for part in dW.split(50000))


def test_scales_of_a_large_table(sq):
    V, H = 1100003, 4096                                       # codes of 2.25e9 bytes
    codes = torch.full((V, H // 2), 0x22, dtype=torch.uint8, device="cuda")          # ones
    scales = torch.full((V, H // 32), 127, dtype=torch.uint8, device="cuda")
    scales[V - 1] = 129
    ids = torch.tensor([V - 1, 7, V - 1], device="cuda", dtype=torch.int32)
    out = sq.sq_embed_fwd("mx", ids, codes, scales=scales)
    assert (out[0] == 4).all() and (out[1] == 1).all() and (out[2] == 4).all()
    dS = sq.sq_embed_bwd_dscale("mx", ids, torch.ones((3, H), device="cuda"), codes)
    assert (dS[V - 1] == 64).all() and (dS[7] == 32).all()
    dS[V - 1] = dS[7] = 0
    assert not dS.any()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_activation_of_many_values(sq, fmt):
    T, I = 540001, 4096                                        # 2.2e9 values
    X = torch.zeros((T, I), dtype=BF16, device="cuda")
    last = inputs.bf16_normal(1, (3, I))
    X[-3:] = last.cuda()
    codes, scales = sq.sq_act4_pack(fmt, X, ws2=0.01)
    rc, rs = student.act4_pack(fmt, last.float().numpy(), 0.01)
    assert np.array_equal(codes[-3:].cpu().numpy(), rc) and np.array_equal(scales[-3:].cpu().numpy(), rs)
    Z = sq.sq_act4_unpack(fmt, codes, scales, ws2=0.01, X=X)
    want = torch.from_numpy(student.act4_values(fmt, rc, rs).astype(np.float32) * np.float32(0.01 if fmt == "nv" else 1)).to(BF16)
    assert torch.equal(Z[-3:].cpu(), want) and not Z[:-3].any()


@pytest.mark.parametrize("N", [40, 3000])
def test_experts_of_many_bytes(sq, N):
    E, O, I = 700, 1544, 4096                                  # codes of 2.2e9 bytes
    codes = torch.zeros((E, O, I // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((E, O, I // 32), 127, dtype=torch.uint8, device="cuda")
    w = inputs.codes_uniform(1, O, I)
    codes[E - 1] = torch.from_numpy(w).cuda()
    offsets = torch.full((E + 1,), N // 2, dtype=torch.int32, device="cuda")
    offsets[0], offsets[E] = 0, N
    xc = inputs.codes_uniform(2, N, I)
    xs = np.full((N, I // 32), 120, np.uint8)
    Y = sq.sq_fwd_act4_batched("mx", torch.from_numpy(xc).cuda(), torch.from_numpy(xs).cuda(), None, offsets, codes, scales)
    from oracle import linear
    ref = linear.dequant("mx", xc[N // 2:], xs[N // 2:]) @ linear.code_values(w).T
    assert not Y[:N // 2].any()
    # sums of multiples of 2^-9 below 2^15: exact in fp32
    assert np.array_equal(Y[N // 2:].double().cpu().numpy(), ref)


@pytest.mark.parametrize("out_dtype", [BF16, torch.float32])
def test_experts_of_many_rows_times_outputs(sq, out_dtype):
    """Rows and outputs of which a bf16 matrix takes more than 2 GiB, and an fp32 one more than 4."""
    E, N, O, I = 4, 131072 + 37, 8448, 32
    codes = torch.from_numpy(inputs.codes_uniform(3, E * O, I)).cuda().view(E, O, I // 2)
    scales = torch.full((E, O, 1), 127, dtype=torch.uint8, device="cuda")
    xc, xs = torch.from_numpy(inputs.codes_uniform(4, N, I)).cuda(), torch.full((N, 1), 120, dtype=torch.uint8, device="cuda")
    ends = [0, 30000, 30000, 100001, N - 20]
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    Y = torch.full((N, O), float("nan"), dtype=out_dtype, device="cuda")
    sq.sq_fwd_act4_batched("mx", xc, xs, None, offsets, codes, scales, Y=Y)
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    values = lambda c: table[torch.stack((c & 15, c >> 4), -1).long()].flatten(-2)
    for e in range(E):
        w = values(codes[e]).t().contiguous()
        for a in range(ends[e], ends[e + 1], 8192):
            b = min(a + 8192, ends[e + 1])
            # sums of multiples of 2^-9 below 2^11 at most: exact in fp32, and rounded once to bf16
            assert torch.equal(Y[a:b], (values(xc[a:b]) @ w * 2.0 ** -7).to(out_dtype))
    assert not Y[ends[-1]:].any()


@pytest.mark.parametrize("fmt,T", [("mx", 25600), ("mx", 26000), ("nv", 25500), ("nv", 25700)])
def test_values_of_about_the_caches_size(sq, fmt, T):
    """Values and codes of a little less and a little more than 256 MiB, which are stored in different ways."""
    I, n, ws2 = 4096, 100, 2.0 ** -9
    block = 32 if fmt == "mx" else 16
    assert (T * I * 2 + T * I // 2 + T * I // block > 256 << 20) == (T in (26000, 25700))
    xc, xs = student.act4_pack(fmt, inputs.bf16_normal(2, (n, I)).float().numpy(), ws2)
    codes, scales = (torch.from_numpy(v).cuda().repeat(T // n, 1) for v in (xc, xs))
    X = torch.full((T, I), float("nan"), dtype=BF16, device="cuda")
    sq.sq_act4_unpack(fmt, codes, scales, ws2=ws2, X=X)
    want = torch.from_numpy(student.act4_values(fmt, xc, xs).astype(np.float32) * np.float32(ws2 if fmt == "nv" else 1)).to(BF16)
    assert (X.view(T // n, n, I) == want.cuda()).all()


@pytest.mark.parametrize("head,T", [("bf16", 16384), ("bf16", 16385), ("mx", 25801), ("mx", 25950), ("nv", 25500), ("nv", 25700)])
def test_lookup_of_about_the_caches_size(sq, head, T):
    """Rows read and written of 256 MiB, or a little less, and of a little more, which are stored in different ways; each
    a row of a small call on the same table."""
    V, H = 40000, 4096
    gen = inputs.device_generator(T)
    scales = None
    if head == "bf16":
        W = torch.randn((V, H), generator=gen, device="cuda").to(BF16)
    else:
        W = torch.randint(0, 256, (V, H // 2), generator=gen, device="cuda", dtype=torch.uint8)
        scales = torch.randint(100, 126, (V, H // (32 if head == "mx" else 16)), generator=gen, device="cuda", dtype=torch.uint8)
    row = 2 * H if head == "bf16" else H // 2 + scales.shape[1]
    assert (T * (2 * H + row) > 256 << 20) == (T in (16385, 25950, 25700))
    ids = torch.randint(-2, V, (T,), generator=gen, device="cuda")
    more = dict(scales=scales, ws2=0.01, factor=1.5)
    out = torch.full((T, H), float("nan"), dtype=BF16, device="cuda")
    sq.sq_embed_fwd(head, ids, W, out=out, **more)
    for a in range(0, T, 4000):
        part = sq.sq_embed_fwd(head, ids[a:a + 4000].contiguous(), W, **more)
        assert torch.equal(out[a:a + 4000], part)
    assert torch.isfinite(out).all() and not out[ids < 0].any() and out[ids >= 0].any(1).all()


@pytest.mark.parametrize("T", [(1 << 30) - 5, 1 << 30])
def test_embedding_of_the_most_tokens(sq, T):
    """As many tokens as the entry points take: two ids in turn, one of them outside the table, and then one id's run
    of a third of them.

    A run's ones are summed in fp32: those before its first whole chunk of 8192 one by one (exact), then the chunks' sums,
    then those past its last one by one.  Up to 2^24 all of it is exact.  From there on a chunk's 8192 is a multiple of the
    sum's step u (at most 32 below 2^29), so the sum is rounded only where the step doubles, by u / 2 at most, 31 in all
    for u = 2 .. 32; and a one added to a multiple of u is off by 1 at most, 8191 of them by 8191."""
    V, I = 700, 8
    if torch.cuda.mem_get_info()[0] < T * 80:
        pytest.skip("needs 80 GB")
    ids = torch.full((T,), 699, dtype=torch.int32, device="cuda")
    n = T // 3 * 2
    ids[:n:2], ids[1:n:2] = 5, -1
    ids[T - 1] = 0
    W = inputs.bf16_normal(1, (V, I)).cuda()
    out = sq.sq_embed_fwd("bf16", ids, W)
    for a in (0, 1 << 22, 1 << 29, T - (1 << 20)):
        part = ids[a:a + (1 << 20)]
        live = part >= 0
        assert torch.equal(out[a:a + (1 << 20)], torch.where(live[:, None], W[torch.where(live, part, 0)], torch.zeros((), dtype=BF16, device="cuda")))
    out.fill_(1.0)
    dW = sq.sq_embed_bwd(ids, out, V)
    want = torch.zeros(V, dtype=torch.float64, device="cuda")
    want[5], want[699], want[0] = (n + 1) // 2, T - n - 1, 1
    off = (dW.double() - want[:, None]).abs()
    assert (off <= torch.where(want > 1 << 24, 8191.0 + 31.0, 0.0)[:, None]).all()
