"""A 4-bit student's operators together: one training step (token ids through a
4-bit embedding, a routed expert layer on 4-bit activations, the distillation loss
of a 4-bit head, and back to the scales of the head's input, of the experts and of
the embedding) against the oracle's, and all of them inside a HIP graph, replayed
on new inputs between eager work, every replay equal to the eager calls bit for
bit."""

import numpy as np
import pytest
import torch

from conftest import ensure_library, gpu_ready
from oracle import linear, step, student
from paper_2609_04526_amd import inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_ready(), reason="needs a GPU")]

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def sq():
    ensure_library()
    from paper_2609_04526_amd import sq as _sq
    return _sq


def _near(got, ref, tol):
    """Normwise: each tensor between two operators is bf16, so an error of a few of its half steps (2^-9 in the mean) is
    what a chain of them leaves."""
    got = got.double().cpu().numpy()
    assert np.linalg.norm(got - ref) <= tol * np.linalg.norm(ref), np.linalg.norm(got - ref) / np.linalg.norm(ref)


@pytest.mark.parametrize("T,K,E,H,F,V,N", [(37, 2, 6, 128, 96, 1003, 8), (300, 2, 5, 256, 160, 700, 20)])
def test_a_training_step(sq, T, K, E, H, F, V, N):
    g = inputs.rng(T)
    table_c, head_c = inputs.codes_uniform(1, V, H), inputs.codes_uniform(2, V, H)
    table_s = inputs.e8m0_uniform_exponents(3, V, H // 32, -6, -3)
    head_s = inputs.e8m0_uniform_exponents(4, V, H // 32, -5, -4)
    up_c, up_s = inputs.codes_uniform(5, E * F, H).reshape(E, F, -1), inputs.e8m0_uniform_exponents(6, E * F, H // 32, -6, -4).reshape(E, F, -1)
    tokens = np.where(g.random(T) < 0.1, -1, (V * g.random(T) ** 2).astype(np.int64))
    experts = g.random((T, E)).argsort(1)[:, :K].copy()
    experts[g.random((T, K)) < 0.05] = -1
    ids, z = (V * g.random((T, N))).astype(np.int64), (2 * g.standard_normal((T, N))).astype(np.float32)
    ids[g.random(T) < 0.2] = -1
    dloss = (g.random(T) / T).astype(np.float32)
    dY = inputs.bf16_normal(7, (T * K, F))
    d = [torch.from_numpy(a).cuda() for a in (table_c, table_s, head_c, head_s, up_c, up_s, tokens, experts, ids, z, dloss)]
    tc, ts, hc, hs, uc, us, tok, exp, idd, zd, dl = d

    # ids -> rows -> experts on 4-bit rows; the rows' own loss through the head
    X = sq.sq_embed_fwd("mx", tok, tc, scales=ts, factor=2.0)
    xc, xs = sq.sq_act4_pack("mx", X)
    offsets, token, slot = sq.sq_moe_sort(exp, E)
    Y = sq.sq_fwd_act4_batched("mx", xc, xs, token, offsets, uc, us)
    loss, lse, picked = sq.sq_distill_fwd("mx", X, hc, idd, zd, scales=hs, temperature=2.0)
    dX = sq.sq_distill_bwd("mx", X, hc, idd, zd, lse, picked, dl, scales=hs, temperature=2.0, out_dtype=BF16)
    # the experts' scales from the kept rows, and the embedding's from what reaches it
    Xs = sq.sq_moe_gather(sq.sq_act4_unpack("mx", xc, xs), slot, offsets)
    dYd, o = dY.cuda(), offsets.tolist()
    dS = torch.stack([sq.sq_bwd_dscale("mx", Xs[a:b], dYd[a:b], uc[e]) for e, (a, b) in enumerate(zip(o[:-1], o[1:]))])
    dT = sq.sq_embed_bwd_dscale("mx", tok, dX, tc, factor=2.0)

    w = linear.dequant("mx", table_c, table_s)
    x = torch.from_numpy(student.embed_fwd(tokens, w, 2.0)).float().to(BF16)
    assert torch.equal(X.cpu(), x)
    rc, rs = student.act4_pack("mx", x.float().numpy())
    assert np.array_equal(xc.cpu().numpy(), rc) and np.array_equal(xs.cpu().numpy(), rs)
    kept = student.act4_values("mx", rc, rs)
    r_off, r_tok, r_slot = step.moe_sort(experts, E)
    uw = linear.dequant("mx", up_c.reshape(E * F, -1), up_s.reshape(E * F, -1)).reshape(E, F, H)
    _near(Y, student.experts(kept, r_tok, r_off, uw), 1e-6)
    hw = linear.dequant("mx", head_c, head_s)
    r_loss, _, _ = student.distill_fwd(x.double().numpy(), hw, ids, z.astype(np.float64), 2.0)
    _near(loss, r_loss, 1e-5)
    r_dX = student.distill_bwd(x.double().numpy(), hw, ids, z.astype(np.float64), 2.0, dloss)
    _near(dX, r_dX, 4e-3)
    ref = [linear.backward_dscale("mx", kept[r_tok[a:b]], dY[a:b].double().numpy(), up_c[e]) for e, (a, b) in enumerate(zip(o[:-1], o[1:]))]
    _near(dS, np.stack(ref), 1e-5)
    _near(dT, student.embed_bwd_dscale("mx", tokens, dX.double().cpu().numpy(), table_c, 2.0), 1e-5)


def _bytes(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


# few and compact rows; the few rows' kernel and tiles, with scales that are not whole words; heads of all kinds
@pytest.mark.parametrize("T,K,E,H,F,V,N,head", [(20, 2, 4, 96, 40, 1003, 8, "mx"), (400, 3, 9, 160, 264, 515, 40, "nv"),
                                                (2100, 2, 8, 512, 264, 300, 20, "bf16"), (300, 1, 3, 512, 136, 900, 256, "mx")])
def test_replays_equal_eager_calls(sq, T, K, E, H, F, V, N, head):
    dev = "cuda"
    fmt = "nv" if head == "nv" else "mx"
    X, dO = (torch.zeros((T, H), dtype=BF16, device=dev) for _ in range(2))
    tokens = torch.zeros(T, dtype=torch.int32, device=dev)
    experts = torch.zeros((T, K), dtype=torch.int64, device=dev)
    ids, z = torch.zeros((T, N), dtype=torch.int64, device=dev), torch.zeros((T, N), device=dev)
    dloss = torch.zeros(T, device=dev)
    layer = inputs.device_codes_uniform(1, F, H), torch.randint(50, 120, (F, H // sq.BLOCK[sq.FORMATS[fmt]]), dtype=torch.uint8, device=dev)
    up = inputs.device_codes_uniform(2, E * F, H).view(E, F, -1), torch.randint(115, 125, (E, F, H // 32), dtype=torch.uint8, device=dev)
    if head == "bf16":
        W, ws = inputs.device_bf16_normal(3, (V, H)) / 8, None
    else:
        W = inputs.device_codes_uniform(3, V, H)
        ws = torch.randint(*((118, 122) if head == "mx" else (40, 70)), (V, H // sq.BLOCK[sq.FORMATS[head]]), dtype=torch.uint8, device=dev)

    def fill(seed):
        g = inputs.rng(seed)
        tokens.copy_(torch.from_numpy(g.integers(-1, V, T)))
        experts.copy_(torch.from_numpy(g.integers(-1, E, (T, K))))
        ids.copy_(torch.from_numpy(np.where(g.random((T, 1)) < 0.2, -1, g.integers(-1, V, (T, N)))))
        for i, t in enumerate((X, dO, z, dloss)):
            t.copy_(inputs.bf16_normal(seed + 10 + i, tuple(t.shape)))

    G = H // sq.BLOCK[sq.FORMATS[fmt]]
    u8, i32, f32 = (dict(dtype=t, device=dev) for t in (torch.uint8, torch.int32, F32))
    out = dict(xc=torch.empty((T, H // 2), **u8), xs=torch.empty((T, G), **u8), X4=torch.empty((T, H), dtype=BF16, device=dev),
               Y=torch.empty((T, F), **f32), mc=torch.empty((T, H // 2), **u8), ms=torch.empty((T, H // 32), **u8),
               offsets=torch.empty(E + 1, **i32), token=torch.empty(T * K, **i32), slot=torch.empty((T, K), **i32),
               Ye=torch.empty((T * K, F), dtype=BF16, device=dev), loss=torch.empty(T, **f32), lse=torch.empty(T, **f32),
               picked=torch.empty((T, N), **f32), dX=torch.empty((T, H), dtype=BF16, device=dev),
               out=torch.empty((T, H), dtype=BF16, device=dev),
               grad=torch.empty((V, H) if head == "bf16" else (V, H // sq.BLOCK[sq.FORMATS[head]]), **f32))
    spaces = [_bytes(n) for n in (sq.sq_moe_sort_workspace(T, K, E), sq.sq_fwd_act4_workspace(fmt, T, F, H),
                                  sq.sq_fwd_act4_batched_workspace("mx", E, T, T * K, F, H), sq.sq_distill_fwd_workspace(head, T, V, H),
                                  sq.sq_distill_bwd_workspace(head, T, V, H), sq.sq_embed_bwd_workspace(T, V, H))]

    def run(o, w):
        sq.sq_act4_pack(fmt, X, ws2=0.01, codes=o["xc"], scales=o["xs"])
        sq.sq_act4_unpack(fmt, o["xc"], o["xs"], ws2=0.01, X=o["X4"])
        sq.sq_fwd_act4(fmt, o["xc"], o["xs"], *layer, x_ws2=0.01, ws2=0.01, Y=o["Y"], workspace=w[1])
        sq.sq_act4_pack("mx", X, codes=o["mc"], scales=o["ms"])
        sq.sq_moe_sort(experts, E, offsets=o["offsets"], token=o["token"], slot=o["slot"], workspace=w[0])
        sq.sq_fwd_act4_batched("mx", o["mc"], o["ms"], o["token"], o["offsets"], *up, Y=o["Ye"], workspace=w[2])
        more = dict(scales=ws, ws2=0.01, temperature=1.5)
        sq.sq_distill_fwd(head, X, W, ids, z, loss=o["loss"], lse=o["lse"], picked=o["picked"], workspace=w[3], **more)
        sq.sq_distill_bwd(head, X, W, ids, z, o["lse"], o["picked"], dloss, dX=o["dX"], workspace=w[4], **more)
        sq.sq_embed_fwd(head, tokens, W, scales=ws, ws2=0.01, factor=3.0, out=o["out"])
        if head == "bf16":
            sq.sq_embed_bwd(tokens, dO, V, factor=3.0, dW=o["grad"], workspace=w[5])
        else:
            sq.sq_embed_bwd_dscale(head, tokens, dO, W, factor=3.0, dS=o["grad"], workspace=w[5])

    fill(1)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        run(out, spaces)                                       # the first launches outside the capture
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(out, spaces)
    for seed in (100, 200, 300):
        fill(seed)
        eager = {k: torch.empty_like(v) for k, v in out.items()}
        run(eager, [s.clone() for s in spaces])
        for t in out.values():
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(torch.nan_to_num(out[k].float(), nan=77.0), torch.nan_to_num(eager[k].float(), nan=77.0)), k


def test_two_streams_at_once(sq):
    """Calls on two streams with workspaces of their own give what they give alone."""
    T, H, V, N = 300, 512, 3000, 16
    W = inputs.device_bf16_normal(1, (V, H)) / 16
    codes = inputs.device_codes_uniform(2, 264, H)
    scales = torch.randint(115, 125, (264, H // 32), dtype=torch.uint8, device="cuda")
    g = inputs.rng(3)
    X = [inputs.device_bf16_normal(4 + i, (T, H)) for i in range(2)]
    ids, z = torch.from_numpy(g.integers(0, V, (T, N))).cuda(), torch.from_numpy(g.standard_normal((T, N))).float().cuda()
    tokens, dl = ids[:, 0].contiguous(), torch.ones(T, device="cuda")

    def run(i):
        loss, lse, picked = sq.sq_distill_fwd("bf16", X[i], W, ids, z)
        return (loss, sq.sq_distill_bwd("bf16", X[i], W, ids, z, lse, picked, dl), sq.sq_embed_bwd(tokens, X[i], V),
                sq.sq_fwd_act4("mx", *sq.sq_act4_pack("mx", X[i]), codes, scales))

    alone = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                both[i] = run(i)
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(alone[i], both[i]))
