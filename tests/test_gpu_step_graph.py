"""The operators of a training step inside a HIP graph: captured once with
buffers of their own, replayed on new inputs between eager work, every replay
equal to the eager calls bit for bit."""

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


def _bytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


# few and compact rows, a sort of one launch and of three, heads of both kinds
@pytest.mark.parametrize("T,K,E,H,F,V,head", [(40, 2, 6, 128, 96, 1003, "mx"), (400, 3, 9, 96, 256, 515, "mx"),
                                              (8200, 8, 16, 64, 32, 300, "bf16"), (9, 1, 4, 1088, 64, 260, "bf16")])
def test_replays_equal_eager_calls(sq, T, K, E, H, F, V, head):
    dev = "cuda"
    ids = torch.zeros((T, K), dtype=torch.int64, device=dev)
    X, dZ = (torch.zeros((T, H), dtype=BF16, device=dev) for _ in range(2))
    dU = torch.zeros((T * K, F), dtype=BF16, device=dev)
    w = torch.zeros((T, K), device=dev)
    y = torch.zeros(T, dtype=torch.int64, device=dev)
    dloss = torch.zeros(T, device=dev)
    codes = inputs.device_codes_uniform(1, E * F, H).view(E, F, H // 2)
    if head == "bf16":
        W, ws = inputs.device_bf16_normal(2, (V, H)) / 8, None
    else:
        W = inputs.device_codes_uniform(2, V, H)
        ws = torch.from_numpy(inputs.e8m0_uniform_exponents(3, V, H // 32, -5, -3)).cuda()

    def fill(seed):
        g = inputs.rng(seed)
        ids.copy_(torch.from_numpy(g.integers(-1, E, (T, K))))
        y.copy_(torch.from_numpy(g.integers(-1, V, T)))
        for i, t in enumerate((X, dZ, dU, w, dloss)):
            t.copy_(inputs.bf16_normal(seed + 10 + i, tuple(t.shape)))

    i32 = dict(dtype=torch.int32, device=dev)
    out = dict(offsets=torch.empty(E + 1, **i32), token=torch.empty(T * K, **i32), slot=torch.empty((T, K), **i32),
               Xs=torch.empty((T * K, H), dtype=BF16, device=dev), Z=torch.empty((T, H), dtype=BF16, device=dev),
               dYs=torch.empty((T * K, H), dtype=BF16, device=dev), dw=torch.empty((T, K), device=dev),
               q=torch.empty((T, H), dtype=torch.uint8, device=dev), s=torch.empty((T, H // 32), dtype=torch.uint8, device=dev),
               dS=torch.empty((E, F, H // 32), device=dev), dS1=torch.empty((F, H // 32), device=dev),
               loss=torch.empty(T, device=dev), lse=torch.empty(T, device=dev), dX=torch.empty((T, H), dtype=BF16, device=dev))
    h = sq.HEADS[head]
    spaces = [_bytes(n) for n in (sq.sq_moe_sort_workspace(T, K, E), sq.sq_bwd_dscale_act8_batched_workspace(E, T, H),
                                  sq.sq_bwd_dscale_act8_workspace(0, T, F, H), sq.sq_ce_fwd_workspace(h, T, V, H),
                                  sq.sq_ce_bwd_workspace(h, T, V, H))]

    def run(o):
        sq.sq_moe_sort(ids, E, o["offsets"], o["token"], o["slot"], spaces[0])
        sq.sq_moe_gather(X, o["slot"], o["offsets"], o["Xs"])
        sq.sq_moe_combine(o["Xs"], o["slot"], o["offsets"], w, out=o["Z"])
        sq.sq_moe_combine_bwd(dZ, o["Xs"], o["slot"], o["offsets"], w, dYs=o["dYs"], dweights=o["dw"])
        sq.sq_act_pack("int8", X, o["q"], o["s"])
        sq.sq_bwd_dscale_act8_batched("mx", "int8", o["q"], o["s"], o["token"], o["offsets"], dU, codes, o["dS"], spaces[1])
        sq.sq_bwd_dscale_act8("mx", "int8", o["q"], o["s"], dU[:T], codes[0], o["dS1"], spaces[2])
        sq.sq_ce_fwd(head, X, W, y, scales=ws, loss=o["loss"], lse=o["lse"], workspace=spaces[3])
        sq.sq_ce_bwd(head, X, W, y, o["lse"], dloss, scales=ws, dX=o["dX"], workspace=spaces[4])

    fill(100)
    eager = {k: torch.empty_like(v) for k, v in out.items()}
    run(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        run(out)
    for seed in (100, 200, 300, 400):
        fill(seed)
        for v in out.values():
            v.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        run(eager)
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], eager[k]), (k, seed)
