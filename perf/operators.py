"""Workloads of what a training step runs around the frozen-code products, each
in a plain form (elementary torch operations in 32 bits) and through the
library's entry points.

  dispatch  routed tokens sorted by expert, and their rows laid out expert by
            expert for the grouped products
  combine   the experts' rows back to tokens with the router's weights, and the
            gradients of the rows, of the weights and of the dispatched tokens
  keep      an activation kept in 8 bits between the forward and the backward
            pass, and read back
  dscale8   the block-scale gradient of one linear from its input kept in 8
            bits (E = 0), or of E stacked experts that pick their rows of the
            layer's tokens (E > 0)
  loss      softmax cross entropy of a language-model head (bf16, or in the
            MXFP4 or NVFP4 storage) over its whole vocabulary, with the
            gradient of the head's input

`own` selects the side: False runs the plain forms, True the library.  Inputs
are synthetic and drawn on the GPU from the seed.
"""

import math

import torch

own = False

BLOCK = {"mx": 32, "nv": 16}
ACT_BLOCK = 32
WS2 = 1.0 / 448.0
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
LINEARS = [(4096, 4096), (1024, 4096), (14336, 4096), (4096, 14336)]     # of the dense model of bench.py
EXPERTS = [(768, 2048), (2048, 768), (1536, 2048)]                       # of its MoE layer: gate or up, down, gate and up


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one token of a serving loop through a 128-expert layer: latency of sort and layout
        dict(name="dispatch t1", kind="dispatch", T=1, K=8, E=128, H=2048, dtype="bf16", ids="i64", drop=0.0),
        # a training step's tokens through the same layer, some of them dropped by a capacity limit
        dict(name="dispatch t4096", kind="dispatch", T=4096, K=8, E=128, H=2048, dtype="bf16", ids="i64", drop=0.05),
        # a few experts' fp32 rows on a ragged batch with an odd width
        dict(name="combine t333", kind="combine", T=333, K=2, E=8, H=4104, dtype="f32", drop=0.1),
        # a long packed batch back from 8 of 128 experts
        dict(name="combine t16384", kind="combine", T=16384, K=8, E=128, H=2048, dtype="bf16", drop=0.0),
        # the small layer of the tests: launch latency
        dict(name="keep int8 t64", kind="keep", act="int8", T=64, I=512),
        # the widest activation of a dense model's layer at 8192 tokens
        dict(name="keep e4m3 t8192", kind="keep", act="e4m3", T=8192, I=14336),
        # the small layer of the tests
        dict(name="dscale8 mx 256x512 t64", kind="dscale8", fmt="mx", act="int8", E=0, T=64, K=1, O=256, I=512),
        # an attention projection at 4 x 1024 tokens: bench.py's step
        dict(name="dscale8 nv 4096x4096 t4096", kind="dscale8", fmt="nv", act="e4m3", E=0, T=4096, K=1, O=4096, I=4096),
        # the MoE layer of bench.py, its experts' rows picked from 4096 kept tokens
        dict(name="dscale8 mx 128x768x2048 t4096", kind="dscale8", fmt="mx", act="int8", E=128, T=4096, K=8, O=768,
             I=2048),
        # the head of a small test model on a few tokens: latency
        dict(name="loss bf16 1000x512 t5", kind="loss", head="bf16", T=5, V=1000, H=512, ignored=0.0),
        # a fine-tuning batch whose prompt tokens are masked, odd vocabulary, head in the layer's storage
        dict(name="loss mx 50001x4096 t1999", kind="loss", head="mx", T=1999, V=50001, H=4096, ignored=0.4),
        # a full training batch over a large vocabulary: the largest call
        dict(name="loss bf16 131072x4096 t4096", kind="loss", head="bf16", T=4096, V=131072, H=4096, ignored=0.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    kind = rng.choice(["dispatch", "combine", "keep", "dscale8", "dscale8", "loss", "loss"])
    if kind in ("dispatch", "combine"):
        E = _log_int(rng, 4, 256)
        c = dict(kind=kind, T=_log_int(rng, 1, 16384), K=rng.randint(1, min(8, E)), E=E, H=8 * _log_int(rng, 32, 1024),
                 dtype=rng.choice(["bf16", "bf16", "f32"]), drop=rng.choice([0.0, 0.0, 0.02, 0.3]))
        if kind == "dispatch":
            c["ids"] = rng.choice(["i64", "i32"])
        while c["T"] * c["K"] * c["H"] > 16384 * 8 * 2048:
            c["T"] = c["T"] * 2 // 3
        return c
    act = rng.choice(["int8", "e4m3"])
    if kind == "keep":
        return dict(kind=kind, act=act, T=_log_int(rng, 1, 16384), I=32 * _log_int(rng, 8, 448))
    if kind == "dscale8":
        fmt = rng.choice(["mx", "nv"])
        if rng.random() < 0.4:
            O, I = rng.choice(EXPERTS)
            return dict(kind=kind, fmt=fmt, act=act, E=rng.choice([8, 32, 64, 128]), T=_log_int(rng, 16, 4096),
                        K=rng.choice([1, 2, 4, 8]), O=O, I=I)
        O, I = rng.choice(LINEARS) if rng.random() < 0.5 else (8 * _log_int(rng, 32, 1792), 32 * _log_int(rng, 16, 448))
        return dict(kind=kind, fmt=fmt, act=act, E=0, T=_log_int(rng, 1, 8192), K=1, O=O, I=I)
    head = rng.choice(["bf16", "bf16", "mx", "nv"])
    c = dict(kind=kind, head=head, T=_log_int(rng, 1, 8192), V=_log_int(rng, 1000, 160000),
             H=32 * _log_int(rng, 16, 256), ignored=rng.choice([0.0, 0.1, 0.5]))
    while c["T"] * c["V"] * c["H"] > 4096 * 131072 * 4096:
        c["T"] = c["T"] * 2 // 3
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1009 + k) % (1 << 62))
    return g


def _normal(seed, k, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=_gen(seed, k), device="cuda").to(dtype)


def _activation(seed, k, T, I):
    """Activations with uneven channels, a few of them far larger than the rest."""
    g = _gen(seed, k)
    chan = torch.exp(0.5 * torch.randn(I, generator=g, device="cuda"))
    chan = torch.where(torch.rand(I, generator=g, device="cuda") < 0.005, 20.0 * chan, chan)
    return (torch.randn((T, I), generator=g, device="cuda") * chan).to(torch.bfloat16)


def _route(case, seed):
    """Top-k experts of uneven router scores, their weights, and the dropped pairs marked -1."""
    T, K, E = case["T"], case["K"], case["E"]
    g = _gen(seed, 11)
    score = torch.randn((T, E), generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    top, ids = torch.topk(score, K, dim=1)
    drop = torch.rand((T, K), generator=g, device="cuda") < case.get("drop", 0.0)
    return torch.where(drop, torch.full_like(ids, -1), ids), torch.softmax(top, 1)


def _codes(seed, k, shape):
    return torch.randint(0, 256, shape, generator=_gen(seed, k), device="cuda", dtype=torch.uint8)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    kind, T = case["kind"], case["T"]
    s = dict(case=case)
    if kind == "dispatch":
        ids, _ = _route(case, seed)
        s["ids"] = ids if case["ids"] == "i64" else ids.to(torch.int32)
        s["X"] = _normal(seed, 1, (T, case["H"]), _dtype(case))
    elif kind == "combine":
        N = T * case["K"]
        ids, s["w"] = _route(case, seed)
        s["offsets"], _, s["slot"] = _sort(ids, case["E"])
        s["Ys"] = _normal(seed, 1, (N, case["H"]), _dtype(case))
        s["dOut"] = _normal(seed, 2, (T, case["H"]), _dtype(case))
        s["dXs"] = _normal(seed, 3, (N, case["H"]), _dtype(case))
    elif kind == "keep":
        s["X"] = _activation(seed, 1, T, case["I"])
    elif kind == "dscale8":
        E, O, I = case["E"], case["O"], case["I"]
        s["kept"], s["kept_scales"] = _keep(case["act"], _activation(seed, 1, T, I))
        s["dY"] = _normal(seed, 2, (T * case["K"], O))
        s["codes"] = _codes(seed, 3, (E, O, I // 2) if E else (O, I // 2))
        if E:
            s["offsets"], s["token"], _ = _sort(_route(case, seed)[0], E)
    else:
        V, H, head = case["V"], case["H"], case["head"]
        if head == "bf16":
            s["W"] = (torch.randn((V, H), generator=_gen(seed, 1), device="cuda") / math.sqrt(H)).to(torch.bfloat16)
        else:
            s["W"] = _codes(seed, 1, (V, H // 2))
            g = _gen(seed, 2)
            z = torch.randn((V, H // BLOCK[head]), generator=g, device="cuda")
            if head == "mx":
                s["scales"] = (torch.round(z - 7.0).clamp_(-127, 127) + 127).to(torch.uint8)
            else:
                s["scales"] = (z.abs() * (448.0 * 0.5 / math.sqrt(H))).to(torch.float8_e4m3fn).view(torch.uint8)
        g = _gen(seed, 4)
        y = torch.randint(0, V, (T,), generator=g, device="cuda")
        # hidden states that lean towards their targets, some of them far: probabilities from 1/V to nearly 1
        lean = _weight(dict(s, W=s["W"][y], scales=s["scales"][y] if "scales" in s else None), torch.float32)
        lean = lean / lean.norm(dim=1, keepdim=True)
        far = 12.0 * torch.rand((T, 1), generator=g, device="cuda")
        s["X"] = (torch.randn((T, H), generator=g, device="cuda") + far * lean).to(torch.bfloat16)
        s["y"] = torch.where(torch.rand(T, generator=g, device="cuda") < case["ignored"], torch.full_like(y, -100), y)
        s["dloss"] = torch.where(s["y"] < 0, 0.0, 1.0 / torch.clamp((s["y"] >= 0).sum(), min=1).float())
        s["dloss"] = s["dloss"] * (0.5 + torch.rand(T, generator=g, device="cuda"))      # per-token loss weights
    return s


# ---------------------------------------------------------------- plain forms
def _sort(ids, E):
    """offsets [E + 1], token [N] and slot [T, K]: the pairs in expert order, stable, dropped ones last."""
    K = ids.shape[1]
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, torch.full_like(flat, E))
    order = torch.argsort(key, stable=True)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(order.numel(), device=ids.device)
    count = torch.bincount(key, minlength=E + 1)[:E]
    offsets = torch.cat((torch.zeros(1, dtype=torch.long, device=ids.device), torch.cumsum(count, 0)))
    return offsets.to(torch.int32), (order // K).to(torch.int32), slot.view(ids.shape).to(torch.int32)


def _gather(X, token, offsets):
    live = torch.arange(token.numel(), device=X.device) < offsets[-1]
    return torch.where(live[:, None], X[token.long()], torch.zeros((), dtype=X.dtype, device=X.device))


def _combine(Ys, slot, offsets, w=None):
    live = (slot < offsets[-1]).float()
    rows = Ys[slot.reshape(-1).long()].float().view(slot.shape + Ys.shape[1:])
    rows = torch.where(live[..., None] > 0, rows, torch.zeros((), device=Ys.device))
    return (rows if w is None else rows * w[..., None]).sum(1).to(Ys.dtype)


def _combine_grad(dOut, Ys, slot, offsets, w):
    live = slot < offsets[-1]
    d = dOut.float()
    at = slot.reshape(-1).long()
    rows = torch.where(live[..., None], Ys[at].float().view(slot.shape + Ys.shape[1:]), torch.zeros((), device=Ys.device))
    dw = (rows * d[:, None]).sum(-1)
    dYs = torch.empty_like(Ys)
    dYs[at] = torch.where(live, w, torch.zeros_like(w))[..., None].mul(d[:, None]).to(Ys.dtype).view(-1, Ys.shape[1])
    return dYs, dw


def _keep(act, X):
    """8-bit values and E8M0 scale bytes of each 32 columns."""
    T, I = X.shape
    x = X.float().view(T, I // ACT_BLOCK, ACT_BLOCK)
    amax = x.abs().amax(-1)
    bad = ~torch.isfinite(x).all(-1)
    m, e = torch.frexp(torch.where(bad, torch.ones_like(amax), amax))
    k = e - 7 if act == "int8" else e - 9 + (m > 0.875).int()
    k = torch.where(amax == 0, torch.full_like(k, -126), k).clamp(-126, 127)
    q = torch.ldexp(torch.where(bad[..., None], torch.zeros_like(x), x), -k[..., None])
    if act == "int8":
        q = q.round().clamp(-127, 127).to(torch.int8)
    else:
        q = q.to(torch.float8_e4m3fn)
    return q.view(torch.uint8).view(T, I), torch.where(bad, torch.full_like(k, 255), k + 127).to(torch.uint8)


def _kept_values(act, q, scales, dtype=torch.float32):
    T, I = q.shape
    v = q.view(torch.int8 if act == "int8" else torch.float8_e4m3fn).to(dtype).view(T, I // ACT_BLOCK, ACT_BLOCK)
    f = torch.where(scales == 255, torch.full((), float("nan"), device=q.device, dtype=dtype),
                    torch.exp2(scales.to(dtype) - 127.0))
    return (v * f[..., None]).view(T, I)


def _code_values(codes, dtype):
    table = torch.tensor(E2M1 + [-v for v in E2M1], dtype=dtype, device=codes.device)
    nib = torch.stack((codes & 15, codes >> 4), dim=-1)
    return table[nib.long()].view(codes.shape[:-1] + (2 * codes.shape[-1],))


def _weight(s, dtype):
    """The head's weight [V, H] as plain values."""
    head = s["case"]["head"]
    if head == "bf16":
        return s["W"].to(dtype)
    w = _code_values(s["W"], dtype)
    if head == "mx":
        eff = torch.exp2(s["scales"].to(dtype) - 127.0)
    else:
        eff = s["scales"].view(torch.float8_e4m3fn).to(dtype) * torch.tensor(WS2, dtype=torch.float32).to(dtype)
    return (w.view(w.shape[0], -1, BLOCK[head]) * eff[..., None]).view(w.shape)


def _padded(rows, offsets, longest):
    """Row numbers [E, longest] of the experts' ranges and which of them are inside."""
    at = offsets[:-1, None].long() + torch.arange(longest, device=rows.device)
    inside = at < offsets[1:, None]
    return torch.where(inside, at, torch.zeros_like(at)), inside


def _dscale8(s, dtype=torch.float32):
    case = s["case"]
    x = _kept_values(case["act"], s["kept"], s["kept_scales"], dtype)
    dy = s["dY"].to(dtype)
    if case["E"]:
        longest = int((s["offsets"][1:] - s["offsets"][:-1]).max())
        at, inside = _padded(s["token"], s["offsets"], max(longest, 1))
        x = torch.where(inside[..., None], x[s["token"].long()[at]], torch.zeros((), dtype=dtype, device=x.device))
        dy = torch.where(inside[..., None], dy[at], torch.zeros((), dtype=dtype, device=x.device))
    dw = dy.transpose(-1, -2).contiguous() @ x
    dw = dw * _code_values(s["codes"], dtype)
    return dw.view(dw.shape[:-1] + (dw.shape[-1] // BLOCK[case["fmt"]], -1)).sum(-1)


def _loss(s):
    x, w = s["X"].float(), _weight(s, torch.float32)
    valid = s["y"] >= 0
    at = torch.where(valid, s["y"], torch.zeros_like(s["y"]))[:, None]
    logits = x @ w.t()
    top = logits.amax(1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    loss = lse - logits.gather(1, at)[:, 0]
    p = p / total
    p.scatter_add_(1, at, torch.full_like(top, -1.0))
    p = p * torch.where(valid, s["dloss"], torch.zeros_like(s["dloss"]))[:, None]
    zero = torch.zeros_like(lse)
    return dict(loss=torch.where(valid, loss, zero), lse=torch.where(valid, lse, zero), dX=(p @ w).to(torch.bfloat16))


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "dispatch":
        offsets, token, slot = _sort(s["ids"], case["E"])
        return dict(offsets=offsets, token=token, slot=slot, Xs=_gather(s["X"], token, offsets))
    if kind == "combine":
        dYs, dw = _combine_grad(s["dOut"], s["Ys"], s["slot"], s["offsets"], s["w"])
        return dict(out=_combine(s["Ys"], s["slot"], s["offsets"], s["w"]), dYs=dYs, dw=dw,
                    dX=_combine(s["dXs"], s["slot"], s["offsets"]))
    if kind == "keep":
        return dict(X=_kept_values(case["act"], *_keep(case["act"], s["X"])).to(torch.bfloat16))
    if kind == "dscale8":
        return dict(dS=_dscale8(s))
    return _loss(s)


# ---------------------------------------------------------------- the library
def _library(s):
    from paper_2609_04526_amd import sq
    case = s["case"]
    kind = case["kind"]
    if kind == "dispatch":
        offsets, token, slot = sq.sq_moe_sort(s["ids"], case["E"])
        return dict(offsets=offsets, token=token, slot=slot, Xs=sq.sq_moe_gather(s["X"], slot, offsets))
    if kind == "combine":
        out = sq.sq_moe_combine(s["Ys"], s["slot"], s["offsets"], s["w"], out_dtype=_dtype(case))
        dYs, dw = sq.sq_moe_combine_bwd(s["dOut"], s["Ys"], s["slot"], s["offsets"], s["w"])
        return dict(out=out, dYs=dYs, dw=dw,
                    dX=sq.sq_moe_combine(s["dXs"], s["slot"], s["offsets"], out_dtype=_dtype(case)))
    if kind == "keep":
        return dict(X=sq.sq_act_unpack(case["act"], *sq.sq_act_pack(case["act"], s["X"])))
    if kind == "dscale8":
        if case["E"]:
            return dict(dS=sq.sq_bwd_dscale_act8_batched(case["fmt"], case["act"], s["kept"], s["kept_scales"],
                                                         s["token"], s["offsets"], s["dY"], s["codes"]))
        return dict(dS=sq.sq_bwd_dscale_act8(case["fmt"], case["act"], s["kept"], s["kept_scales"], s["dY"], s["codes"]))
    loss, lse = sq.sq_ce_fwd(case["head"], s["X"], s["W"], s["y"], scales=s.get("scales"), ws2=WS2)
    dX = sq.sq_ce_bwd(case["head"], s["X"], s["W"], s["y"], lse, s["dloss"], scales=s.get("scales"), ws2=WS2,
                      out_dtype=torch.bfloat16)
    return dict(loss=loss, lse=lse, dX=dX)


def run(state):
    return _library(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, T = case["kind"], case["T"]
    if kind in ("dispatch", "combine"):
        N, H, K = T * case["K"], case["H"], case["K"]
        b = 2 if case["dtype"] == "bf16" else 4
        kept = 1.0 - case["drop"]
        if kind == "dispatch":
            return dict(bytes=N * ((8 if case["ids"] == "i64" else 4) + 8) + 4 * (case["E"] + 1) + (T + N) * H * b,
                        flops=0)
        # Ys, dOut and dXs read; out, dYs and dX written; slots, weights and their gradients
        return dict(bytes=(2 * kept * N + N + 3 * T) * H * b + 12 * N, flops=(3 * kept + 3) * N * H)
    if kind == "keep":
        n = T * case["I"]
        return dict(bytes=n * (2 + 2 * (1 + 1 / ACT_BLOCK) + 2), flops=4 * n)
    if kind == "dscale8":
        O, I, E, N = case["O"], case["I"], max(1, case["E"]), T * case["K"]
        G = I // BLOCK[case["fmt"]]
        return dict(bytes=T * I * (1 + 1 / ACT_BLOCK) + N * O * 2 + E * (O * I / 2 + O * G * 4) + (4 * N if case["E"] else 0),
                    flops=2 * N * O * I)
    V, H = case["V"], case["H"]
    rows = max(1, T * (1.0 - case["ignored"]))
    w = V * H * (2 if case["head"] == "bf16" else 0.5 + 1 / BLOCK[case["head"]])
    # the logits once and dX; the weight once for the statistics and once for the gradient, which needs them
    return dict(bytes=2 * w + T * (2 * H * 2 + 8 + 12), flops=4 * rows * V * H)


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    kind = case["kind"]
    if kind == "dispatch":
        E, K = case["E"], case["K"]
        key = s["ids"].reshape(-1).long()
        key = torch.where((key < 0) | (key >= E), torch.full_like(key, E), key)
        # the rows in order of the composite key (expert, pair)
        n = key.numel()
        by = torch.sort(key * n + torch.arange(n, device=key.device)).values % n
        rows = s["X"].to(f64)[torch.div(by, K, rounding_mode="floor")]
        rows[int((key < E).sum()):] = 0
        return dict(offsets=None, token=None, slot=None, Xs=rows)
    if kind == "combine":
        R = int(s["offsets"][-1])
        slot, w = s["slot"].long(), s["w"].to(f64)
        T, K = slot.shape
        N, H = s["Ys"].shape
        pair = torch.empty(N, dtype=torch.long, device=slot.device)
        pair[slot.reshape(-1)] = torch.arange(N, device=slot.device)
        tok, wr = pair[:R] // K, w.reshape(-1)[pair[:R]]
        out, dX = (torch.zeros((T, H), dtype=f64, device=slot.device) for _ in range(2))
        out.index_add_(0, tok, s["Ys"][:R].to(f64) * wr[:, None])
        dX.index_add_(0, tok, s["dXs"][:R].to(f64))
        dYs = torch.zeros((N, H), dtype=f64, device=slot.device)
        d = s["dOut"].to(f64)[tok]
        dYs[:R] = d * wr[:, None]
        dw = torch.zeros(N, dtype=f64, device=slot.device)
        dw[pair[:R]] = (d * s["Ys"][:R].to(f64)).sum(1)
        return dict(out=out, dYs=dYs, dw=dw.view(T, K), dX=dX)
    if kind == "keep":
        x = s["X"].to(f64).view(case["T"], -1, ACT_BLOCK)
        amax = x.abs().amax(-1, keepdim=True).clamp(min=1e-300)
        if case["act"] == "int8":
            step = torch.exp2((torch.floor(torch.log2(amax)) - 6).clamp(-126, 127))
            v = torch.round(x / step).clamp(-127, 127) * step
        else:
            unit = torch.exp2(torch.ceil(torch.log2(amax / 448.0)).clamp(-126, 127))
            r = x / unit
            # four significant bits down to 2^-6, steps of 2^-9 below
            step = torch.exp2(torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -6))) - 3)
            v = torch.round(r / step) * step * unit
        return dict(X=v.view(case["T"], -1))
    if kind == "dscale8":
        if not case["E"]:
            return dict(dS=_exact_dscale(s, _kept_values(case["act"], s["kept"], s["kept_scales"], f64), s["dY"], s["codes"]))
        x = _kept_values(case["act"], s["kept"], s["kept_scales"], f64)
        o, tok = s["offsets"].tolist(), s["token"].long()
        return dict(dS=torch.stack([_exact_dscale(s, x[tok[a:b]], s["dY"][a:b], s["codes"][e])
                                    for e, (a, b) in enumerate(zip(o[:-1], o[1:]))]))
    # pieces of the tokens, so that the logits in 64 bits fit
    w = _weight(s, f64)
    loss, lse, dX = [], [], []
    for a in range(0, case["T"], 1024):
        y, x = s["y"][a:a + 1024], s["X"][a:a + 1024].to(f64)
        valid = (y >= 0).to(f64)
        logits = x @ w.t()
        z = torch.logsumexp(logits, 1)
        lse.append(z * valid)
        loss.append((z - torch.gather(logits, 1, y.clamp(min=0)[:, None])[:, 0]) * valid)
        c = s["dloss"][a:a + 1024].to(f64) * valid
        dX.append(c[:, None] * (torch.exp(logits - z[:, None]) @ w - w[y.clamp(min=0)]))
    return dict(loss=torch.cat(loss), lse=torch.cat(lse), dX=torch.cat(dX))


def _exact_dscale(s, x, dy, codes):
    v = _code_values(codes, torch.float64) * (dy.to(torch.float64).t().contiguous() @ x)
    return v.view(v.shape[0], -1, BLOCK[s["case"]["fmt"]]).sum(-1)
