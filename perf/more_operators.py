"""Workloads of a 4-bit student that learns from a teacher, each in a plain form
(elementary torch operations in 32 bits) and through the library's entry points.

  keep4     an activation in the layer's 4-bit storage, and read back
  linear4   one linear with both operands in 4 bits: its input is quantised and
            multiplied with the frozen codes
  experts4  stacked experts on routed rows of one layer's tokens, both operands
            in 4 bits, the experts' ranges read on the device
  distill   divergence of a language-model head from a teacher's top logits,
            with the gradient of the head's input
  embed     token ids through an embedding (bf16, or in the MXFP4 or NVFP4
            storage), and the gradient of what is trained of it: the rows of a
            bf16 table, the block scales of a 4-bit one

`own` selects the side: False runs the plain forms, True the library.  Inputs
are synthetic and drawn on the GPU from the seed.
"""

import math

import torch

own = False

BLOCK = {"mx": 32, "nv": 16}
X_WS2 = 2.0 ** -9                # of a calibrated activation: values up to 5.25 are not cut off
W_WS2 = 1.0 / 448.0
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
LINEARS = [(4096, 4096), (1024, 4096), (14336, 4096), (4096, 14336)]     # of the dense model of bench.py
EXPERTS = [(768, 2048), (2048, 768), (1536, 2048)]                       # of its MoE layer: gate or up, down, gate and up


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # a kept activation of an odd batch
        dict(name="keep4 mx t333", kind="keep4", fmt="mx", T=333, I=4096),
        # the widest activation of a dense model's layer at 8192 tokens
        dict(name="keep4 nv t8192", kind="keep4", fmt="nv", T=8192, I=14336),
        # one token of a serving loop: the bytes of the codes, and latency
        dict(name="linear4 mx 4096x4096 t1", kind="linear4", fmt="mx", T=1, O=4096, I=4096, out="bf16"),
        # a small batch of a serving loop with an odd count, through the widest layer
        dict(name="linear4 mx 14336x4096 t37", kind="linear4", fmt="mx", T=37, O=14336, I=4096, out="bf16"),
        # a training batch's or a long prompt's tokens through the same layer
        dict(name="linear4 mx 14336x4096 t8192", kind="linear4", fmt="mx", T=8192, O=14336, I=4096, out="bf16"),
        # a step of 16 sequences of a served MoE layer: most experts have a row or none
        dict(name="experts4 128x768x2048 t16", kind="experts4", E=128, T=16, K=8, O=768, I=2048, drop=0.0),
        # a training step's tokens through it, some of them dropped by a capacity limit
        dict(name="experts4 128x1536x2048 t4096", kind="experts4", E=128, T=4096, K=8, O=1536, I=2048, drop=0.05),
        # the head of a small test model on a few tokens: latency
        dict(name="distill bf16 1000x512 t5", kind="distill", head="bf16", T=5, V=1000, H=512, K=16, tau=1.0,
             z="f32", ignored=0.0),
        # a batch whose prompt tokens are masked, odd vocabulary, head in the layer's storage
        dict(name="distill mx 50001x4096 t1999", kind="distill", head="mx", T=1999, V=50001, H=4096, K=64, tau=2.0,
             z="bf16", ignored=0.4),
        # a full training batch over a large vocabulary: the largest call
        dict(name="distill bf16 131072x4096 t4096", kind="distill", head="bf16", T=4096, V=131072, H=4096, K=64,
             tau=1.0, z="f32", ignored=0.0),
        # a bf16 table of an odd vocabulary on a short batch
        dict(name="embed bf16 50001x2048 t1999", kind="embed", head="bf16", T=1999, V=50001, H=2048, ids="i64",
             out="bf16", ignored=0.1),
        # a long packed batch through a table in the layer's storage
        dict(name="embed mx 131072x4096 t16384", kind="embed", head="mx", T=16384, V=131072, H=4096, ids="i64",
             out="bf16", ignored=0.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    kind = rng.choice(["keep4", "linear4", "linear4", "experts4", "experts4", "distill", "distill", "embed", "embed"])
    if kind == "keep4":
        return dict(kind=kind, fmt=rng.choice(["mx", "nv"]), T=_log_int(rng, 1, 8192), I=32 * _log_int(rng, 8, 448))
    if kind == "linear4":
        fmt = rng.choice(["mx", "mx", "mx", "nv"])
        O, I = rng.choice(LINEARS) if rng.random() < 0.5 else (8 * _log_int(rng, 32, 1792), 32 * _log_int(rng, 16, 448))
        c = dict(kind=kind, fmt=fmt, T=_log_int(rng, 1, 8192), O=O, I=I, out=rng.choice(["bf16", "f32"]))
        while c["T"] * O * I > 8192 * 14336 * 4096:
            c["T"] = c["T"] * 2 // 3
        return c
    if kind == "experts4":
        O, I = rng.choice(EXPERTS) if rng.random() < 0.6 else (8 * _log_int(rng, 32, 256), 32 * _log_int(rng, 8, 64))
        E = rng.choice([8, 32, 60, 128])
        return dict(kind=kind, E=E, T=_log_int(rng, 1, 4096), K=rng.choice([1, 2, 4, 8]), O=O, I=I,
                    drop=rng.choice([0.0, 0.0, 0.05]))
    head = rng.choice(["bf16", "mx", "nv"])
    if kind == "distill":
        c = dict(kind=kind, head=head, T=_log_int(rng, 1, 8192), V=_log_int(rng, 1000, 160000),
                 H=32 * _log_int(rng, 16, 256), K=_log_int(rng, 1, 256), tau=rng.choice([1.0, 2.0, 0.7]),
                 z=rng.choice(["f32", "bf16"]), ignored=rng.choice([0.0, 0.1, 0.5]))
        while c["T"] * c["V"] * c["H"] > 4096 * 131072 * 4096 or c["T"] * c["K"] * c["H"] > 4096 * 64 * 4096:
            c["T"] = c["T"] * 2 // 3
        return c
    c = dict(kind=kind, head=head, T=_log_int(rng, 1, 16384), V=_log_int(rng, 1000, 131072), H=32 * _log_int(rng, 8, 128),
             ids=rng.choice(["i64", "i32"]), out=rng.choice(["bf16", "f32"]), ignored=rng.choice([0.0, 0.1, 0.5]))
    while head == "bf16" and c["V"] * c["H"] > 50001 * 4096:
        c["V"] = c["V"] * 2 // 3
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1009 + k) % (1 << 62))
    return g


def _normal(seed, k, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=_gen(seed, k), device="cuda").to(dtype)


def _uniform(seed, k, shape):
    return torch.rand(shape, generator=_gen(seed, k), device="cuda")


def _activation(seed, k, T, I):
    """Activations with uneven channels, a few of them far larger than the rest."""
    g = _gen(seed, k)
    chan = torch.exp(0.5 * torch.randn(I, generator=g, device="cuda"))
    chan = torch.where(torch.rand(I, generator=g, device="cuda") < 0.005, 20.0 * chan, chan)
    return (torch.randn((T, I), generator=g, device="cuda") * chan).to(torch.bfloat16)


def _codes(seed, k, shape):
    return torch.randint(0, 256, shape, generator=_gen(seed, k), device="cuda", dtype=torch.uint8)


def _scales(seed, k, shape, fmt, H):
    """Scale bytes of a weight whose rows of H values have a norm of about one."""
    z = torch.randn(shape + (H // BLOCK[fmt],), generator=_gen(seed, k), device="cuda")
    if fmt == "mx":
        mid = round(-1.55 - 0.5 * math.log2(H))               # E2M1's mean square is 8.6
        return (torch.round(0.7 * z + mid).clamp_(-127, 127) + 127).to(torch.uint8)
    return (z.abs() * (448.0 * 0.4 / math.sqrt(H))).to(torch.float8_e4m3fn).view(torch.uint8)


def _table(s, case, seed, rows):
    """The embedding's or the head's rows: s["W"], and s["scales"] in 4 bits."""
    H, head = case["H"], case["head"]
    s["scales"] = None
    if head == "bf16":
        s["W"] = (torch.randn((rows, H), generator=_gen(seed, 1), device="cuda") / math.sqrt(H)).to(torch.bfloat16)
    else:
        s["W"] = _codes(seed, 1, (rows, H // 2))
        s["scales"] = _scales(seed, 2, (rows,), head, H)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def prepare(case, seed):
    kind, T = case["kind"], case["T"]
    s = dict(case=case)
    if kind == "keep4":
        s["X"] = _activation(seed, 1, T, case["I"])
    elif kind == "linear4":
        s["X"] = _activation(seed, 1, T, case["I"])
        s["codes"] = _codes(seed, 2, (case["O"], case["I"] // 2))
        s["scales"] = _scales(seed, 3, (case["O"],), case["fmt"], case["I"])
    elif kind == "experts4":
        E, K = case["E"], case["K"]
        s["X"] = _activation(seed, 1, T, case["I"])
        s["codes"] = _codes(seed, 2, (E, case["O"], case["I"] // 2))
        s["scales"] = _scales(seed, 3, (E, case["O"]), "mx", case["I"])
        # the top experts of uneven router scores, the dropped pairs last, as the sort by expert leaves them
        score = _normal(seed, 4, (T, E), torch.float32) + 0.5 * _normal(seed, 5, (E,), torch.float32)
        ids = torch.topk(score, K, dim=1).indices
        key = torch.where(_uniform(seed, 6, (T, K)) < case["drop"], torch.full_like(ids, E), ids).reshape(-1)
        order = torch.argsort(key, stable=True)
        s["rows"] = (order // K).to(torch.int32)
        count = torch.bincount(key, minlength=E + 1)[:E]
        s["offsets"] = torch.cat((count.new_zeros(1), torch.cumsum(count, 0))).to(torch.int32)
    elif kind == "distill":
        V, H, K = case["V"], case["H"], case["K"]
        _table(s, case, seed, V)
        # frequent tokens are frequent among a teacher's candidates too
        ids = (V * _uniform(seed, 4, (T, K)) ** 3).long().clamp_(max=V - 1)
        z = torch.sort(2.5 * _normal(seed, 5, (T, K), torch.float32), dim=1, descending=True).values
        s["z"] = (z + 6.0).to(_dtype(case["z"]))
        # some tokens have fewer entries, ignored ones none
        keep = (1 + (K * (0.5 + 4.0 * _uniform(seed, 6, (T, 1)))).long()).clamp_(max=K)
        keep = torch.where(_uniform(seed, 7, (T, 1)) < case["ignored"], torch.zeros_like(keep), keep)
        s["ids"] = torch.where(torch.arange(K, device="cuda") < keep, ids, torch.full_like(ids, -1))
        # hidden states that lean towards the teacher's first choice, some of them far
        first = dict(s, W=s["W"][ids[:, 0]], scales=None if s["scales"] is None else s["scales"][ids[:, 0]])
        lean = _values(first, torch.float32)
        lean = lean / lean.norm(dim=1, keepdim=True)
        s["X"] = (_normal(seed, 8, (T, H), torch.float32) + 9.0 * _uniform(seed, 9, (T, 1)) * lean).to(torch.bfloat16)
        s["dloss"] = (0.5 + _uniform(seed, 10, (T,))) / max(1, T)
    else:
        V, H = case["V"], case["H"]
        _table(s, case, seed, V)
        # frequent tokens, one of them (a space, a line's end) every twentieth
        ids = (V * _uniform(seed, 4, (T,)) ** 4).long().clamp_(max=V - 1)
        ids = torch.where(_uniform(seed, 5, (T,)) < 0.05, torch.full_like(ids, V // 3), ids)
        ids = torch.where(_uniform(seed, 6, (T,)) < case["ignored"], torch.full_like(ids, -1), ids)
        s["ids"] = ids if case["ids"] == "i64" else ids.to(torch.int32)
        s["dOut"] = _normal(seed, 7, (T, H), _dtype(case["out"]))
        s["factor"] = math.sqrt(H)
    return s


# ---------------------------------------------------------------- plain forms
def _e2m1(a):
    """Index of the nearest E2M1 magnitude to a >= 0, ties to the even index; NaN gives 0."""
    n = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int()
    return n + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int()


def _quantised(fmt, X):
    """The values of X in the layer's 4-bit storage (without the NVFP4 scalar), fp32 [T, I]."""
    T, I = X.shape
    x = X.float().view(T, I // BLOCK[fmt], BLOCK[fmt])
    amax = x.abs().amax(-1, keepdim=True)
    table = torch.tensor(E2M1, device=X.device)
    if fmt == "mx":
        m, e = torch.frexp(amax / 6.0)
        k = torch.where(m > 0.5, e, e - 1)
        k = torch.where(amax == 0, torch.full_like(k, -127), k).clamp(-127, 127)
        v = torch.ldexp(table[_e2m1(torch.ldexp(x.abs(), -k)).long()], k)
    else:
        ws2 = torch.tensor(X_WS2, device=X.device)
        scale = (amax / 6.0 / ws2).clamp(max=448.0).to(torch.float8_e4m3fn).float()
        q = torch.where(scale > 0, x.abs() / (scale * ws2), torch.zeros((), device=X.device))
        v = table[_e2m1(q).long()] * scale
    return torch.where(x < 0, -v, v).view(T, I)


def _code_values(codes, dtype):
    table = torch.tensor(E2M1 + [-v for v in E2M1], dtype=dtype, device=codes.device)
    nib = torch.stack((codes & 15, codes >> 4), dim=-1)
    return table[nib.long()].view(codes.shape[:-1] + (2 * codes.shape[-1],))


def _weight(fmt, codes, scales, dtype):
    """Values of codes [.., I/2] and scales [.., G], with the NVFP4 scalar."""
    w = _code_values(codes, dtype)
    if fmt == "mx":
        eff = torch.exp2(scales.to(dtype) - 127.0)
    else:
        eff = scales.view(torch.float8_e4m3fn).to(dtype) * torch.tensor(W_WS2, dtype=torch.float32).to(dtype)
    return (w.view(scales.shape + (BLOCK[fmt],)) * eff[..., None]).view(w.shape)


def _values(s, dtype):
    """The rows of an embedding or a head as plain values."""
    head = s["case"]["head"]
    return s["W"].to(dtype) if head == "bf16" else _weight(head, s["W"], s["scales"], dtype)


def _experts4(s):
    case, rows = s["case"], s["rows"].long()
    N, o = rows.numel(), s["offsets"].long()
    x = _quantised("mx", s["X"])
    longest = max(1, int((o[1:] - o[:-1]).max()))
    at = o[:-1, None] + torch.arange(longest, device=rows.device)
    inside = at < o[1:, None]
    at = torch.where(inside, at, torch.full_like(at, N))
    w = _weight("mx", s["codes"], s["scales"], torch.float32).transpose(1, 2).contiguous()
    y = torch.bmm(torch.cat((x[rows], x.new_zeros(1, x.shape[1])))[at], w)
    out = y.new_zeros((N + 1, case["O"]))
    out[at.reshape(-1)] = y.view(-1, case["O"])               # the padding goes to the row behind the last
    return out[:N].to(torch.bfloat16)


def _distill(s):
    case = s["case"]
    tau, x, w = case["tau"], s["X"].float(), _values(s, torch.float32)
    counts = s["ids"] >= 0
    live = counts.any(1)
    at = torch.where(counts, s["ids"], torch.zeros_like(s["ids"]))
    sl = (x @ w.t()) / tau
    top = sl.amax(1, keepdim=True)
    p = torch.exp(sl - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    zero = torch.zeros((), device=x.device)
    picked = torch.where(counts, sl.gather(1, at), zero)
    del sl
    z = torch.where(counts, s["z"].float() / tau, torch.full((), -1e30, device=x.device))
    z = z - z.amax(1, keepdim=True)
    q = torch.where(counts, torch.exp(z), zero)
    mass = q.sum(1, keepdim=True).clamp(min=1e-30)
    q = q / mass
    log_q = torch.where(q > 0, z - torch.log(mass), zero)
    loss = tau * tau * (q * (log_q + ((top - picked) + torch.log(total)))).sum(1)
    p = p / total
    p.scatter_add_(1, at, -q)
    p = p * torch.where(live, tau * s["dloss"], zero)[:, None]
    return dict(loss=torch.where(live, loss, zero), lse=torch.where(live, lse, zero), picked=picked,
                dX=(p @ w).to(torch.bfloat16))


def _embed(s):
    case = s["case"]
    head, V, H = case["head"], case["V"], case["H"]
    ids = s["ids"].long()
    live = (ids >= 0) & (ids < V)
    at = torch.where(live, ids, torch.zeros_like(ids))
    rows = _values(dict(s, W=s["W"][at], scales=None if s["scales"] is None else s["scales"][at]), torch.float32)
    zero = torch.zeros((), device=ids.device)
    out = torch.where(live[:, None], rows * s["factor"], zero).to(_dtype(case["out"]))
    d = torch.where(live[:, None], s["dOut"].float() * s["factor"], zero)
    if head != "bf16":
        d = (d * _code_values(s["W"][at], torch.float32)).view(-1, H // BLOCK[head], BLOCK[head]).sum(-1)
    grad = d.new_zeros((V, d.shape[1]))
    grad.index_add_(0, at, d)
    return dict(out=out, grad=grad)


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "keep4":
        x = _quantised(case["fmt"], s["X"])
        return dict(X=(x if case["fmt"] == "mx" else x * X_WS2).to(torch.bfloat16))
    if kind == "linear4":
        y = _quantised(case["fmt"], s["X"]) @ _weight(case["fmt"], s["codes"], s["scales"], torch.float32).t()
        return dict(Y=(y if case["fmt"] == "mx" else y * X_WS2).to(_dtype(case["out"])))
    if kind == "experts4":
        return dict(Y=_experts4(s))
    return _distill(s) if kind == "distill" else _embed(s)


# ---------------------------------------------------------------- the library
def _library(s):
    from paper_2609_04526_amd import sq
    case = s["case"]
    kind = case["kind"]
    if kind == "keep4":
        return dict(X=sq.sq_act4_unpack(case["fmt"], *sq.sq_act4_pack(case["fmt"], s["X"], ws2=X_WS2), ws2=X_WS2))
    if kind == "linear4":
        x, xs = sq.sq_act4_pack(case["fmt"], s["X"], ws2=X_WS2)
        return dict(Y=sq.sq_fwd_act4(case["fmt"], x, xs, s["codes"], s["scales"], x_ws2=X_WS2, ws2=W_WS2,
                                     out_dtype=_dtype(case["out"])))
    if kind == "experts4":
        x, xs = sq.sq_act4_pack("mx", s["X"])
        return dict(Y=sq.sq_fwd_act4_batched("mx", x, xs, s["rows"], s["offsets"], s["codes"], s["scales"],
                                             out_dtype=torch.bfloat16))
    if kind == "distill":
        head = dict(temperature=case["tau"], scales=s["scales"], ws2=W_WS2)
        loss, lse, picked = sq.sq_distill_fwd(case["head"], s["X"], s["W"], s["ids"], s["z"], **head)
        dX = sq.sq_distill_bwd(case["head"], s["X"], s["W"], s["ids"], s["z"], lse, picked, s["dloss"],
                               out_dtype=torch.bfloat16, **head)
        return dict(loss=loss, lse=lse, picked=picked, dX=dX)
    out = sq.sq_embed_fwd(case["head"], s["ids"], s["W"], scales=s["scales"], ws2=W_WS2, factor=s["factor"],
                          out_dtype=_dtype(case["out"]))
    if case["head"] == "bf16":
        return dict(out=out, grad=sq.sq_embed_bwd(s["ids"], s["dOut"], case["V"], factor=s["factor"]))
    return dict(out=out, grad=sq.sq_embed_bwd_dscale(case["head"], s["ids"], s["dOut"], s["W"], factor=s["factor"]))


def run(state):
    return _library(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, T = case["kind"], case["T"]
    if kind == "keep4":
        n = T * case["I"]
        return dict(bytes=n * (2 + 2 * (0.5 + 1 / BLOCK[case["fmt"]]) + 2), flops=4 * n)
    if kind in ("linear4", "experts4"):
        O, I = case["O"], case["I"]
        fmt, E, N = case.get("fmt", "mx"), case.get("E", 1), T * case.get("K", 1)
        routed = N * (1.0 - case.get("drop", 0.0))
        b = 4 if case.get("out") == "f32" else 2
        # the input read and its codes written; of many experts only those that have a row
        used = E * (1.0 - (1.0 - 1.0 / E) ** routed) if E > 1 else 1.0
        return dict(bytes=T * I * (2 + 0.5 + 1 / BLOCK[fmt]) + used * O * I * (0.5 + 1 / BLOCK[fmt]) + N * O * b
                    + (4 * N if E > 1 else 0), flops=2 * routed * O * I)
    V, H, head = case["V"], case["H"], case["head"]
    row = H * (2 if head == "bf16" else 0.5 + 1 / BLOCK[head])
    kept = 1.0 - case["ignored"]
    if kind == "distill":
        # the logits once and dX; the head once for the statistics and once for the gradient, which needs them
        return dict(bytes=2 * V * row + T * (2 * H * 2 + 12 + case["K"] * (2 * 8 + 2 * 4 + 8)),
                    flops=4 * max(1.0, T * kept) * V * H)
    b = 2 if case["out"] == "bf16" else 4
    seen = min(V, T * kept)                                   # rows of the table, read again for the scales' gradient
    grad = V * H * 4 if head == "bf16" else V * (H // BLOCK[head]) * 4 + seen * H / 2
    return dict(bytes=seen * row + T * H * b * (1 + kept) + grad + 8 * T, flops=(2 if head == "bf16" else 4) * T * kept * H)


# ---------------------------------------------------------------- the same in 64 bits
def _exact_quantised(fmt, X):
    f64 = torch.float64
    x = X.to(f64).view(X.shape[0], -1, BLOCK[fmt])
    amax = x.abs().amax(-1, keepdim=True)
    if fmt == "mx":
        unit = torch.exp2(torch.ceil(torch.log2((amax / 6.0).clamp(min=2.0 ** -127))).clamp(-127, 127))
        step_of = unit
    else:
        # the scale's byte and the quotients are defined as fp32 steps
        unit = ((amax / 6.0).float().to(f64) / X_WS2).float().to(f64).clamp(max=448.0)
        low = torch.exp2(torch.floor(torch.log2(unit.clamp(min=2.0 ** -6))) - 3)
        unit = torch.round(unit / low) * low
        step_of = (unit * X_WS2).float().to(f64)
    q = torch.where(step_of > 0, x / step_of, torch.zeros_like(x)).float().to(f64)
    step = 0.5 * torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=1.0, max=6.0))))
    return (torch.round(q / step) * step).clamp(-6.0, 6.0).mul(unit).view(X.shape)


def exact(case, seed):
    s = prepare(case, seed)
    f64, kind, T = torch.float64, case["kind"], case["T"]
    if kind in ("keep4", "linear4"):
        fmt = case["fmt"]
        w = None if kind == "keep4" else _weight(fmt, s["codes"], s["scales"], f64)
        parts = []
        for a in range(0, T, 2048):
            x = _exact_quantised(fmt, s["X"][a:a + 2048]) * (1.0 if fmt == "mx" else X_WS2)
            parts.append(x if w is None else x @ w.t())
        return {"X" if w is None else "Y": torch.cat(parts)}
    if kind == "experts4":
        x, o, rows = _exact_quantised("mx", s["X"]), s["offsets"].tolist(), s["rows"].long()
        y = torch.zeros((rows.numel(), case["O"]), dtype=f64, device=rows.device)
        for e, (a, b) in enumerate(zip(o[:-1], o[1:])):
            if b > a:
                y[a:b] = x[rows[a:b]] @ _weight("mx", s["codes"][e], s["scales"][e], f64).t()
        return dict(Y=y)
    if kind == "distill":
        tau, w = case["tau"], _values(s, f64)
        loss, lse, picked, dX = [], [], [], []
        # pieces of the tokens, so that the logits in 64 bits fit
        for a in range(0, T, 1024):
            b = min(T, a + 1024)
            ids, n = s["ids"][a:b], b - a
            counts = (ids >= 0).to(f64)
            live = counts.amax(1)
            logits = (s["X"][a:b].to(f64) @ w.t()) / tau
            norm = torch.logsumexp(logits, 1)
            mine = torch.gather(logits, 1, ids.clamp(min=0))
            teacher = torch.softmax(s["z"][a:b].to(f64) / tau + torch.log(counts).clamp(min=-1e9), 1) * counts
            terms = torch.special.xlogy(teacher, teacher) - teacher * (mine - norm[:, None])
            loss.append(tau ** 2 * terms.sum(1))
            lse.append(norm * live)
            picked.append(mine * counts)
            c = (s["dloss"][a:b].to(f64) * live * tau)[:, None]
            flat = w[ids.clamp(min=0).reshape(-1)].view(n, -1, case["H"]) if n * ids.shape[1] * case["H"] < 1 << 28 else None
            if flat is not None:
                mean = torch.bmm(teacher[:, None], flat)[:, 0]
            else:
                mean = torch.stack([teacher[i] @ w[ids[i].clamp(min=0)] for i in range(n)])
            dX.append(c * (torch.exp(logits - norm[:, None]) @ w - mean))
        return dict(loss=torch.cat(loss), lse=torch.cat(lse), picked=torch.cat(picked), dX=torch.cat(dX))
    head, V, H = case["head"], case["V"], case["H"]
    ids, f = s["ids"].long(), s["factor"]
    kept = torch.nonzero((ids >= 0) & (ids < V))[:, 0]
    at = ids[kept]
    out = torch.zeros((T, H), dtype=f64, device=ids.device)
    out[kept] = f * _values(dict(s, W=s["W"][at], scales=None if head == "bf16" else s["scales"][at]), f64)
    # the rows of one id summed first, then written to their place
    seen, where = torch.unique(at, return_inverse=True)
    sums = torch.zeros((seen.numel(), H), dtype=f64, device=ids.device)
    sums.index_put_((where,), s["dOut"][kept].to(f64) * f, accumulate=True)
    if head != "bf16":
        sums = (sums * _code_values(s["W"][seen], f64)).view(-1, H // BLOCK[head], BLOCK[head]).sum(-1)
    grad = torch.zeros((V, sums.shape[1]), dtype=f64, device=ids.device)
    grad[seen] = sums
    return dict(out=out, grad=grad)
