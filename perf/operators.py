"""Timed cases of the operators around the MoE layer: the residual addition with its norm, the 8-bit integer rows and
products of a dense FFN (the always-on shared expert), and the routing by scores.

`run` computes a case in elementary torch operations, or, where `own` is true, through the library's entry points.
"""
from __future__ import annotations

import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the norm between two layers: one token of interactive decoding
        dict(name="norm 1x2048", op="norm", T=1, d=2048, delta="bf16", h=True),
        # a decode batch whose layer output is the fp32 sum of the separate calls; only the 8-bit output is wanted
        dict(name="norm 61x3584 f32", op="norm", T=61, d=3584, delta="f32", h=False),
        # a prefill batch, both outputs: bf16 for the router, 8 bits for the products
        dict(name="norm 4096x2048", op="norm", T=4096, d=2048, delta="bf16", h=True),
        # SwiGLU activations of a ragged batch on their way into the down projection
        dict(name="rows 333x2816", op="rows", rows=333, cols=2816),
        # the gate/up weights of a wide shared expert, quantised when they are loaded
        dict(name="rows 40960x3584", op="rows", rows=40960, cols=3584),
        # the shared expert's down projection for one token
        dict(name="product 1x2048x2816", op="product", T=1, n=2048, k=2816, out="bf16"),
        # the same of a wide shared expert for an odd decode batch, as the fp32 rows that other experts are added to
        dict(name="product 77x3584x20480", op="product", T=77, n=3584, k=20480, out="f32"),
        # the down projection of a prefill batch
        dict(name="product 4096x2048x2816", op="product", T=4096, n=2048, k=2816, out="bf16"),
        # the shared expert's gate/up products of a decode batch
        dict(name="swiglu 16x2816x2048", op="swiglu", T=16, inter=2816, k=2048),
        # the same of a wide shared expert at prefill
        dict(name="swiglu 4096x20480x3584", op="swiglu", T=4096, inter=20480, k=3584),
        # one token, softmax scores, groups by their best expert
        dict(name="route 1x64", op="route", T=1, N=64, K=6, score="softmax", bias=False, groups=8, top_groups=3, pair=False,
             norm=False, scale=16.0),
        # a prefill batch, sigmoid scores with a balancing bias, groups by their two best experts
        dict(name="route 8192x256", op="route", T=8192, N=256, K=8, score="sigmoid", bias=True, groups=8, top_groups=4, pair=True,
             norm=True, scale=2.5),
    ]


def _spread(rng, low, high, step=1):
    """A multiple of `step` between low and high, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(low, min(high, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["norm", "rows", "product", "swiglu", "route"])
    if op == "norm":
        return dict(op=op, T=_spread(rng, 1, 4096), d=_spread(rng, 64, 8192, 8), delta=rng.choice(["bf16", "f32"]),
                    h=rng.random() < 0.7)
    if op == "rows":
        return dict(op=op, rows=_spread(rng, 1, 8192), cols=_spread(rng, 64, 20480, 8))
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        N = groups * _spread(rng, 8, 512 // groups)
        top = rng.randint(max(1, groups // 4), groups)
        return dict(op=op, T=_spread(rng, 1, 8192), N=N, K=rng.randint(1, min(10, top * (N // groups))),
                    score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.6, groups=groups, top_groups=top,
                    pair=groups > 1 and rng.random() < 0.5, norm=rng.random() < 0.6, scale=rng.choice([1.0, 2.5, 16.0]))
    T, n, k = _spread(rng, 1, 4096), _spread(rng, 64, 20480, 8), _spread(rng, 64, 20480, 16)
    while T * n * k > 4096 * 20480 * 3584:
        T = max(1, T // 2)
    if op == "product":
        return dict(op=op, T=T, n=n, k=k, out=rng.choice(["bf16", "f32"]))
    return dict(op=op, T=T, inter=n, k=k)


# ------------------------------------------------------------------------------------------------ inputs
def _codes(rows, cols, std, gen):
    """Codes and scales of normally distributed rows, as a quantiser of rows leaves them."""
    w = torch.randn(rows, cols, device="cuda", generator=gen)
    big = w.abs().amax(1, keepdim=True)
    return torch.round(w * (127.0 / big)).to(torch.int8), (big[:, 0] * (std / 127.0)).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c, dev, f32 = case, "cuda", torch.float32
    randn = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
    s = dict(case=c)
    if c["op"] == "norm":
        T, d = c["T"], c["d"]
        wide = 1 + 15 * (torch.rand(d, device=dev, generator=gen) < 0.01)   # a residual stream has a few large channels
        s["x"] = (randn(T, d) * wide).bfloat16()
        s["delta"] = randn(T, d).mul_(0.5).to(torch.bfloat16 if c["delta"] == "bf16" else f32)
        s["weight"] = (1 + 0.1 * randn(d)).bfloat16()
        s["h"] = torch.empty(T, d, dtype=torch.bfloat16, device=dev) if c["h"] else None
        s["q"] = torch.empty(T, d, dtype=torch.int8, device=dev)
        s["scale"] = torch.empty(T, dtype=f32, device=dev)
    elif c["op"] == "rows":
        s["w"] = randn(c["rows"], c["cols"]).mul_(0.02).bfloat16()
        s["q"] = torch.empty(c["rows"], c["cols"], dtype=torch.int8, device=dev)
        s["scale"] = torch.empty(c["rows"], dtype=f32, device=dev)
    elif c["op"] == "route":
        T, N, K = c["T"], c["N"], c["K"]
        s["logits"] = randn(T, N) + 0.5 * randn(N)
        s["bias"] = 0.1 * randn(N) if c["bias"] else None
        s["idx"] = torch.empty(T, K, dtype=torch.int32, device=dev)
        s["gate"] = torch.empty(T, K, dtype=f32, device=dev)
    else:
        n = c["n"] if c["op"] == "product" else 2 * c["inter"]
        s["x"], s["x_scale"] = _codes(c["T"], c["k"], 1.0, gen)
        s["w"], s["w_scale"] = _codes(n, c["k"], 0.02, gen)
        out = f32 if c.get("out") == "f32" else torch.bfloat16
        s["y"] = torch.empty(c["T"], n if c["op"] == "product" else c["inter"], dtype=out, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _plain_rows(p):
    """8-bit rows of p (fp64; the codes go by borders): codes, and the largest magnitude of each row."""
    big = p.abs().amax(1, keepdim=True)
    return torch.round(torch.where(big > 0, 127 * p / big, 0.0)), big[:, 0]


def _plain_norm(s, eps=1e-6):
    x = (s["x"].float() + s["delta"].float()).bfloat16()
    s["x"].copy_(x)
    v, w = x.float(), s["weight"].float()
    r = torch.rsqrt(v.square().mean(1) + eps)
    codes, big = _plain_rows((v * w).double())
    scale = torch.where(big > 0, big * r.double() / 127, 1.0).float()
    h = (v * w * r[:, None]).bfloat16() if s["case"]["h"] else None
    return dict(x=x, h=h, values=codes.float() * scale[:, None], scale=scale)


def _plain_route(s):
    c = s["case"]
    T, N, K, G = c["T"], c["N"], c["K"], c["groups"]
    l = s["logits"].double()
    if c["score"] == "softmax":
        e = (l - l.amax(1, keepdim=True)).exp()
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1 / (1 + (-l).exp())
    worth = score if s["bias"] is None else score + s["bias"].double()
    key = l if s["bias"] is None else worth      # without a bias the scores are in the order of the logits
    if G > 1:
        if c["pair"]:
            of = worth.view(T, G, N // G).sort(dim=2, descending=True).values[:, :, :2].sum(2)
        else:
            of = key.view(T, G, N // G).amax(2)
        best = of.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros(T, G, dtype=torch.bool, device=l.device).scatter_(1, best, True)
        key = torch.where(keep.repeat_interleave(N // G, 1), key, -torch.inf)
    idx = key.sort(dim=1, descending=True, stable=True).indices[:, :K]
    gate = score.gather(1, idx)
    if c["norm"]:
        gate = gate / gate.sum(1, keepdim=True)
    return dict(idx=idx.int(), gate=(gate * c["scale"]).float())


def _run_plain(s):
    c = s["case"]
    if c["op"] == "norm":
        return _plain_norm(s)
    if c["op"] == "rows":
        codes, big = _plain_rows(s["w"].double())
        scale = torch.where(big > 0, big / 127, 1.0).float()
        return dict(values=codes.float() * scale[:, None], scale=scale)
    if c["op"] == "route":
        return _plain_route(s)
    y = (s["x"].float() @ s["w"].float().T) * s["x_scale"][:, None] * s["w_scale"]
    if c["op"] == "product":
        return y.to(s["y"].dtype)
    g, u = y[:, :c["inter"]], y[:, c["inter"]:]
    return (g / (1 + (-g).exp()) * u).bfloat16()


def _run_own(s):
    from paper_2608_21240_b200 import binding as B
    c = s["case"]
    if c["op"] == "norm":
        B.spice_residual_rmsnorm(s["x"], s["weight"], 1e-6, s["q"], s["scale"], h=s["h"], delta=s["delta"])
        return dict(x=s["x"], h=s["h"], values=s["q"] * s["scale"][:, None], scale=s["scale"])
    if c["op"] == "rows":
        B.spice_quantize_i8_rows(s["w"], s["q"], s["scale"])
        return dict(values=s["q"] * s["scale"][:, None], scale=s["scale"])
    if c["op"] == "route":
        B.spice_route_scored(s["logits"], s["idx"], s["gate"], bias=s["bias"],
                             score=B.SCORE_SOFTMAX if c["score"] == "softmax" else B.SCORE_SIGMOID, n_groups=c["groups"],
                             top_groups=c["top_groups"], group_score=B.GROUP_TOP2 if c["pair"] else B.GROUP_MAX,
                             norm_topk=c["norm"], scale=c["scale"])
        return dict(idx=s["idx"], gate=s["gate"])
    if c["op"] == "product":
        B.spice_gemm_i8(s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"])
    else:
        B.spice_swiglu_i8(s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"])
    return s["y"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "norm":
        per = 2 + (2 if c["delta"] == "bf16" else 4) + 2 + (2 if c["h"] else 0) + 1
        return dict(bytes=c["T"] * c["d"] * per + 2 * c["d"] + 4 * c["T"], flops=8 * c["T"] * c["d"])
    if c["op"] == "rows":
        return dict(bytes=c["rows"] * c["cols"] * 3 + 4 * c["rows"], flops=3 * c["rows"] * c["cols"])
    if c["op"] == "route":
        return dict(bytes=4 * c["T"] * c["N"] + 8 * c["T"] * c["K"] + (4 * c["N"] if c["bias"] else 0),
                    flops=6 * c["T"] * c["N"])
    n = c["n"] if c["op"] == "product" else 2 * c["inter"]
    out = c["T"] * n * (4 if c["out"] == "f32" else 2) if c["op"] == "product" else c["T"] * c["inter"] * 2
    return dict(bytes=c["T"] * c["k"] + n * c["k"] + 4 * (c["T"] + n) + out, flops=2 * c["T"] * n * c["k"])


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _to_bf16_grid(v):
    """fp64 values at the nearest value with 8 significant bits, ties to even."""
    m, e = torch.frexp(v)
    return torch.ldexp(torch.round(m * 256), e - 8)


def _exact_codes(p):
    values, scale = [], []
    for part in p.split(8192):
        top = torch.maximum(part.amax(1), -part.amin(1)).unsqueeze(1)
        step = torch.where(top == 0, torch.ones_like(top), top / 127)
        values.append(torch.round(part * 127 / torch.where(top == 0, torch.ones_like(top), top)) * step)
        scale.append(step[:, 0])
    return torch.cat(values), torch.cat(scale)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "norm":
        x = _to_bf16_grid(s["x"].double() + s["delta"].double())
        p = x * s["weight"].double()
        rms = torch.sqrt((x * x).sum(1) / c["d"] + 1e-6)
        values, scale = _exact_codes(p)
        zero = (p == 0).all(1)
        r = torch.where(zero, torch.ones_like(rms), 1 / rms)
        return dict(x=x, h=p / rms[:, None] if c["h"] else None, values=values * r[:, None], scale=scale * r)
    if c["op"] == "rows":
        values, scale = _exact_codes(s["w"].double())
        return dict(values=values, scale=scale)
    if c["op"] == "route":
        return _exact_route(s)
    xs, ws = s["x_scale"].double(), s["w_scale"].double()
    x, w = s["x"].double(), s["w"].double()
    if c["op"] == "product":
        return torch.mm(x, w.T).mul_(xs[:, None]).mul_(ws[None, :])
    gate = torch.mm(x, w[:c["inter"]].T).mul_(xs[:, None]).mul_(ws[None, :c["inter"]])
    up = torch.mm(x, w[c["inter"]:].T).mul_(xs[:, None]).mul_(ws[None, c["inter"]:])
    return torch.sigmoid(gate).mul_(gate).mul_(up)


def _exact_route(s):
    """One winner at a time: the best expert left among the groups that stay."""
    c = s["case"]
    l, N, size = s["logits"].double(), c["N"], c["N"] // c["groups"]
    T = l.shape[0]
    score = torch.softmax(l, 1) if c["score"] == "softmax" else torch.sigmoid(l)
    value = score + (0 if s["bias"] is None else s["bias"].double())
    rows = torch.arange(T, device=l.device)
    order = value if s["bias"] is not None else l
    open_ = torch.ones(T, N, dtype=torch.bool, device=l.device)
    if c["groups"] > 1:
        if c["pair"]:
            top = value.view(T, c["groups"], size).topk(min(2, size), dim=2).values.sum(2)
        else:
            top = torch.stack([order[:, g * size:(g + 1) * size].max(1).values for g in range(c["groups"])], 1)
        open_[:] = False
        for _ in range(c["top_groups"]):
            g = (top == top.max(1, keepdim=True).values).int().argmax(1)
            top[rows, g] = -math.inf
            open_.view(T, c["groups"], size)[rows, g] = True
    left = torch.where(open_, order, torch.full_like(order, -math.inf))
    idx = []
    for _ in range(c["K"]):
        e = (left == left.max(1, keepdim=True).values).int().argmax(1)
        left[rows, e] = -math.inf
        idx.append(e)
    idx = torch.stack(idx, 1)
    gate = torch.stack([score[rows, idx[:, k]] for k in range(c["K"])], 1)
    if c["norm"]:
        gate = gate / gate.sum(1, keepdim=True)
    return dict(idx=idx.int(), gate=gate * c["scale"])
