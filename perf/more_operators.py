"""Timed cases of the experts' path around a router: tokens sorted by expert and brought back with their weights, the
gradient of that, and products of 8-bit floats with a scale for each block of 128 over the sorted rows.

`run` computes a case in elementary torch operations, or, where `own` is true, through the library's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3, LARGEST = torch.float8_e4m3fn, 448.0


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # interactive decoding, half of the experts resident: the kept entries of one token, with its bf16 row
        dict(name="sort 1x6 of 32", op="sort", T=1, K=6, N=64, S=32, d=2048, kind="bf16"),
        # a prefill batch whose 8-bit rows and scales go to all experts
        dict(name="sort 4096x6 of 64", op="sort", T=4096, K=6, N=64, S=64, d=2048, kind="e4m3"),
        # a decode batch of the wider layer, brought back into an fp32 sum
        dict(name="combine 17x8x3584", op="combine", T=17, K=8, N=64, S=24, d=3584, rows="bf16", out="f32", gates=True),
        # the gradient of the gather of a prefill batch: the same without weights
        dict(name="combine 4096x6x2048", op="combine", T=4096, K=6, N=64, S=64, d=2048, rows="bf16", out="bf16", gates=False),
        # backward pass of the weighted sum: a small ragged batch in fp32, and a training batch
        dict(name="gradient 61x8x3584", op="gradient", T=61, K=8, N=64, S=64, d=3584, rows="f32", dy="f32"),
        dict(name="gradient 4096x6x2048", op="gradient", T=4096, K=6, N=64, S=64, d=2048, rows="bf16", dy="bf16"),
        # hidden states of a ragged batch in front of the experts
        dict(name="blocks 333x2048", op="blocks", rows=333, cols=2048, square=False),
        # the down projections of all experts, quantised when they are loaded
        dict(name="blocks 64x2048x1408", op="blocks", rows=131072, cols=1408, square=True),
        # the wide shared expert's down projection for an odd decode batch, as fp32 rows that others are added to
        dict(name="product 77x3584x20480", op="product", R=77, G=0, skew=0.0, n=3584, k=20480, out="f32"),
        # the down projections of a prefill batch, unevenly spread over the experts
        dict(name="product 24576x2048x1408", op="product", R=24576, G=64, skew=0.6, n=2048, k=1408, out="bf16"),
        # gate and up products of a decode batch of 16 tokens: a row or two for each expert
        dict(name="swiglu 96x1408x2048", op="swiglu", R=96, G=64, skew=0.6, inter=1408, k=2048),
        # the same of a prefill batch
        dict(name="swiglu 24576x1408x2048", op="swiglu", R=24576, G=64, skew=0.6, inter=1408, k=2048),
    ]


def _spread(rng, low, high, step=1):
    """A multiple of `step` between low and high, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(low, min(high, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["sort", "combine", "gradient", "blocks", "product", "swiglu"])
    if op == "blocks":
        return dict(op=op, rows=_spread(rng, 1, 16384), cols=_spread(rng, 64, 8192, 16), square=rng.random() < 0.4)
    if op in ("sort", "combine", "gradient"):
        N, d = _spread(rng, 8, 256), _spread(rng, 64, 8192, 16)
        K, T = rng.randint(1, min(8, N)), _spread(rng, 1, 8192)
        while T * K * d > 4096 * 6 * 2048:
            T = max(1, T // 2)
        c = dict(op=op, T=T, K=K, N=N, S=rng.choice([N, max(1, N // 2)]), d=d)
        if op == "sort":
            return dict(c, kind=rng.choice(["bf16", "e4m3"]))
        if op == "combine":
            return dict(c, rows=rng.choice(["bf16", "bf16", "f32"]), out=rng.choice(["bf16", "f32"]), gates=rng.random() < 0.7)
        kind = rng.choice(["bf16", "bf16", "f32"])
        return dict(c, rows=kind, dy=kind)
    G = rng.choice([0, 0, 8, 64, _spread(rng, 2, 128)])
    R, k = _spread(rng, 1, 24576), _spread(rng, 64, 8192, 16)
    n = _spread(rng, 128, 4096, 128) if op == "swiglu" else _spread(rng, 64, 8192, 8)
    rows = n * (2 if op == "swiglu" else 1)
    while R * rows * k > 24576 * 2816 * 2048:
        R = max(1, R // 2)
    while max(G, 1) * rows * k > 64 * 2816 * 2048:
        G //= 2
    c = dict(op=op, R=R, G=G, skew=rng.choice([0.0, 0.6, 1.2]) if G else 0.0, k=k)
    return dict(c, inter=n) if op == "swiglu" else dict(c, n=n, out=rng.choice(["bf16", "f32"]))


# ------------------------------------------------------------------------------------------------ inputs
def _blocks(n):
    return (n + 127) // 128


def _sizes(c):
    """Rows of each group, largest first: what a router whose favourites are `skew` apart hands out."""
    G, R = max(c["G"], 1), c["R"]
    p = [(g + 1) ** -c["skew"] for g in range(G)]
    total, run, last, out = sum(p), 0.0, 0, []
    for v in p:
        run += v
        at = min(R, round(run / total * R))
        out.append(at - last)
        last = at
    out[-1] += R - last
    return out


def _quantised(w, square):
    """E4M3 codes (as bytes) and scales of the blocks of w [..., rows, cols]."""
    r, c = w.shape[-2:]
    pr, pc = (-r % 128 if square else 0), -c % 128
    p = torch.nn.functional.pad(w, (0, pc, 0, pr))
    p = p.view(*w.shape[:-2], (r + pr) // (128 if square else 1), 128 if square else 1, (c + pc) // 128, 128)
    scale = p.abs().amax((-3, -1)).clamp_min(1e-30) / LARGEST
    q = (p / scale[..., :, None, :, None]).view(*w.shape[:-2], r + pr, c + pc)[..., :r, :c]
    return q.to(E4M3).contiguous().view(torch.uint8), scale.contiguous()


def _routed(c, s, gen):
    """idx [T,K]: the slots of the K favourites of each token, -1 where an expert has none."""
    T, K, N, S, dev = c["T"], c["K"], c["N"], c["S"], "cuda"
    rand = lambda *n: torch.randn(*n, device=dev, generator=gen)  # noqa: E731
    logits = rand(T, N) + 0.7 * rand(N)
    best = logits.topk(K, 1)
    slot = torch.full((N,), -1, dtype=torch.int32, device=dev)
    slot[torch.randperm(N, device=dev, generator=gen)[:S]] = torch.arange(S, dtype=torch.int32, device=dev)
    s["idx"] = slot[best.indices].contiguous()
    s["gate"] = torch.softmax(best.values, 1).contiguous()


def _sorted(idx, S):
    """offset, pos, entry of a stable sort by slot."""
    n = idx.numel()
    flat = idx.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < S), flat, S)
    got = key.sort(stable=True)
    kept = got.values < S
    at = torch.arange(n, device=idx.device)
    entry = torch.where(kept, got.indices, -1)
    pos = torch.empty_like(at).scatter_(0, got.indices, torch.where(kept, at, -1))
    ends = (key[:, None] < torch.arange(S + 1, device=idx.device)).sum(0) if n * S < 1 << 22 else torch.searchsorted(
        got.values, torch.arange(S + 1, device=idx.device))
    return ends.int(), pos.view_as(idx).int(), entry.int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c, dev, f32, bf, i32 = case, "cuda", torch.float32, torch.bfloat16, torch.int32
    randn = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
    types = dict(bf16=bf, f32=f32)
    s = dict(case=c)
    if c["op"] in ("sort", "combine", "gradient"):
        T, K, d = c["T"], c["K"], c["d"]
        _routed(c, s, gen)
        if c["op"] == "sort":
            s["offset"] = torch.empty(c["S"] + 1, dtype=i32, device=dev)
            s["pos"], s["entry"] = torch.empty(T, K, dtype=i32, device=dev), torch.empty(T * K, dtype=i32, device=dev)
            if c["kind"] == "bf16":
                s["x"] = randn(T, d).to(bf)
                s["rows"] = torch.zeros(T * K, d, dtype=bf, device=dev)
            else:
                s["x"], s["x_scale"] = _quantised(randn(T, d), False)
                s["rows"] = torch.zeros(T * K, d, dtype=torch.uint8, device=dev)
                s["rows_scale"] = torch.zeros(T * K, _blocks(d), dtype=f32, device=dev)
            return s
        s["offset"], s["pos"], s["entry"] = _sorted(s["idx"], c["S"])
        s["rows"] = randn(T * K, d).to(types[c["rows"]])
        if c["op"] == "combine":
            s["y"] = torch.empty(T, d, dtype=types[c["out"]], device=dev)
            if not c["gates"]:
                s["gate"] = None
        else:
            s["dy"] = randn(T, d).to(types[c["dy"]])
            s["d_rows"] = torch.zeros(T * K, d, dtype=types[c["rows"]], device=dev)
            s["d_gate"] = torch.empty(T, K, dtype=f32, device=dev)
    elif c["op"] == "blocks":
        rows, cols = c["rows"], c["cols"]
        s["w"] = randn(rows, cols).mul_(0.02).to(bf)
        s["q"] = torch.empty(rows, cols, dtype=torch.uint8, device=dev)
        s["scale"] = torch.empty(_blocks(rows) if c["square"] else rows, _blocks(cols), dtype=f32, device=dev)
    else:
        n = c["n"] if c["op"] == "product" else 2 * c["inter"]
        R, G, k = c["R"], c["G"], c["k"]
        s["x"], s["x_scale"] = _quantised(randn(R, k), False)
        s["w"], s["w_scale"] = _quantised(randn(max(G, 1), n, k).mul_(0.02), True)
        order = torch.randperm(max(G, 1), generator=torch.Generator().manual_seed(seed)).tolist()
        sizes = _sizes(c)
        s["sizes"] = [sizes[g] for g in order]
        if G:
            s["offset"] = torch.tensor([0] + s["sizes"], dtype=i32, device=dev).cumsum(0).to(i32)
        else:
            s["offset"], s["w"], s["w_scale"] = None, s["w"][0], s["w_scale"][0]
        if c["op"] == "product":
            s["y"] = torch.empty(R, n, dtype=types[c["out"]], device=dev)
        else:
            s["act"] = torch.empty(R, c["inter"], dtype=torch.uint8, device=dev)
            s["act_scale"] = torch.empty(R, _blocks(c["inter"]), dtype=f32, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _plain_sort(s):
    c = s["case"]
    offset, pos, entry = _sorted(s["idx"], c["S"])
    kept, token = (entry >= 0)[:, None], (entry.clamp_min(0) // c["K"]).long()
    rows = torch.where(kept, s["x"][token], 0)
    out = dict(offset=offset, pos=pos, entry=entry, rows=rows if c["kind"] == "bf16" else rows.view(E4M3))
    if c["kind"] == "e4m3":
        out["rows_scale"] = torch.where(kept, s["x_scale"][token], 0.0)
    return out


def _taken(s):
    """The fp32 rows of each token's entries [T,K,d], zeros for those that were dropped."""
    pos = s["pos"].long()
    return torch.where((pos >= 0)[..., None], s["rows"][pos.clamp_min(0)].float(), 0.0)


def _plain_blocks(v, square):
    """E4M3 codes and scales of v (fp64; the codes go by borders)."""
    r, c = v.shape
    pr, pc = (-r % 128 if square else 0), -c % 128
    p = torch.nn.functional.pad(v, (0, pc, 0, pr)).view((r + pr) // (128 if square else 1), -1, (c + pc) // 128, 128)
    big = p.abs().amax((1, 3))
    u = torch.where(big[:, None, :, None] > 0, p * LARGEST / big[:, None, :, None], 0.0).view(r + pr, c + pc)[:r, :c]
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)   # codes have four significant bits
    q = (torch.round(u / step) * step).float().to(E4M3)
    return q, torch.where(big > 0, big / LARGEST, 1.0).float()


def _plain_product(s):
    k, n = s["x"].shape[1], s["w"].shape[-2]
    x = s["x"].view(E4M3).float() * s["x_scale"].repeat_interleave(128, 1)[:, :k]
    y = torch.empty(x.shape[0], n, device=x.device)
    w_all, scales = s["w"].view(-1, n, k), s["w_scale"].view(-1, _blocks(n), _blocks(k))
    at = 0
    for g, m in enumerate(s["sizes"]):
        if m:
            scale = scales[g].repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
            torch.mm(x[at:at + m], (w_all[g].view(E4M3).float() * scale).T, out=y[at:at + m])
            at += m
    return y


def _run_plain(s):
    c = s["case"]
    if c["op"] == "sort":
        return _plain_sort(s)
    if c["op"] == "combine":
        v = _taken(s)
        return ((v if s["gate"] is None else v * s["gate"][..., None]).sum(1)).to(s["y"].dtype)
    if c["op"] == "gradient":
        dy, entry = s["dy"].float(), s["entry"].long()
        weight = torch.where(entry >= 0, s["gate"].reshape(-1)[entry.clamp_min(0)], 0.0)
        d_rows = (dy[entry.clamp_min(0) // c["K"]] * weight[:, None]).to(s["d_rows"].dtype)
        return dict(d_rows=d_rows, d_gate=(_taken(s) * dy[:, None]).sum(2))
    if c["op"] == "blocks":
        q, scale = _plain_blocks(s["w"].double(), c["square"])
        return dict(q=q, scale=scale)
    y = _plain_product(s)
    if c["op"] == "product":
        return y.to(s["y"].dtype)
    g, u = y[:, :c["inter"]], y[:, c["inter"]:]
    q, scale = _plain_blocks((g / (1 + (-g).exp()) * u).double(), False)
    return dict(q=q, scale=scale)


def _run_own(s):
    from paper_2608_21240_b200 import binding as B
    c = s["case"]
    if c["op"] == "sort":
        B.spice_sort_tokens(s["idx"], s["offset"], s["pos"], s["entry"], x=s["x"], rows=s["rows"], x_scale=s.get("x_scale"),
                            rows_scale=s.get("rows_scale"))
        out = dict(offset=s["offset"], pos=s["pos"], entry=s["entry"], rows=s["rows"] if c["kind"] == "bf16" else s["rows"].view(E4M3))
        if c["kind"] == "e4m3":
            out["rows_scale"] = s["rows_scale"]
        return out
    if c["op"] == "combine":
        B.spice_combine_tokens(s["rows"], s["pos"], s["y"], gate=s["gate"])
        return s["y"]
    if c["op"] == "gradient":
        B.spice_combine_tokens_grad(s["dy"], s["rows"], s["pos"], s["gate"], s["d_rows"], s["d_gate"])
        return dict(d_rows=s["d_rows"], d_gate=s["d_gate"])
    if c["op"] == "blocks":
        B.spice_quantize_e4m3_blocks(s["w"], s["q"], s["scale"], block_rows=128 if c["square"] else 1)
        return dict(q=s["q"].view(E4M3), scale=s["scale"])
    if c["op"] == "product":
        B.spice_gemm_e4m3_blocks(s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"], offset=s["offset"])
        return s["y"]
    B.spice_swiglu_e4m3_blocks(s["x"], s["x_scale"], s["w"], s["w_scale"], s["act"], s["act_scale"], offset=s["offset"])
    return dict(q=s["act"].view(E4M3), scale=s["act_scale"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] in ("sort", "combine", "gradient"):
        T, K, d = c["T"], c["K"], c["d"]
        kept = T * K * c["S"] // c["N"]            # (as many as are resident, on average)
        if c["op"] == "sort":
            row = 2 * d if c["kind"] == "bf16" else d + 4 * _blocks(d)
            return dict(bytes=12 * T * K + 4 * (c["S"] + 1) + (min(T, kept) + kept) * row, flops=0)
        size = 2 if c["rows"] == "bf16" else 4
        if c["op"] == "combine":
            return dict(bytes=kept * d * size + T * K * (8 if c["gates"] else 4) + T * d * (2 if c["out"] == "bf16" else 4),
                        flops=2 * kept * d)
        return dict(bytes=2 * kept * d * size + T * d * (2 if c["dy"] == "bf16" else 4) + 12 * T * K, flops=3 * kept * d)
    if c["op"] == "blocks":
        return dict(bytes=3 * c["rows"] * c["cols"] + 4 * _blocks(c["cols"]) * (_blocks(c["rows"]) if c["square"] else c["rows"]),
                    flops=3 * c["rows"] * c["cols"])
    R, k = c["R"], c["k"]
    n = c["n"] if c["op"] == "product" else 2 * c["inter"]
    used = sum(1 for m in _sizes(c) if m)
    out = R * n * (4 if c["out"] == "f32" else 2) if c["op"] == "product" else R * (c["inter"] + 4 * _blocks(c["inter"]))
    return dict(bytes=R * (k + 4 * _blocks(k)) + used * (n * k + 4 * _blocks(n) * _blocks(k)) + out, flops=2 * R * n * k)


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _exact_codes(v, square):
    """Code values and scales of v's blocks, by the exponents of the quotients."""
    r, c = v.shape
    tall = 128 if square else 1
    scale = v.new_empty(-(-r // tall), _blocks(c))
    u = torch.empty_like(v)
    for b in range(_blocks(c)):
        part = v[:, b * 128:(b + 1) * 128]
        high = torch.maximum(part.amax(1), -part.amin(1))
        if square:
            high = torch.cat([high, high.new_zeros(-r % 128)]).view(-1, 128).amax(1)
        scale[:, b] = torch.where(high == 0, torch.ones_like(high), high / LARGEST)
        high = high.repeat_interleave(tall)[:r, None]
        u[:, b * 128:(b + 1) * 128] = torch.where(high == 0, torch.zeros_like(part), LARGEST * part / high)
    m, e = torch.frexp(u)
    fine = torch.ldexp(torch.round(m * 16), e - 4)           # four significant bits
    low = torch.round(u * 512) / 512                         # the evenly spaced ones next to zero
    return torch.where(u.abs() < 2.0 ** -6, low, fine), scale


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "sort":
        flat = s["idx"].reshape(-1)                          # one expert after the other
        found = [(flat == e).nonzero()[:, 0] for e in range(c["S"])]
        ends = torch.tensor([0] + [f.numel() for f in found], device="cuda").cumsum(0)
        found = torch.cat(found)
        pos, entry = torch.full_like(flat, -1), torch.full_like(flat, -1)
        pos[found] = torch.arange(found.numel(), dtype=torch.int32, device="cuda")
        entry[:found.numel()] = found.int()
        x = s["x"] if c["kind"] == "bf16" else s["x"].view(E4M3)
        rows = torch.zeros(flat.numel(), c["d"], dtype=torch.float64, device="cuda")
        rows[:found.numel()] = x.double()[found // c["K"]]
        out = dict(offset=ends.int(), pos=pos.view_as(s["idx"]), entry=entry, rows=rows)
        if c["kind"] == "e4m3":
            out["rows_scale"] = s["rows_scale"].double()
            out["rows_scale"][:found.numel()] = s["x_scale"].double()[found // c["K"]]
        return out
    if c["op"] == "combine":
        y = torch.zeros(c["T"], c["d"], dtype=torch.float64, device="cuda")
        for k in range(c["K"]):
            p = s["pos"][:, k].long()
            some = p >= 0
            part = s["rows"][p[some]].double()
            y[some] += part if s["gate"] is None else part * s["gate"][some, k].double()[:, None]
        return y
    if c["op"] == "gradient":
        d_rows = torch.zeros(c["T"] * c["K"], c["d"], dtype=torch.float64, device="cuda")
        d_gate = torch.zeros(c["T"], c["K"], dtype=torch.float64, device="cuda")
        for k in range(c["K"]):
            p = s["pos"][:, k].long()
            some = p >= 0
            dy = s["dy"][some].double()
            d_rows[p[some]] = dy * s["gate"][some, k].double()[:, None]
            d_gate[some, k] = torch.linalg.vecdot(dy, s["rows"][p[some]].double())
        return dict(d_rows=d_rows, d_gate=d_gate)
    if c["op"] == "blocks":
        q, scale = _exact_codes(s["w"].double(), c["square"])
        return dict(q=q, scale=scale)
    k, n = s["x"].shape[1], s["w"].shape[-2]
    x = s["x"].view(E4M3).double()
    xs = s["x_scale"].double()
    y = torch.empty(x.shape[0], n, dtype=torch.float64, device="cuda")
    at = 0
    for g, m in enumerate(s["sizes"]):
        w = (s["w"] if s["w"].dim() == 2 else s["w"][g]).view(E4M3).double()
        ws = (s["w_scale"] if s["w"].dim() == 2 else s["w_scale"][g]).double()
        for b in range(_blocks(k)):                          # block after block: scales outside of the sums
            w[:, b * 128:(b + 1) * 128] *= ws[:, b].repeat_interleave(128)[:n, None]
        y[at:at + m] = torch.mm(x[at:at + m] * xs[at:at + m].repeat_interleave(128, 1)[:, :k], w.T)
        at += m
    if c["op"] == "product":
        return y
    g, u = y[:, :c["inter"]], y[:, c["inter"]:]
    q, scale = _exact_codes(torch.sigmoid(g) * g * u, False)
    return dict(q=q, scale=scale)
