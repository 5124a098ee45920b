"""The steps next to the layer as a decode or prefill step uses them, two layers in a row: residual addition and norm, router
logits, routing by scores, classification, resident experts in bf16, the shared expert in 8-bit integers added to their sum,
whose fp32 rows are the next norm's residual.  Against a 64-bit evaluation of the same definitions.

Tolerance: the outputs' own of the layer's parity tests, 1e-2 max |reference| + 1e-3.  What separates the two: bf16 h and
activations (2^-8 each), 8-bit codes of activations whose bf16 value falls on the other side of a border (one step of
m / 127 in few of them), all relative to sums of hundreds of terms."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2608_21240_b200 import binding as B
from paper_2608_21240_b200 import workloads as W
from tests._gpu import cfg_of, upload, y_close

pytestmark = pytest.mark.gpu
f64 = torch.float64


def codes64(p):
    m = p.abs().amax(1, keepdim=True)
    return torch.round(127 * p / m) * m / 127


def silu_acts(x, gate_up):
    g, u = (x @ gate_up.T).chunk(2, 1)
    return g / (1 + (-g).exp()) * u


def silu_ffn(x, gate_up, down):
    return silu_acts(x, gate_up) @ down.T


def one_layer(L, w, w8, x, delta, weight, conf, bias, route):
    """One step through the library; x is updated.  Returns the fp32 output rows and what the routing chose."""
    T, d, K = x.shape[0], x.shape[1], L.cfg.top_k
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    h, q, s = e(T, d, t=torch.bfloat16), e(T, d, t=torch.int8), e(T)
    B.spice_residual_rmsnorm(x, weight, 1e-6, q, s, h=h, delta=delta)
    _, _, logits = L.route_topk(h, w.w_router, want_logits=True)
    idx, gate = e(T, K, t=torch.int32), e(T, K)
    B.spice_route_scored(logits, idx, gate, bias=bias, **route)
    cls, slot, counts, _ = L.classify_misses(idx, gate, w.slot_of_expert, conf)
    y = torch.zeros(T, d, device="cuda")
    L.grouped_expert_ffn(w, h, idx, gate, cls, slot, y)
    B.shared_expert_i8(w8, q, s, y, accumulate=True)
    return y, h, logits, idx, gate, cls, slot


@pytest.mark.parametrize("T", [1, 7, 300])
def test_two_layers_in_a_row(T):
    wl = W.make_layer("tiny", T, variant=70)
    s = wl.shape
    L = B.SpiceLayer(cfg_of(s), T)
    w = upload(wl)
    w8 = B.quantize_shared_i8(w)
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    x, weight, bias = rnd(T, s.d).bfloat16(), (1 + 0.1 * rnd(s.d)).bfloat16(), 0.05 * rnd(s.n_experts)
    conf = torch.from_numpy(wl.conf).cuda()
    route = dict(score=B.SCORE_SIGMOID, n_groups=4, top_groups=2, group_score=B.GROUP_TOP2, norm_topk=True, scale=2.5)
    wgu, wd = codes64(w.shared_w_gate_up.to(f64)), codes64(w.shared_w_down.to(f64))
    delta = None
    for layer in range(2):
        before = x.clone()
        y, h, logits, idx, gate, cls, slot = one_layer(L, w, w8, x, delta, weight, conf, bias, route)
        torch.cuda.synchronize()
        # the norm
        stream = before if delta is None else (before.float() + delta).bfloat16()
        assert torch.equal(x, stream)
        p = x.to(f64) * weight.to(f64)
        r = 1 / (x.to(f64).square().mean(1, keepdim=True) + 1e-6).sqrt()
        assert ((h.to(f64) - p * r).abs() <= (2.0 ** -8 + 3e-6) * (p * r).abs()).all()
        # the routing of the logits that the library computed
        sc = 1 / (1 + (-logits.to(f64)).exp())
        key = sc + bias.to(f64)
        G = s.n_experts // 4
        of = key.view(T, 4, G).sort(dim=2, descending=True).values[:, :, :2].sum(2)
        keep = torch.zeros_like(of, dtype=torch.bool).scatter_(1, of.sort(dim=1, descending=True, stable=True).indices[:, :2], True)
        key = torch.where(keep.repeat_interleave(G, 1), key, -torch.inf)
        ri = key.sort(dim=1, descending=True, stable=True).indices[:, :s.top_k]
        assert torch.equal(idx.long(), ri)
        rg = sc.gather(1, ri)
        rg = 2.5 * rg / rg.sum(1, keepdim=True)
        assert ((gate - rg).abs() <= 1.1e-5 * rg).all()
        res = w.slot_of_expert.long()[ri]
        assert torch.equal(cls == B.HIT, res >= 0) and torch.equal(slot.long(), res)
        # the experts: resident ones in bf16, the shared one in 8 bits
        a = silu_acts(codes64(p) * r, wgu)
        ref = codes64(a.bfloat16().to(f64)) @ wd.T
        for k in range(s.top_k):
            for sl in range(s.n_slots):
                rows = (res[:, k] == sl).nonzero()[:, 0]
                if len(rows):
                    ref[rows] += rg[rows, k:k + 1] * silu_ffn(h[rows].to(f64), w.slot_w_gate_up[sl].to(f64), w.slot_w_down[sl].to(f64))
        err, bound = y_close(y.cpu().numpy(), ref.cpu().numpy())
        assert err <= bound, (layer, err, bound)
        delta = y
    assert L.device_status() == 0
    L.close()


def test_a_captured_step_replays():
    """The same chain in one graph, replayed on changed inputs, gives what the separate calls give."""
    T = 5
    wl = W.make_layer("tiny", T, variant=71)
    s = wl.shape
    L = B.SpiceLayer(cfg_of(s), T)
    w = upload(wl)
    w8 = B.quantize_shared_i8(w)
    weight, conf = torch.ones(s.d, dtype=torch.bfloat16, device="cuda"), torch.from_numpy(wl.conf).cuda()
    bias = torch.zeros(s.n_experts, device="cuda")
    x, delta = torch.randn(T, s.d, device="cuda").bfloat16(), torch.randn(T, s.d, device="cuda")
    keep = x.clone()
    one_layer(L, w, w8, x, delta, weight, conf, bias, {})
    torch.cuda.synchronize()
    x.copy_(keep)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = one_layer(L, w, w8, x, delta, weight, conf, bias, {})[0]
    for i in range(3):
        fresh = torch.randn(T, s.d, device="cuda").bfloat16()
        x.copy_(fresh)
        graph.replay()
        got, gx = y.clone(), x.clone()
        x2 = fresh.clone()
        ref = one_layer(L, w, w8, x2, delta, weight, conf, bias, {})[0]
        assert torch.equal(gx, x2)
        # (the routed experts' rows are added in the order of the batch: bitwise equal)
        assert torch.equal(got, ref)
    L.close()


def test_products_beside_the_fused_layer_on_another_stream():
    """The fused decode layer on one stream and 8-bit products of several sizes on another, many times over: each gives what
    it gives alone."""
    T = 16
    wl = W.make_layer("dsv2lite", T, variant=72)
    s = wl.shape
    L = B.SpiceLayer(cfg_of(s), T)
    dev = "cuda"
    rnd = lambda *shape: (torch.randn(*shape, device=dev) * 0.02).bfloat16()  # noqa: E731
    w = B.LayerWeights(rnd(s.n_experts, s.d), rnd(s.n_slots, 2 * s.inter, s.d), rnd(s.n_slots, s.d, s.inter),
                       torch.from_numpy(wl.slot_of_expert.copy()).to(dev), rnd(2 * s.inter_shared, s.d), rnd(s.d, s.inter_shared),
                       rnd(s.n_experts, s.lore_rank, s.d), rnd(s.n_experts, s.d, s.lore_rank))
    w8 = B.quantize_shared_i8(w)
    h, conf = torch.randn(T, s.d, device=dev).bfloat16(), torch.from_numpy(wl.conf).cuda()
    y_ref = L.moe_layer_fwd(w, h, conf).y.clone()
    batches, refs = [], []
    for n in (3, 40, 200, 700):
        x, q, sc = torch.randn(n, s.d, device=dev).bfloat16(), torch.empty(n, s.d, dtype=torch.int8, device=dev), torch.empty(n, device=dev)
        B.spice_quantize_i8_rows(x, q, sc)
        act, y = torch.empty(n, s.inter_shared, dtype=torch.bfloat16, device=dev), torch.empty(n, s.d, device=dev)
        B.spice_swiglu_i8(q, sc, w8.q_gate_up, w8.s_gate_up, act)
        B.spice_gemm_i8(q, sc, w8.q_gate_up[:s.d].contiguous(), w8.s_gate_up[:s.d].contiguous(), y)
        batches.append((q, sc, act, y))
        refs.append((act.clone(), y.clone()))
    wq, ws = w8.q_gate_up[:s.d].contiguous(), w8.s_gate_up[:s.d].contiguous()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for i in range(60):
        outs.append(L.moe_layer_fwd(w, h, conf, stream=one).y)
        for q, sc, act, y in batches:
            B.spice_swiglu_i8(q, sc, w8.q_gate_up, w8.s_gate_up, act, stream=two)
            B.spice_gemm_i8(q, sc, wq, ws, y, stream=two)
    torch.cuda.synchronize()
    assert L.device_status() == 0
    assert all(torch.equal(y, y_ref) for y in outs)
    for (_, _, act, y), (ra, ry) in zip(batches, refs):
        assert torch.equal(act, ra) and torch.equal(y, ry)
    L.close()


FIRST = """
import torch
from paper_2608_21240_b200 import binding as B
dev, bf, i8 = "cuda", torch.bfloat16, torch.int8
x, w = torch.randn(300, 512, device=dev).to(bf), torch.ones(512, device=dev, dtype=bf)
q, s = torch.zeros(300, 512, device=dev, dtype=i8), torch.zeros(300, device=dev)
wq, ws = torch.randint(-127, 128, (64, 512), device=dev).to(i8), torch.rand(64, device=dev)
ys = [torch.zeros(T, 64, device=dev, dtype=bf) for T in (1, 40, 300)]
act = torch.zeros(300, 32, device=dev, dtype=bf)
lg, idx, gate = torch.randn(5, 64, device=dev), torch.zeros(5, 6, device=dev, dtype=torch.int32), torch.zeros(5, 6, device=dev)
def step():
    B.spice_residual_rmsnorm(x, w, 1e-6, q, s)
    for y in ys:
        T = y.shape[0]
        B.spice_gemm_i8(q[:T], s[:T], wq, ws, y)
    B.spice_swiglu_i8(q, s, wq, ws, act)
    B.spice_route_scored(lg, idx, gate)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (q, s, *ys, act, idx, gate)]
assert all(bool(t.float().abs().sum() > 0) for t in got)
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (q, s, *ys, act, idx, gate)))
print("captured")
"""


def test_the_first_calls_of_a_process_may_be_captured():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("T", [1, 7, 300])
@pytest.mark.parametrize("tau", [0.0, 0.5])
def test_layers_with_and_without_low_confidence_misses(tau, T):
    """The layer's formula, routed by scores: y = (1 + sum of the LOWCONF gates) S(h) + sum over HIT of g E(h) + sum over LOWCONF
    of g B A h.  Without such misses S(h) is the shared expert in 8-bit integers, with them the call for the surrogate."""
    wl = W.make_layer("tiny", T, variant=73)
    s = wl.shape
    L = B.SpiceLayer(cfg_of(s, tau=tau), T)
    w = upload(wl)
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    x, weight, bias = rnd(T, s.d).bfloat16(), (1 + 0.1 * rnd(s.d)).bfloat16(), 0.05 * rnd(s.n_experts)
    conf = torch.from_numpy(wl.conf).cuda()
    e = lambda *shape, t=torch.float32: torch.empty(*shape, dtype=t, device="cuda")  # noqa: E731
    h, q, sc = e(T, s.d, t=torch.bfloat16), e(T, s.d, t=torch.int8), e(T)
    B.spice_residual_rmsnorm(x, weight, 1e-6, q, sc, h=h)
    _, _, logits = L.route_topk(h, w.w_router, want_logits=True)
    idx, gate = e(T, s.top_k, t=torch.int32), e(T, s.top_k)
    B.spice_route_scored(logits, idx, gate, bias=bias, score=B.SCORE_SIGMOID, n_groups=4, top_groups=2, scale=2.5)
    cls, slot, counts, _ = L.classify_misses(idx, gate, w.slot_of_expert, conf)
    y = torch.zeros(T, s.d, device="cuda")
    L.grouped_expert_ffn(w, h, idx, gate, cls, slot, y)
    if tau == 0:
        B.shared_expert_i8(B.quantize_shared_i8(w), q, sc, y, accumulate=True)
    else:
        L.lore_surrogate(w, h, idx, gate, cls, y)
    torch.cuda.synchronize()
    low = cls == B.LOWCONF
    assert int(counts[2]) == int(low.sum()) and (int(low.sum()) > 0 if tau > 0 and T > 1 else tau > 0 or not low.any())
    h64, g64 = h.to(f64), gate.to(f64)
    if tau == 0:
        p = x.to(f64) * weight.to(f64)
        r = 1 / (x.to(f64).square().mean(1, keepdim=True) + 1e-6).sqrt()
        a = silu_acts(codes64(p) * r, codes64(w.shared_w_gate_up.to(f64)))
        shared = codes64(a.bfloat16().to(f64)) @ codes64(w.shared_w_down.to(f64)).T
    else:
        shared = silu_ffn(h64, w.shared_w_gate_up.to(f64), w.shared_w_down.to(f64))
    ref = shared * (1 + (g64 * low).sum(1, keepdim=True))
    for t in range(T):
        for k in range(s.top_k):
            ex = int(idx[t, k])
            if low[t, k]:
                ref[t] += g64[t, k] * (w.lore_B[ex].to(f64) @ (w.lore_A[ex].to(f64) @ h64[t]))
            elif cls[t, k] == B.HIT:
                sl = int(slot[t, k])
                ref[t] += g64[t, k] * silu_ffn(h64[t:t + 1], w.slot_w_gate_up[sl].to(f64), w.slot_w_down[sl].to(f64))[0]
    err, bound = y_close(y.cpu().numpy(), ref.cpu().numpy())
    assert err <= bound, (err, bound)
    assert L.device_status() == 0
    L.close()
