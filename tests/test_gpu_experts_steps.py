"""The experts' path step by step: SwiGLU over long reductions with sums that leave no choice of codes, and the whole chain with every
step's result held to its formula on that step's own inputs.

SwiGLU's tolerances are those of its formula (slack(k) of the sums, then (4 |g| + 16) 2^-24 for the fast exponential and quotient): the codes
have to be what some value within them gives.  Where operands are small integers times powers of two, every partial sum is below 2^24
units and exact in fp32 in any order, the sums' part is 0, and the interval holds a single code for all but a few values: its width
against a code's step, 2 (4 |g| + 32) 2^-24 / 2^-4, is below 1e-4 for |g| < 8."""
import pytest
import torch

from paper_2608_21240_b200 import binding as B
from tests.test_gpu_e4m3_blocks import E4M3, H16, H32, bf, compare, exact, f32, f64, i32, nearest, plain_quantiser, slack, split, u8
from tests.test_gpu_sort_tokens import plain_sort, taken

pytestmark = pytest.mark.gpu


def check_activations(q, s, e, d):
    """Codes q [T,inter] and scales s of activations whose gate and up products e [T, 2 inter] are known within d; returns the share of
    values that have a choice of codes."""
    T, inter = q.shape
    gt, up, dg, du = e[:, :inter], e[:, inter:], d[:, :inter], d[:, inter:]
    silu = gt * torch.sigmoid(gt)
    act = silu * up
    da = 1.1 * dg * up.abs() + silu.abs() * du + 1.1 * dg * du + act.abs() * (4 * gt.abs() + 16) * H32 + 1e-37
    big = lambda v: v.view(T, inter // 128, 128).amax(2)  # noqa: E731
    wide = lambda v: v.repeat_interleave(128, 1)  # noqa: E731
    m, dm = big(act.abs()), big(da)
    assert (m > 0).all()
    assert ((s.to(f64) - m / 448).abs() <= dm / 448 + 4 * H32 * m / 448).all()
    v = 448 * act / wide(m)
    dv = 448 * da / wide(m) + v.abs() * (wide(dm / m) * 1.01 + 8 * H32)
    got, low, high = q.view(E4M3).to(f64), nearest(v - dv), nearest(v + dv)
    assert ((low <= got) & (got <= high)).all()
    return float((low != high).double().mean())


def whole_numbers(T, inter, k, G, seed):
    """Operands that are small integers, scales that are powers of two of two sizes; gates of some units."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    code = lambda *s: torch.randint(-2, 3, s, device="cuda", generator=g).to(f32).to(E4M3).view(u8)  # noqa: E731
    kb = -(-k // 128)
    base = 2.0 ** -round(torch.tensor(float(k)).log2().item() / 4)
    power = lambda *s: base * 2.0 ** -torch.randint(0, 2, s, device="cuda", generator=g).to(f32)  # noqa: E731
    assert 4 * k * 4 < 2 ** 24                                    # units of a quarter of base^2
    return code(T, k), power(T, kb), code(G, 2 * inter, k), power(G, 2 * inter // 128, kb)


@pytest.mark.parametrize("T,inter,k,G", [(1, 128, 2048, 0), (9, 256, 8208, 0), (25, 128, 8208, 0), (32, 1408, 2048, 0), (40, 256, 8192, 0), (77, 384, 20480, 0),
                                         (130, 128, 16400, 0), (300, 128, 16400, 0), (1500, 256, 2048, 0), (24, 384, 8208, 16), (60, 256, 4112, 8),
                                         (700, 256, 8208, 5), (3000, 384, 1040, 24)])
def test_codes_of_exact_sums(T, inter, k, G):
    x, xs, w, ws = whole_numbers(T, inter, k, max(G, 1), T + inter + k)
    bounds = split(T, G, T) if G else [0, T]
    q, s = torch.full((T, inter), 0x55, dtype=u8, device="cuda"), torch.full((T, inter // 128), 3.0, device="cuda")
    off = torch.tensor(bounds, dtype=i32, device="cuda") if G else None
    B.spice_swiglu_e4m3_blocks(x, xs, w if G else w[0], ws if G else ws[0], q, s, off)
    torch.cuda.synchronize()
    e, _ = exact(x, xs, w, ws, bounds)
    e = e[bounds[0]:bounds[-1]]
    assert float(e.abs().max()) < 60
    assert check_activations(q[bounds[0]:bounds[-1]], s[bounds[0]:bounds[-1]], e, torch.zeros_like(e)) < 1e-3


@pytest.mark.parametrize("T", [1, 20, 300])
def test_gates_that_count_as_zero(T):
    """Gates of -100 under up products of 1e20: activations of 4e-22, where exp(100) is beyond fp32, count as 0.  A block of nothing else is a block of zeros; beside
    other gates they have codes of zero."""
    inter, k = 256, 128
    one, x = 0x38, torch.full((T, k), 0x38, dtype=u8, device="cuda")
    w = torch.full((2 * inter, k), one, dtype=u8, device="cuda")
    w[:inter] = one | 0x80                                        # -1
    w[128:256:3] = 0x08                                           # 2^-6
    ws = torch.tensor([[100 / 128], [100 / 128], [1e20 / 128], [1e20 / 128]], device="cuda")
    q, s = torch.full((T, inter), 0x55, dtype=u8, device="cuda"), torch.full((T, 2), 3.0, device="cuda")
    B.spice_swiglu_e4m3_blocks(x, torch.ones(T, 1, device="cuda"), w, ws, q, s)
    torch.cuda.synchronize()
    g = torch.tensor(100 / 64, dtype=f64)
    a = float(g * torch.sigmoid(g) * 1e20)
    v = q.view(E4M3).to(f64)
    assert (v[:, :128] == 0).all() and (s[:, 0] == 1).all()
    assert (v[:, 128::3] == 448).all() and (v[:, 129::3] == 0).all() and (v[:, 130::3] == 0).all()
    assert ((s[:, 1].to(f64) * 448 - a).abs() <= 32 * H32 * a).all()


@pytest.mark.parametrize("T,n,k,G", [(1, 264, 2048, 0), (8, 136, 4112, 0), (32, 520, 20480, 0), (77, 264, 20480, 0), (300, 136, 16400, 0), (24, 264, 8208, 16),
                                     (700, 264, 8208, 5)])
def test_products_of_exact_sums(T, n, k, G):
    """The same for products: fp32 results are equal to the exact ones."""
    x, xs, w, ws = whole_numbers(T, 128 * -(-n // 256), k, max(G, 1), T + n + k)
    w, ws = w[:, :n].contiguous(), ws[:, :-(-n // 128)].contiguous()
    bounds = split(T, G, T) if G else [0, T]
    y = torch.full((T, n), 3.0, device="cuda")
    off = torch.tensor(bounds, dtype=i32, device="cuda") if G else None
    B.spice_gemm_e4m3_blocks(x, xs, w if G else w[0], ws if G else ws[0], y, off)
    torch.cuda.synchronize()
    e, _ = exact(x, xs, w, ws, bounds)
    a, b = bounds[0], bounds[-1]
    assert torch.equal(y[a:b].to(f64), e[a:b])


@pytest.mark.parametrize("T,G,drop", [(1, 8, 0.0), (16, 16, 0.4), (90, 8, 0.2), (700, 16, 0.3)])
def test_every_step_of_the_chain(T, G, drop):
    d, K, I = 528, 4, 384
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(bf)  # noqa: E731
    h, gu, dn = rnd(T, d), rnd(G, 2 * I, d, std=0.04), rnd(G, d, I, std=0.05)
    idx = torch.rand(T, G, device="cuda", generator=g).argsort(1)[:, :K].to(i32)
    idx = torch.where(torch.rand(T, K, device="cuda", generator=g) < drop, -1, idx).contiguous()
    gate = torch.rand(T, K, device="cuda", generator=g)
    w = B.quantize_experts_e4m3(gu, dn)
    y = torch.full((T, d), 0.5, device="cuda")
    B.routed_experts_e4m3(w, h, idx, gate, y, accumulate=True)
    for t, q, s in ((gu, w.q_gate_up, w.s_gate_up), (dn, w.q_down, w.s_down)):
        eq, es = plain_quantiser(t, 128)
        assert torch.equal(q.view(E4M3).to(f64), eq) and ((s.to(f64) - es).abs() <= H32 * es).all()
    kb = -(-d // 128)
    q, s = torch.empty(T, d, dtype=u8, device="cuda"), torch.empty(T, kb, device="cuda")
    B.spice_quantize_e4m3_blocks(h, q, s)
    eq, es = plain_quantiser(h, 1)
    assert torch.equal(q.view(E4M3).to(f64), eq) and ((s.to(f64) - es).abs() <= H32 * es).all()
    off, pos, entry = (torch.empty(*n, dtype=i32, device="cuda") for n in ((G + 1,), (T, K), (T * K,)))
    rows, rs = torch.zeros(T * K, d, dtype=u8, device="cuda"), torch.zeros(T * K, kb, device="cuda")
    B.spice_sort_tokens(idx, off, pos, entry, q, rows, s, rs)
    for got, want in zip((off, pos, entry), plain_sort(idx, G)):
        assert torch.equal(got.cpu(), want)
    bounds = off.tolist()
    kept = bounds[-1]
    token = (entry[:kept] // K).long()
    assert torch.equal(rows[:kept], q[token]) and torch.equal(rs[:kept], s[token])
    act, acts = torch.zeros(T * K, I, dtype=u8, device="cuda"), torch.zeros(T * K, I // 128, device="cuda")
    B.spice_swiglu_e4m3_blocks(rows, rs, w.q_gate_up, w.s_gate_up, act, acts, off)
    e, A = exact(rows, rs, w.q_gate_up, w.s_gate_up, bounds)
    assert check_activations(act[:kept], acts[:kept], e[:kept], slack(d) * A[:kept]) < 0.1
    down = torch.zeros(T * K, d, dtype=bf, device="cuda")
    B.spice_gemm_e4m3_blocks(act, acts, w.q_down, w.s_down, down, off)
    e, A = exact(act, acts, w.q_down, w.s_down, bounds)
    compare(down[:kept], e[:kept], A[:kept], I, "bf16")
    parts = taken(down, pos) * gate.to(f64)[..., None]
    want, tol = parts.sum(1) + 0.5, K * H32 * parts.abs().sum(1)
    tol = tol + H32 * (want.abs() + tol)
    assert ((y.to(f64) - want).abs() <= tol * (1 + 1e-6)).all()   # (of the chain as a whole: the steps by themselves give the same bits)
    rounded = torch.empty(T, d, dtype=bf, device="cuda")
    B.routed_experts_e4m3(w, h, idx, gate, rounded)
    torch.cuda.synchronize()
    want = parts.sum(1)
    tol = K * H32 * parts.abs().sum(1)
    assert ((rounded.to(f64) - want).abs() <= (tol + H16 * (want.abs() + tol)) * (1 + 1e-6)).all()
