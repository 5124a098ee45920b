"""spice_residual_rmsnorm and spice_quantize_i8_rows against their definitions in 64 bits.  Codes are exact by definition
(127 p / m to the nearest, ties to even, p a product of bf16 values) and have to be equal; so has the stream.

Tolerances: r = 1 / sqrt(sum / d + eps) in fp32: a thread adds at most 64 squares in turn, then two shuffle trees of 5 steps:
(64 + 10) half steps of 2^-24 on the sum, half of that on r, and 6 more roundings (square, quotient, root, reciprocal, the two
products of the scale): (37 + 6) 2^-24 < 3e-6 relative.  h is rounded once more, by at most 2^-8."""
import numpy as np
import pytest
import torch

from paper_2608_21240_b200 import binding as B

pytestmark = pytest.mark.gpu

R_RTOL = 3e-6
bf, f32 = torch.bfloat16, torch.float32


def codes64(p):
    """codes of the rows of p (fp64 numpy, exactly known) and their largest magnitudes."""
    m = np.abs(p).max(1, keepdims=True)
    ok = np.isfinite(p).all(1, keepdims=True)
    with np.errstate(all="ignore"):
        q = np.where(ok & (m > 0), np.rint(127 * p / m), 0)
    return q.astype(np.int8), m[:, 0], ok[:, 0]


def d64(t):
    return t.double().cpu().numpy()


def check_norm(x, delta, weight, eps, want_h=True, want_q=True):
    T, d = x.shape
    pad = 3                                         # rows behind the last one stay as they are
    h = torch.full((T + pad, d), 7.0, dtype=bf, device="cuda")
    q = torch.full((T + pad, d), 77, dtype=torch.int8, device="cuda")
    s = torch.full((T + pad,), 7.0, device="cuda")
    xs = torch.full((T + pad, d), 7.0, dtype=bf, device="cuda")
    xs[:T] = x
    B.spice_residual_rmsnorm(xs[:T], weight, eps, q[:T] if want_q else None, s[:T] if want_q else None,
                             h=h[:T] if want_h else None, delta=delta)
    torch.cuda.synchronize()
    stream = x if delta is None else (x.float() + delta.float()).to(bf)
    assert torch.equal(xs[:T].view(torch.int16), stream.view(torch.int16))
    assert (h[T:] == 7).all() and (q[T:] == 77).all() and (s[T:] == 7).all() and (xs[T:] == 7).all()
    v, w = d64(stream), d64(weight)
    with np.errstate(all="ignore"):
        p = v * w
        r = 1 / np.sqrt((v * v).mean(1) + eps)
    if want_q:
        cq, m, ok = codes64(p)
        assert np.array_equal(q[:T].cpu().numpy(), cq)
        got = d64(s[:T])
        assert np.isnan(got[~ok]).all()
        want = np.where(m > 0, m * r / 127, 1.0)[ok]
        assert (np.abs(got[ok] - want) <= R_RTOL * want).all()
    else:
        assert (q == 77).all() and (s == 7).all()
    if want_h:
        fine = np.isfinite(p).all(1)
        e = (p * r[:, None])[fine]
        assert (np.abs(d64(h[:T])[fine] - e) <= (2.0 ** -8 + R_RTOL) * np.abs(e) + 1e-38).all()
    else:
        assert (h == 7).all()
    return h[:T], q[:T], s[:T]


def draw(T, d, seed, delta="bf16"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, d, device="cuda", generator=g) * (1 + 20 * (torch.rand(d, device="cuda", generator=g) < 0.02))
    dl = torch.randn(T, d, device="cuda", generator=g)
    w = 1 + 0.2 * torch.randn(d, device="cuda", generator=g)
    return x.to(bf), None if delta is None else dl.to(bf if delta == "bf16" else f32), w.to(bf)


@pytest.mark.parametrize("T,d,delta", [(1, 8, "bf16"), (2, 64, None), (5, 256, "f32"), (9, 264, "bf16"), (33, 520, "f32"),
                                       (3, 2048, "bf16"), (7, 3584, "f32"), (1, 4104, "bf16"), (2, 8200, None), (2, 8192, "f32"),
                                       (2, 16392, "bf16"), (1, 32768, "f32"), (2500, 72, "bf16"), (1201, 2816, "bf16")])
def test_norm_matches_its_definition(T, d, delta):
    check_norm(*draw(T, d, T * 7 + d, delta), 1e-6)


@pytest.mark.parametrize("want_h,want_q", [(True, False), (False, True)])
@pytest.mark.parametrize("d", [128, 2048, 20480])
def test_norm_with_one_output(want_h, want_q, d):
    check_norm(*draw(5, d, d), 1e-5, want_h, want_q)


def test_norm_codes_at_their_borders():
    """Rows whose quotients lie on k + 1/2 and one step of bf16 beside it: m = 127 and p = k + 1/2 tie; factors of two and
    weights move m and p through the binades."""
    rows, weights = [], torch.ones(256, dtype=bf, device="cuda")
    weights[::3] = -2.0
    k = torch.arange(0, 120, device="cuda", dtype=f32) + 0.5
    for scale in (1.0, 2.0 ** -100, 2.0 ** 90, 3.0, 7.0 / 127):
        row = torch.zeros(256, device="cuda")
        row[1:121] = k * scale
        row[121] = 127 * scale
        rows += [row, row * (1 + 2 ** -7), row * (1 - 2 ** -8), -row]
    for step in (1, -1):                            # neighbours of the ties among the bf16 values
        r = rows[0].to(bf).view(torch.int16).clone()
        r[1:121] += step
        rows.append(r.view(bf).float())
    x = torch.stack(rows).to(bf)
    one = torch.ones(256, dtype=bf, device="cuda")
    check_norm(x, None, one, 0.0)
    check_norm(x, None, weights, 1e-6)


def test_norm_of_special_rows():
    """Zeros (codes 0, scale 1), squares beyond fp32, tiny values, and values that are not finite."""
    x, _, w = draw(9, 384, 5, None)
    x[0] = 0
    x[1] = 0
    x[1, 17] = -3e-38
    x[2] *= 1e25
    x[3, 4] = float("inf")
    x[4, 300] = float("nan")
    x[5] = torch.finfo(bf).min
    x[6] *= 2.0 ** -60
    x[7, 3] = -float("inf")
    h, q, s = check_norm(x, None, torch.ones_like(w), 1e-6)
    assert float(s[0]) == 1.0 and (q[0] == 0).all() and (h[0] == 0).all() and (q[5] == -127).all()
    assert torch.isnan(s[[3, 4, 7]]).all() and (q[[3, 4, 7]] == 0).all() and torch.isnan(h[4]).all()
    # 1 / sqrt(infinity) = 0: the finite values of such a row become 0, the infinite one NaN
    for row, at in ((3, 4), (7, 3)):
        assert torch.isnan(h[row, at]) and (h[row, torch.arange(384, device="cuda") != at] == 0).all()
    y, _, _ = draw(2, 2048, 6, None)                # the same over several warps
    y[0] *= 1e25
    check_norm(y, None, torch.ones(2048, dtype=bf, device="cuda"), 1e-6)


@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 72), (40, 512), (333, 2816), (2, 20480), (1, 32768), (5000, 24), (2, 4104)])
def test_quantise_rows(rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    w = (torch.randn(rows, cols, device="cuda", generator=g) * 10 ** torch.randint(-30, 30, (rows, 1), device="cuda", generator=g)).to(bf)
    if rows > 2:
        w[1] = 0
        w[2, cols // 2] = float("nan")
    q = torch.full((rows + 2, cols), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows + 2,), 7.0, device="cuda")
    B.spice_quantize_i8_rows(w, q[:rows], s[:rows])
    torch.cuda.synchronize()
    cq, m, ok = codes64(d64(w))
    assert np.array_equal(q[:rows].cpu().numpy(), cq) and (q[rows:] == 77).all() and (s[rows:] == 7).all()
    want, got = np.where(m > 0, m / 127, 1.0), d64(s[:rows])
    # m r (1 / 127): the constant's rounding and one product
    assert np.isnan(got[~ok]).all() and (np.abs(got - want)[ok] <= 2 * 2.0 ** -24 * want[ok] + 1e-45).all()


def test_every_pair_of_bf16_significands_is_rounded_exactly():
    """All 128 significands of the largest value against all values of three binades below it: 127 p / m for every pair."""
    m = (128 + torch.arange(128, device="cuda", dtype=f32)) * 2.0 ** 8
    v = torch.cat([(128 + torch.arange(128, device="cuda", dtype=f32)) * 2.0 ** e for e in (0, 3, 5, 6, 7)])
    w = torch.zeros(128, 648, device="cuda")
    w[:, :640] = torch.where(v[None] < m[:, None], v[None], 0)
    w[:, 640] = m
    w = w.to(bf)
    q, s = torch.empty(w.shape, dtype=torch.int8, device="cuda"), torch.empty(128, device="cuda")
    B.spice_quantize_i8_rows(w, q, s)
    torch.cuda.synchronize()
    assert np.array_equal(q.cpu().numpy(), codes64(d64(w))[0])


def test_empty_calls_other_streams_and_graphs():
    x, delta, w = draw(6, 2048, 11, "f32")
    e = torch.empty
    B.spice_residual_rmsnorm(x[:0], w, 1e-6, e(0, 2048, dtype=torch.int8, device="cuda"), e(0, device="cuda"))
    B.spice_quantize_i8_rows(x[:0], e(0, 2048, dtype=torch.int8, device="cuda"), e(0, device="cuda"))
    ref_x, ref = x.clone(), (torch.empty_like(x, dtype=torch.int8), e(6, device="cuda"), torch.empty_like(x))
    B.spice_residual_rmsnorm(ref_x, w, 1e-6, ref[0], ref[1], h=ref[2], delta=delta)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got_x, got = x.clone(), [torch.zeros_like(t) for t in ref]
    side.wait_stream(torch.cuda.current_stream())
    B.spice_residual_rmsnorm(got_x, w, 1e-6, got[0], got[1], h=got[2], delta=delta, stream=side)
    side.synchronize()
    assert torch.equal(got_x, ref_x) and all(torch.equal(a, b) for a, b in zip(got, ref))
    got_x.copy_(x)
    for t in got:
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.spice_residual_rmsnorm(got_x, w, 1e-6, got[0], got[1], h=got[2], delta=delta)
        B.spice_quantize_i8_rows(got[2], got[0], got[1])
    assert not got[1].any()
    for _ in range(2):
        got_x.copy_(x)
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got_x, ref_x) and torch.equal(got[2], ref[2])
    q, m, _ = codes64(d64(ref[2]))
    assert np.array_equal(got[0].cpu().numpy(), q)


def test_refusals_on_tensors():
    x, delta, w = draw(4, 64, 3)
    q, s = torch.empty(4, 64, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    for args, kw in (((x, w, 1e-6, q, None), {}), ((x, w, 1e-6), {}), ((x, w[:32], 1e-6, q, s), {}), ((x, w, 1e-6, q[:3], s), {}),
                     ((x, w, 1e-6, q, s), dict(delta=delta[:3])), ((x, w, 1e-6, q, s), dict(delta=delta.half())),
                     ((x.t(), w, 1e-6, q, s), {}), ((x, w.float(), 1e-6, q, s), {}), ((x, w, -1.0, q, s), {}),
                     ((x, w.cpu(), 1e-6, q, s), {})):
        with pytest.raises(B.SpiceError):
            B.spice_residual_rmsnorm(*args, **kw)
    flat = torch.zeros(4 * 64 + 8, dtype=bf, device="cuda")
    with pytest.raises(B.SpiceError, match="invalid"):
        B.spice_residual_rmsnorm(flat[4:4 + 256].view(4, 64), w, 1e-6, q, s)      # 8-byte aligned rows
    with pytest.raises(B.SpiceError):
        B.spice_quantize_i8_rows(x, q[:, :32], s)


def test_norm_of_products_beyond_fp32():
    """Squares beyond fp32 and one product that is, too (the codes are 0 and the scale NaN then): h is what the formula gives,
    in every column."""
    for d in (384, 2048, 20480):
        x, _, w = draw(4, d, d, None)
        x[:3] *= 1e25
        x[:3, 7] = 2e25
        w[7] = 1e15
        h, q = torch.empty_like(x), torch.full((4, d), 77, dtype=torch.int8, device="cuda")
        s = torch.zeros(4, device="cuda")
        B.spice_residual_rmsnorm(x, w, 1e-6, q, s, h=h)
        torch.cuda.synchronize()
        assert torch.isnan(s[:3]).all() and (q[:3] == 0).all() and float(s[3]) > 0 and int(q[3].abs().max()) == 127
        v = x.double()
        e = v * w.double() / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()
        assert ((h.double() - e).abs() <= (2.0 ** -8 + R_RTOL) * e.abs()).all()


@pytest.mark.parametrize("T,d,delta", [(5, 72, None), (3, 384, "bf16"), (4, 512, "f32"), (6, 2048, None), (3, 4104, "f32"),
                                       (2, 8200, "bf16"), (2, 20480, None)])
def test_norm_of_products_below_fp32(T, d, delta):
    """Products at and below the smallest numbers of fp32 and above 2^100: the codes stay those of the exact products, a row
    whose products are all below the range included."""
    for e_x, e_w in ((-74, -64), (-60, -64), (-90, -70), (-40, -100), (58, 58), (-100, 20)):
        x, dl, w = draw(T, d, T + d, delta)
        x, w = x * 2.0 ** e_x, w * 2.0 ** e_w
        if dl is not None:
            dl = dl * 2.0 ** e_x
        if T > 3:
            x[1] = 0
            if dl is not None:
                dl[1] = 0
        check_norm(x, dl, w, 0.0 if T <= 3 else 1e-30)
    # a row that has values only where the weight is 0
    x, _, w = draw(T, d, 3, None)
    w[::2] = 0
    x[:, 1::2] = 0
    check_norm(x, None, w, 1e-6)


@pytest.mark.parametrize("d", [72, 512, 2048, 20480])
def test_rows_of_zeros_between_others(d):
    """Rows that fill up a batch: codes 0, scale 1, h a zero of the product's sign; an infinite weight makes them NaN."""
    x, _, w = draw(6, d, d, None)
    x[1] = 0
    x[3] = -0.0
    x[5, ::2], x[5, 1::2] = 0, -0.0
    w[::3] *= -1
    h, q, s = check_norm(x, None, w, 1e-6)
    for r in (1, 3, 5):
        assert torch.equal(h[r].view(torch.int16), (x[r].float() * w.float()).to(bf).view(torch.int16))
        assert float(s[r]) == 1.0 and (q[r] == 0).all()
    w[5] = float("inf")
    h, q, s = torch.empty_like(x), torch.full((6, d), 77, dtype=torch.int8, device="cuda"), torch.zeros(6, device="cuda")
    B.spice_residual_rmsnorm(x, w, 1e-6, q, s, h=h)
    torch.cuda.synchronize()
    assert torch.isnan(s).all() and (q == 0).all() and torch.isnan(h[[1, 3, 5], 5]).all()
    assert torch.isinf(h[[0, 2, 4], 5]).all() and torch.isfinite(h[:, :5]).all()


@pytest.mark.parametrize("rows,cols", [(1100, 520), (1030, 2816), (1024, 8200), (1024, 16384), (3, 12296), (1050, 18000)])
def test_quantise_many_rows_and_wide_ones(rows, cols):
    """As above at 1024 rows and more, where a thread holds four vectors of a block's row, and at two vectors of one."""
    test_quantise_rows(rows, cols)
