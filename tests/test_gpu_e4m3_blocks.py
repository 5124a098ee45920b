"""spice_quantize_e4m3_blocks, spice_gemm_e4m3_blocks and spice_swiglu_e4m3_blocks against their formulas in 64 bits.

Quantiser: codes are compared for equality (the formula leaves no choice), scales within half a step of fp32.

Products: a block's 128 products are added on the tensor cores in 4 steps of 32 terms (or in the same order by warp-wide ones).  With at
least 24 bits kept of every addend, aligned to the largest of a step, a step is off by at most (32 + 2) 2^-23 of sum |x w| over the
block, a block by 4 of those; its two scales are a rounding each, and the sum over kb blocks (and over 8 warps) makes kb + 8 roundings
of partial sums.  With A = sum |xs ws x w|: |error| <= (4 * 34 * 2 + kb + 10) 2^-24 A.  bf16 rounds once more (2^-8), adding to y too.

SwiGLU: with dg, du of that kind, |da| <= 1.1 dg |u| + |silu(g)| du + |a| (4 |g| + 16) 2^-24 (the fast exponential and quotient).  The codes
must be what some value within that of the exact 448 a / m gives: between the codes of the two ends of the interval."""
import pytest
import torch

from paper_2608_21240_b200 import binding as B

pytestmark = pytest.mark.gpu

bf, f32, f64, i32, u8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
E4M3 = torch.float8_e4m3fn
H32, H16 = 2.0 ** -24, 2.0 ** -8


def nearest(u):
    """The E4M3 value nearest to u (fp64), ties to even, saturating."""
    _, e = torch.frexp(u)
    step = torch.ldexp(torch.ones_like(u), torch.clamp(e - 4, min=-9))
    return (torch.round(u / step) * step).clamp(-448, 448)


def per_block(v, tall):
    """v [..., rows, cols] -> [..., row blocks, tall, column blocks, 128], filled up with zeros."""
    r, c = v.shape[-2:]
    p = torch.nn.functional.pad(v, (0, -c % 128, 0, -r % tall))
    return p.view(*v.shape[:-2], p.shape[-2] // tall, tall, p.shape[-1] // 128, 128)


def spread(scale, tall, r, c):
    return scale.repeat_interleave(tall, -2)[..., :r, :].repeat_interleave(128, -1)[..., :c]


def plain_quantiser(w, tall):
    r, c = w.shape[-2:]
    m = per_block(w.to(f64).abs(), tall).amax((-3, -1))
    finite = torch.isfinite(m)
    safe = torch.where(finite & (m > 0), m, 1.0)
    q = nearest(448 * torch.where(spread(finite & (m > 0), tall, r, c), w.to(f64), 0.0) / spread(safe, tall, r, c))
    scale = torch.where(m == 0, 1.0, m / 448)
    return q, torch.where(finite, scale, float("nan"))


def check_quantiser(w, tall):
    lead, (r, c) = w.shape[:-2], w.shape[-2:]
    q = torch.full((*lead, r, c), 0x55, dtype=u8, device="cuda")
    scale = torch.full((*lead, -(-r // tall), -(-c // 128)), -3.0, device="cuda")
    B.spice_quantize_e4m3_blocks(w, q, scale, tall)
    torch.cuda.synchronize()
    eq, es = plain_quantiser(w, tall)
    assert torch.equal(q.view(E4M3).to(f64), eq)
    assert torch.equal(torch.isnan(scale), torch.isnan(es))
    ok = ~torch.isnan(es)
    assert ((scale.to(f64) - es).abs()[ok] <= H32 * es[ok] + 2.0 ** -150).all()   # (half of fp32's smallest step for denormal scales)


@pytest.mark.parametrize("shape", [(1, 8), (1, 128), (3, 136), (16, 2048), (33, 1040), (129, 3584), (5, 20480), (4097, 264), (2, 130, 200), (3, 256, 128),
                                   (2, 1, 72), (1500, 1408)])
@pytest.mark.parametrize("tall", [1, 128])
def test_quantiser(shape, tall):
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    check_quantiser(torch.randn(*shape, device="cuda", generator=g).to(bf), tall)


@pytest.mark.parametrize("tall", [1, 128])
def test_quantiser_at_borders_and_at_the_ends_of_the_range(tall):
    """Every pair of significands as (value, largest value) of a block, at several distances of their exponents, from bf16's smallest
    numbers to its largest: all the quotients there are, ties among them."""
    sig = torch.arange(128, 256, device="cuda", dtype=f64)
    for top in (-126, -101, -100, -99, -10, 0, 50, 120):        # exponent of the largest: 2^top * [1, 2)
        v = torch.zeros(128, 16, 128, device="cuda", dtype=f64)   # [largest, distance, value]
        for i, dist in enumerate((0, 1, 2, 3, 4, 5, 7, 9, 10, 11, 12, 14, 15, 16, 17, 18)):
            v[:, i] = sig[None] * 2.0 ** (top - 7 - dist)
        v[:, 0] = torch.minimum(v[:, 0], sig[:, None] * 2.0 ** (top - 7))
        v[:, 1:, 0] = sig[:, None] * 2.0 ** (top - 7)
        v[:, ::2] *= -1
        w = v.view(2048, 128).to(f32).to(bf)
        check_quantiser(w if tall == 1 else w[::16].contiguous(), tall)
    tiny = torch.randint(-9, 10, (300, 256), device="cuda").to(f64) * 2.0 ** -133      # bf16's denormal numbers
    check_quantiser(tiny.to(f32).to(bf), tall)
    check_quantiser(torch.full((130, 256), 3.3e38, device="cuda").to(bf), tall)


@pytest.mark.parametrize("tall", [1, 128])
def test_quantiser_of_zeros_and_of_what_is_not_finite(tall):
    w = torch.randn(300, 400, device="cuda").to(bf)
    w[3] = 0
    w[128:256, 128:256] = 0
    w[10, 5] = float("nan")
    w[200, 399] = float("inf")
    w[299, 130] = -float("inf")
    w[50, 300] = -0.0
    check_quantiser(w, tall)


# ------------------------------------------------------------------------------------------------ products
def quantised(w, tall, seed=None):
    """Codes and scales of w, the scales with all their bits in use."""
    r, c = w.shape[-2:]
    m = per_block(w.abs(), tall).amax((-3, -1)).clamp_min(1e-20)
    scale = m / 448 * (1 + 1e-3)
    return (w / spread(scale, tall, r, c)).to(E4M3).contiguous().view(u8), scale.contiguous()


def operands(T, n, k, G, seed, std=0.03):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, k, device="cuda", generator=g) * (0.2 + torch.rand(T, 1, device="cuda", generator=g) * 3)
    w = torch.randn(max(G, 1), n, k, device="cuda", generator=g) * std
    w *= 0.1 + 2 * torch.rand(max(G, 1), n, 1, device="cuda", generator=g)
    return (*quantised(x, 1), *quantised(w, 128))


def values(x, xs, w, ws, tall=128):
    xv = x.view(E4M3).to(f64) * spread(xs.to(f64), 1, *x.shape)
    return xv, lambda i: w[i].view(E4M3).to(f64) * spread(ws[i].to(f64), tall, *w.shape[-2:])


def exact(x, xs, w, ws, bounds):
    """(product, sum of magnitudes) [T,n] in 64 bits; rows outside of the groups: zeros."""
    xv, wv = values(x, xs, w, ws)
    e = torch.zeros(x.shape[0], w.shape[-2], dtype=f64, device="cuda")
    A = torch.zeros_like(e)
    for i in range(len(bounds) - 1):
        a, b = bounds[i], bounds[i + 1]
        if b > a:
            v = wv(i)
            e[a:b], A[a:b] = xv[a:b] @ v.T, xv[a:b].abs() @ v.abs().T
    return e, A


def slack(k):
    return (4 * 34 * 2 + -(-k // 128) + 10) * H32


def split(T, G, seed, first=0, tail=0):
    """Offsets of G ragged groups over rows first .. T - tail, some of them empty."""
    g = torch.Generator().manual_seed(seed)
    cuts = torch.sort(torch.randint(first, T - tail + 1, (G - 1,), generator=g)).values.tolist() if G > 1 else []
    return [first, *cuts, T - tail]


def run(x, xs, w, ws, out="f32", bounds=None, pad=2, status=0):
    T, n = x.shape[0], w.shape[-2]
    y = torch.full((T + pad, n), 3.0, dtype=bf if out == "bf16" else f32, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    off = None if bounds is None else torch.tensor(bounds, dtype=i32, device="cuda")
    B.spice_gemm_e4m3_blocks(x, xs, w if bounds is not None else w[0], ws if bounds is not None else ws[0], y[:T], off, out == "add", st)
    torch.cuda.synchronize()
    assert int(st) == status and (y[T:] == 3).all()
    return y[:T]


def compare(y, e, A, k, out):
    tol = slack(k) * A
    if out == "bf16":
        tol = tol + H16 * (e.abs() + tol)
    if out == "add":
        e = e + 3
        tol = tol + H32 * (e.abs() + tol)
    err = (y.to(f64) - e).abs()
    assert (err <= tol * (1 + 1e-6)).all(), float((err / tol.clamp_min(1e-300)).max())


def check(T, n, k, out="f32", G=0, first=0, tail=0):
    x, xs, w, ws = operands(T, n, k, G, T + n + k + G)
    bounds = split(T, G, T + G, first, tail) if G else None
    y = run(x, xs, w, ws, out, bounds)
    e, A = exact(x, xs, w, ws, bounds or [0, T])
    a, b = (bounds[0], bounds[-1]) if G else (0, T)
    assert (y[:a] == 3).all() and (y[b:] == 3).all()
    compare(y[a:b], e[a:b], A[a:b], k, out)


DENSE = [(1, 8, 16), (1, 2048, 2816), (2, 72, 48), (3, 136, 144), (5, 264, 1040), (9, 3584, 528), (16, 128, 4096), (17, 8, 16), (17, 2048, 2816), (31, 72, 128),
         (33, 136, 400), (64, 3584, 1040), (77, 264, 20480), (128, 200, 256), (129, 512, 4096), (241, 72, 80), (256, 256, 128), (257, 264, 144),
         (300, 2048, 400), (513, 520, 1408), (1000, 128, 16), (1025, 2816, 272), (2600, 2056, 1040), (5000, 3592, 144)]


@pytest.mark.parametrize("T,n,k", DENSE)
def test_dense_product(T, n, k):
    check(T, n, k)


@pytest.mark.parametrize("T,n,k", [(1, 2048, 2816), (7, 136, 144), (77, 264, 1040), (257, 264, 144), (700, 520, 528), (77, 264, 8208), (30, 72, 8208)])
@pytest.mark.parametrize("out", ["bf16", "add"])
def test_other_outputs(T, n, k, out):
    check(T, n, k, out)
    check(T, n, k, out, G=5)


# (the largest rows a group: 16 rows and fewer on average stay in the kernel of few rows, whatever a group has)
@pytest.mark.parametrize("T,n,k,G,first,tail", [(1, 64, 128, 1, 0, 0), (1, 136, 256, 64, 0, 0), (6, 2048, 1408, 64, 0, 0), (40, 72, 144, 7, 3, 5),
                                                (96, 512, 528, 64, 0, 7), (300, 264, 272, 24, 0, 0), (500, 128, 64, 1000, 0, 0), (90, 8, 16, 5, 1, 1),
                                                (400, 264, 272, 3, 7, 9), (1000, 200, 1040, 40, 0, 0), (3000, 520, 400, 9, 1, 2), (5000, 2048, 1408, 64, 0, 100),
                                                (20000, 136, 144, 1000, 0, 0), (17000, 72, 48, 3, 0, 0)])
def test_grouped_product(T, n, k, G, first, tail):
    check(T, n, k, "f32", G, first, tail)


@pytest.mark.parametrize("T", [30, 800])
def test_groups_at_the_ends_and_all_rows_in_one(T):
    x, xs, w, ws = operands(T, 136, 272, 6, T)
    for bounds in ([0, 0, 0, T, T, T, T], [0] * 6 + [T], [0] + [T] * 6, [0, 1, 2, 3, 4, 5, T], [T] * 7, [0] * 7):
        y = run(x, xs, w, ws, "f32", bounds)
        e, A = exact(x, xs, w, ws, bounds)
        rows = torch.zeros(T, dtype=torch.bool, device="cuda")
        rows[bounds[0]:bounds[-1]] = True
        assert (y[~rows] == 3).all()
        compare(y[rows], e[rows], A[rows], 272, "f32")


# (up to eight tokens, on both sides of what is multiplied without a ring: 16 blocks of the reduction, 32 MiB of weights)
@pytest.mark.parametrize("T,n,k", [(1, 512, 1024), (8, 24, 4096), (5, 200, 2064), (8, 2056, 2064), (4, 40, 4112), (8, 264, 8208), (7, 8184, 4096),
                                   (8, 8200, 4096), (8, 24, 2048), (3, 2056, 2032), (7, 16384, 2048), (8, 16392, 2048), (8, 136, 1040), (2, 72, 16)])
@pytest.mark.parametrize("out", ["bf16", "f32", "add"])
def test_up_to_eight_tokens(T, n, k, out):
    check(T, n, k, out)


@pytest.mark.parametrize("n,k", [(136, 272), (72, 4096), (264, 5136)])
@pytest.mark.parametrize("bounds", [[0, 0, 0, 8, 8, 8, 8], [0] * 6 + [8], [0] + [8] * 6, [0, 1, 2, 3, 4, 5, 8], [2, 2, 3, 3, 5, 6, 6], [8] * 7, [0] * 7])
def test_up_to_eight_tokens_in_groups(n, k, bounds):
    x, xs, w, ws = operands(8, n, k, 6, n)
    y = run(x, xs, w, ws, "f32", bounds)
    e, A = exact(x, xs, w, ws, bounds)
    rows = torch.zeros(8, dtype=torch.bool, device="cuda")
    rows[bounds[0]:bounds[-1]] = True
    assert (y[~rows] == 3).all()
    compare(y[rows], e[rows], A[rows], k, "f32")


def test_up_to_eight_tokens_in_many_groups_and_bad_ones():
    T, n, k = 8, 136, 528
    x, xs, w, ws = operands(T, n, k, 1, 3)
    e, A = exact(x, xs, w, ws, [0, T])
    for G in (8, 40, 1024):
        many, scales = w.expand(G, -1, -1).contiguous(), ws.expand(G, -1, -1).contiguous()
        compare(run(x, xs, many, scales, "f32", split(T, G, G)), e, A, k, "f32")
        compare(run(x, xs, many, scales, "f32", [0, T] * (G // 2) + [T], status=5), e, A, k, "f32")   # more groups with rows than rows
        y = run(x, xs, many, scales, "f32", [0, 3, T + 1, 5] + [T] * (G - 3), status=5)
        compare(y[[0, 1, 2, 5, 6, 7]], e[[0, 1, 2, 5, 6, 7]], A[[0, 1, 2, 5, 6, 7]], k, "f32")
        assert (y[3:5] == 3).all()


@pytest.mark.parametrize("T", [30, 800])
def test_bad_offsets_are_reported_and_their_groups_left_out(T):
    x, xs, w, ws = operands(T, 72, 144, 4, T)
    # offsets, and the (group, first row, last row) that are nobody else's
    for bounds, good in (([0, 5, 3, 9, T], [(0, 0, 3), (2, 5, 9), (3, 9, T)]), ([-4, 5, 7, 9, T], [(1, 5, 7), (2, 7, 9), (3, 9, T)]),
                         ([0, 5, 7, 9, T + 1], [(0, 0, 5), (1, 5, 7), (2, 7, 9)]), ([0, 5, 2 ** 31 - 1, 9, T], [(0, 0, 5), (3, 9, T)])):
        y = run(x, xs, w, ws, "f32", bounds, status=5)            # SPICE_ERR_BAD_TABLE
        left = torch.ones(T, dtype=torch.bool, device="cuda")
        left[3:5] = bounds[2] != 3                                # (rows of two groups: either may have written them last)
        for i, a, b in good:
            e, A = exact(x, xs, w[i:i + 1], ws[i:i + 1], [a, b])
            compare(y[a:b], e[a:b], A[a:b], 144, "f32")
            left[a:b] = False
        assert (y[left] == 3).all()


def test_a_row_does_not_depend_on_its_place():
    """The same rows, dense and spread over groups with the same weights, in other orders: the same bits."""
    for T, G in ((48, 8), (600, 4)):
        x, xs, w, ws = operands(T, 264, 1040, 1, T)
        many, scales = w.expand(G, -1, -1).contiguous(), ws.expand(G, -1, -1).contiguous()
        a = run(x, xs, many, scales, "f32", split(T, G, 1))
        b = run(x, xs, many, scales, "f32", [0] * G + [T])
        order = torch.randperm(T, device="cuda")
        c = run(x[order].contiguous(), xs[order].contiguous(), many, scales, "f32", split(T, G, 2))
        assert torch.equal(a, b) and torch.equal(a[order], c)


@pytest.mark.parametrize("T,G", [(20, 4), (700, 4)])
def test_nan_stays_in_its_rows_and_groups(T, G):
    x, xs, w, ws = operands(T, 264, 400, G, T)
    bounds = [0, T // 4, T // 2, T // 2 + 3, T]
    clean = run(x, xs, w, ws, "f32", bounds).clone()
    x[2, 7] = 0x7f                                                # E4M3's NaN
    xs[T // 2 + 1, 1] = float("nan")
    ws[3, 1, 2] = float("inf")                                    # 128 columns of the last group
    y = run(x, xs, w, ws, "f32", bounds)
    odd = torch.zeros(T, 264, dtype=torch.bool, device="cuda")
    odd[2] = odd[T // 2 + 1] = True
    odd[bounds[3]:, 128:256] = True
    assert not torch.isfinite(y[odd]).any() and torch.equal(y[~odd], clean[~odd])


@pytest.mark.parametrize("T", [5, 300])
def test_scales_of_any_size_and_sign(T):
    """Scales far apart, of either sign and zero; the largest codes everywhere."""
    k, n = 1040, 200
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randint(0, 256, (T, k), device="cuda", generator=g).to(u8)
    w = torch.randint(0, 256, (1, n, k), device="cuda", generator=g).to(u8)
    x[(x & 0x7f) == 0x7f] = 0x7e
    w[(w & 0x7f) == 0x7f] = 0xfe
    xs = torch.randn(T, 9, device="cuda", generator=g) * 10.0 ** torch.randint(-9, 9, (T, 9), device="cuda", generator=g)
    ws = torch.randn(1, 2, 9, device="cuda", generator=g) * 10.0 ** torch.randint(-9, 9, (1, 2, 9), device="cuda", generator=g)
    xs[0, 3] = ws[0, 1, 4] = 0
    y = run(x, xs, w, ws)
    e, A = exact(x, xs, w, ws, [0, T])
    compare(y, e, A, k, "f32")


def test_weights_beyond_32_bits():
    """Groups that lie more than 2^32 bytes into the weights."""
    G, n, k = 70, 8192, 8192
    w = torch.zeros(G, n, k, dtype=u8, device="cuda")
    ws = torch.ones(G, 64, 64, device="cuda")
    for T in (70, 1400):
        x, xs, last, last_s = operands(T, n, k, 1, T)
        w[-1], ws[-1] = last[0], last_s[0]
        bounds = [0] * (G - 1) + [0 if T > 100 else 3, T]
        bounds = [0, *bounds][-(G + 1):]
        y = run(x, xs, w, ws, "f32", bounds)
        e, A = exact(x, xs, last, last_s, [bounds[-2], T])
        a = bounds[-2]
        compare(y[a:], e[a:], A[a:], k, "f32")


# ------------------------------------------------------------------------------------------------ SwiGLU
def check_swiglu(T, inter, k, G=0, first=0, tail=0, std=0.03):
    x, xs, w, ws = operands(T, 2 * inter, k, G, T + inter + k, std)
    bounds = split(T, G, T + G, first, tail) if G else None
    q = torch.full((T + 2, inter), 0x55, dtype=u8, device="cuda")
    s = torch.full((T + 2, inter // 128), 3.0, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    off = None if bounds is None else torch.tensor(bounds, dtype=i32, device="cuda")
    B.spice_swiglu_e4m3_blocks(x, xs, w if G else w[0], ws if G else ws[0], q[:T], s[:T], off, st)
    torch.cuda.synchronize()
    a, b = (bounds[0], bounds[-1]) if G else (0, T)
    assert int(st) == 0 and (q[:a] == 0x55).all() and (q[b:] == 0x55).all() and (s[:a] == 3).all() and (s[b:] == 3).all()
    e, A = exact(x, xs, w, ws, bounds or [0, T])
    e, A, q, s = e[a:b], A[a:b], q[a:b], s[a:b]
    gt, up, dg, du = e[:, :inter], e[:, inter:], slack(k) * A[:, :inter], slack(k) * A[:, inter:]
    silu = gt * torch.sigmoid(gt)
    act = silu * up
    da = 1.1 * dg * up.abs() + silu.abs() * du + 1.1 * dg * du + act.abs() * (4 * gt.abs() + 16) * H32 + 1e-37
    big = lambda v: v.view(b - a, inter // 128, 128).amax(2)  # noqa: E731
    m = big(act.abs())
    dm = big(da)                                                  # the largest value is off by no more than the largest error
    assert ((s.to(f64) - m / 448).abs() <= dm / 448 + 4 * H32 * m / 448).all()
    wide = lambda v: v.repeat_interleave(128, 1)  # noqa: E731
    u = 448 * act / wide(m)
    du = 448 * da / wide(m) + u.abs() * (wide(dm / m) * 1.01 + 8 * H32)
    got = q.view(E4M3).to(f64)
    low, high = nearest(u - du), nearest(u + du)
    assert ((low <= got) & (got <= high)).all()
    # The interval says something: most values have no choice.  (Its width against a code's step, 2 slack(k) A / |e| of each factor against
    # 2^-4 to 2^-3, grows with k: A / |e| like k^0.5, the worst case of the sums like k.  From k = 8208 on it is a percent and more for a
    # typical factor and ten times that for one in ten: there the check is that of the intervals above alone.)
    if k <= 4096:
        assert float((low != high).double().mean()) < 0.5


@pytest.mark.parametrize("T,inter,k", [(1, 128, 16), (1, 1408, 2048), (3, 256, 144), (8, 2816, 528), (16, 384, 1040), (17, 128, 48), (33, 256, 2048), (100, 640, 528),
                                       (256, 128, 144), (257, 384, 272), (513, 256, 1408), (1500, 1408, 256), (4000, 1408, 144),
                                       (40, 256, 8192), (300, 128, 16400), (25, 128, 8208)])
def test_swiglu(T, inter, k):
    check_swiglu(T, inter, k)


@pytest.mark.parametrize("T,inter,k,G,first,tail", [(1, 128, 128, 64, 0, 0), (6, 1408, 2048, 64, 0, 0), (40, 128, 144, 7, 3, 5), (96, 384, 528, 64, 0, 7),
                                                    (300, 256, 272, 24, 0, 0), (500, 128, 64, 1000, 0, 0), (400, 256, 272, 3, 7, 9), (1000, 256, 1040, 40, 0, 0),
                                                    (3000, 384, 400, 9, 1, 2), (5000, 1408, 2048, 64, 0, 100)])
def test_grouped_swiglu(T, inter, k, G, first, tail):
    check_swiglu(T, inter, k, G, first, tail)


@pytest.mark.parametrize("T", [9, 300])
def test_swiglu_of_large_gates(T):
    check_swiglu(T, 256, 512, std=0.2)                            # |g| of several ten


@pytest.mark.parametrize("T", [9, 300])
def test_swiglu_of_zeros_and_of_what_is_not_finite(T):
    inter, k = 256, 272
    x, xs, w, ws = operands(T, 2 * inter, k, 0, T)
    def call():
        q, s = torch.empty(T, inter, dtype=u8, device="cuda"), torch.empty(T, 2, device="cuda")
        B.spice_swiglu_e4m3_blocks(x, xs, w[0], ws[0], q, s)
        torch.cuda.synchronize()
        return q, s
    q0, s0 = call()
    x[1] = 0
    xs[2, 0] = float("inf")
    x[4, 9] = 0xff
    ws[0, 3, 1] = float("nan")                                    # up rows 128 ..: the second block of every token
    q, s = call()
    assert (q[1] == 0).all() and s[1, 0] == 1
    assert torch.isnan(s[2, 0]) and torch.isnan(s[4, 0]) and (q[2] == 0).all() and (q[4] == 0).all()
    assert torch.isnan(s[:, 1]).all() and (q[:, 128:] == 0).all()
    rest = torch.tensor([i for i in range(T) if i not in (1, 2, 4)], device="cuda")
    assert torch.equal(q[rest, :128], q0[rest, :128]) and torch.equal(s[rest, 0], s0[rest, 0])


# ------------------------------------------------------------------------------------------------ streams, limits, the chain
@pytest.mark.parametrize("T,G", [(12, 0), (96, 16), (400, 0), (1500, 16)])
def test_captured_calls_on_two_streams(T, G):
    """Two captured chains replayed on two streams at the same time, many times over: no workspace to share."""
    data = []
    for i in range(2):
        x, xs, w, ws = operands(T, 512, 1024 + 128 * i, G, i)
        off = torch.tensor(split(T, G, i), dtype=i32, device="cuda") if G else None
        w, ws = (w, ws) if G else (w[0], ws[0])
        y = torch.zeros(T, 512, dtype=bf, device="cuda")
        q, s = torch.zeros(T, 256, dtype=u8, device="cuda"), torch.zeros(T, 2, device="cuda")

        def chain(x=x, xs=xs, w=w, ws=ws, y=y, q=q, s=s, off=off):
            B.spice_gemm_e4m3_blocks(x, xs, w, ws, y, off)
            B.spice_swiglu_e4m3_blocks(x, xs, w, ws, q, s, off)
        chain()
        torch.cuda.synchronize()
        data.append((chain, (y, q, s), [v.clone() for v in (y, q, s)]))
    graphs = []
    for chain, outs, _ in data:
        for v in outs:
            v.zero_()
        torch.cuda.synchronize()
        st, gr = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            for _ in range(5):
                chain()
        graphs.append((st, gr))
    for _ in range(20):
        for st, gr in graphs:
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    for _, outs, want in data:
        for v, ref in zip(outs, want):
            assert torch.equal(v, ref)


@pytest.mark.parametrize("T,n,k,G", [(300, 512, 2048, 0), (700, 2048, 528, 0), (2600, 512, 528, 9), (64, 256, 8192, 0), (12, 512, 2048, 0), (96, 512, 528, 16)])
def test_expired_waits_are_reported(T, n, k, G):
    """With waits that give up at once, a call ends by itself, reports it, and writes nothing behind its rows; the next call is as
    always."""
    x, xs, w, ws = operands(T, n, k, G, 1)
    bounds = split(T, G, 1) if G else None
    off = torch.tensor(bounds, dtype=i32, device="cuda") if G else None
    w1, ws1 = (w, ws) if G else (w[0], ws[0])
    st = torch.zeros(2, dtype=i32, device="cuda")
    y = torch.full((T + 2, n), 3.0, device="cuda")
    q, s = torch.full((T + 2, n // 2), 3, dtype=u8, device="cuda"), torch.full((T + 2, n // 256), 3.0, device="cuda")
    torch.cuda.synchronize()
    B.spice_set_option(None, B.OPT_E4M3_WAIT_LIMIT, 0)
    try:
        B.spice_gemm_e4m3_blocks(x, xs, w1, ws1, y[:T], off, device_status=st[:1])
        B.spice_swiglu_e4m3_blocks(x, xs, w1, ws1, q[:T], s[:T], off, device_status=st[1:])
        torch.cuda.synchronize()
    finally:
        B.spice_set_option(None, B.OPT_E4M3_WAIT_LIMIT, 1 << 22)
    assert st.tolist() == [6, 6]                                  # SPICE_ERR_TIMEOUT
    assert (y[T:] == 3).all() and (q[T:] == 3).all() and (s[T:] == 3).all()
    e, A = exact(x, xs, w, ws, bounds or [0, T])
    compare(run(x, xs, w, ws, "f32", bounds), e, A, k, "f32")


def test_empty_batches_and_refusals_on_tensors():
    x, xs, w, ws = operands(4, 256, 144, 0, 1)
    w, ws = w[0], ws[0]
    y, q, s = torch.empty(4, 256, dtype=bf, device="cuda"), torch.empty(4, 128, dtype=u8, device="cuda"), torch.empty(4, 1, device="cuda")
    B.spice_gemm_e4m3_blocks(x[:0], xs[:0], w, ws, y[:0])
    B.spice_swiglu_e4m3_blocks(x[:0], xs[:0], w, ws, q[:0], s[:0])
    B.spice_quantize_e4m3_blocks(y[:0], torch.empty(0, 256, dtype=u8, device="cuda"), torch.empty(0, 2, device="cuda"))
    for args in ((x, xs, w, ws, y[:, :8]), (x, xs[:3], w, ws, y), (x, xs, w[:, :128], ws, y), (x, xs, w, ws, y.half()), (x.cpu(), xs, w, ws, y),
                 (x[:, :136].contiguous(), xs, w[:, :136].contiguous(), ws, y), (x.to(torch.int8), xs, w, ws, y)):
        with pytest.raises(B.SpiceError):
            B.spice_gemm_e4m3_blocks(*args)
    with pytest.raises(B.SpiceError):
        B.spice_swiglu_e4m3_blocks(x, xs, w[:144], ws, q, s)


@pytest.mark.parametrize("T,half", [(1, False), (16, True), (300, False), (1000, True)])
def test_experts_of_a_slot_pool(T, half):
    """The whole chain beside the layer's own calls: routing and classification by the library, the resident experts in E4M3 blocks, their
    weighted sum added to a sum that is there.  Every step's result is held to its formula on the step's own inputs; the whole to the
    layer's bf16 experts: with each of h, the three weights and the activation off by 2^-4 at most (scale and code), a term of the sums
    is off by less than (1 + 2^-4)^5 - 1 < 0.36 of its magnitude with gate and up products' magnitudes taken for theirs."""
    d, N, K, I, S = 512, 16, 4, 384, 8 if half else 16
    g = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).to(bf)  # noqa: E731
    h, gu, dn, wr = rnd(T, d), rnd(S, 2 * I, d, std=0.04), rnd(S, d, I, std=0.05), rnd(N, d, std=0.1)
    slot_of = torch.full((N,), -1, dtype=i32, device="cuda")
    slot_of[torch.randperm(N, device="cuda", generator=g)[:S]] = torch.arange(S, dtype=i32, device="cuda")
    layer = B.SpiceLayer(B.make_cfg(d, N, K, I, 128, 8, S, 0.0), T)
    idx, gate = layer.route_topk(h, wr)
    cls, slot, counts, _ = layer.classify_misses(idx, gate, slot_of, torch.ones(T, N, device="cuda"))
    w = B.quantize_experts_e4m3(gu, dn)
    y = torch.full((T, d), 0.5, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    B.routed_experts_e4m3(w, h, slot, gate, y, accumulate=True, device_status=st)
    torch.cuda.synchronize()
    assert int(st) == 0 and int(counts[0]) == int((slot >= 0).sum())
    layer.close()
    # the steps by themselves give the same bits
    q, s = torch.empty(T, d, dtype=u8, device="cuda"), torch.empty(T, d // 128, device="cuda")
    B.spice_quantize_e4m3_blocks(h, q, s)
    off, pos, entry = (torch.empty(*n, dtype=i32, device="cuda") for n in ((S + 1,), (T, K), (T * K,)))
    rows, rs = torch.zeros(T * K, d, dtype=u8, device="cuda"), torch.zeros(T * K, d // 128, device="cuda")
    B.spice_sort_tokens(slot, off, pos, entry, q, rows, s, rs)
    act, acts = torch.zeros(T * K, I, dtype=u8, device="cuda"), torch.zeros(T * K, I // 128, device="cuda")
    B.spice_swiglu_e4m3_blocks(rows, rs, w.q_gate_up, w.s_gate_up, act, acts, off)
    down = torch.zeros(T * K, d, dtype=bf, device="cuda")
    B.spice_gemm_e4m3_blocks(act, acts, w.q_down, w.s_down, down, off)
    again = torch.full((T, d), 0.5, device="cuda")
    B.spice_combine_tokens(down, pos, again, gate, accumulate=True)
    torch.cuda.synchronize()
    assert torch.equal(again, y)
    bounds = off.tolist()
    e, A = exact(act, acts, w.q_down, w.s_down, bounds)
    kept = bounds[-1]
    compare(down[:kept], e[:kept], A[:kept], I, "bf16")
    # the layer's formula on the bf16 weights
    want, most = torch.zeros(T, d, dtype=f64, device="cuda"), torch.zeros(T, d, dtype=f64, device="cuda")
    for t in range(T):
        for k in range(K):
            e = int(slot[t, k])
            if e < 0:
                continue
            hv, W, D, wt = h[t].to(f64), gu[e].to(f64), dn[e].to(f64), float(gate[t, k])
            p = W @ hv
            a = p[:I] * torch.sigmoid(p[:I]) * p[I:]
            pa = W.abs() @ hv.abs()
            want[t] += wt * (D @ a)
            most[t] += wt * (D.abs() @ (1.1 * pa[:I] * pa[I:]))
    assert ((y.to(f64) - 0.5 - want).abs() <= 0.36 * most + 1e-3).all()
