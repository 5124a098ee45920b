"""spice_gemm_i8 and spice_swiglu_i8 against the exact integer products (64 bits).

Tolerances: the sum is exact; its conversion to fp32 and the two scales are one rounding each (3 half steps of 2^-24), the
addition of SPICE_OUT_F32_ADD one more of the result, bf16 one of 2^-8.  SwiGLU: g and u carry 3 * 2^-24 each; e^-g carries
the relative error |g| (3 * 2^-24 + 1.2 * 2^-23) + 2 * 2^-23 of its argument and of the fast exponential; quotient, product:
below (4 |g| + 16) 2^-24 in all before the rounding to bf16."""
import pytest
import torch

from paper_2608_21240_b200 import binding as B

pytestmark = pytest.mark.gpu

bf, f32, f64, i8 = torch.bfloat16, torch.float32, torch.float64, torch.int8
HALF = 2.0 ** -24


def codes(rows, cols, seed, full=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-128 if full else -127, 128, (rows, cols), device="cuda", generator=g).to(i8)
    return q, torch.rand(rows, device="cuda", generator=g) * 0.02 + 1e-3


def exact(xq, xs, wq, ws):
    return (xq.to(f64) @ wq.to(f64).T) * xs.to(f64)[:, None] * ws.to(f64)


def run(xq, xs, wq, ws, out, pad=2):
    T, n = xq.shape[0], wq.shape[0]
    y = torch.full((T + pad, n), 3.0, dtype=bf if out == "bf16" else f32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.spice_gemm_i8(xq, xs, wq, ws, y[:T], accumulate=out == "add", device_status=st)
    torch.cuda.synchronize()
    assert int(st) == 0 and (y[T:] == 3).all()      # rows behind the last one stay as they are
    return y[:T]


def check(T, n, k, out, full=False):
    xq, xs = codes(T, k, T + n, full)
    wq, ws = codes(n, k, k + 1, full)
    e = exact(xq, xs, wq, ws)
    y = run(xq, xs, wq, ws, out).to(f64)
    tol = 3 * HALF * e.abs()
    if out == "bf16":
        tol = tol + 2.0 ** -8 * e.abs()
    if out == "add":
        e = e + 3
        tol = tol + HALF * e.abs()
    assert ((y - e).abs() <= tol * (1 + 1e-6)).all(), float(((y - e).abs() - tol).max())


SHAPES = [(1, 8, 16), (1, 2048, 2816), (3, 72, 48), (16, 136, 144), (17, 128, 2048), (33, 1000, 528), (64, 3584, 1040),
          (77, 264, 20480), (128, 200, 256), (129, 512, 4096), (256, 72, 128), (257, 264, 80), (300, 2048, 400), (512, 256, 128),
          (513, 520, 1408), (1000, 128, 16), (1025, 2816, 272), (130, 3592, 8192), (256, 264, 20480), (300, 1000, 8208), (512, 3584, 6160),
          (700, 520, 20480)]


@pytest.mark.parametrize("T,n,k", SHAPES)
@pytest.mark.parametrize("out", ["bf16", "f32", "add"])
def test_product_matches_the_exact_sums(T, n, k, out):
    check(T, n, k, out)


@pytest.mark.parametrize("T", [5, 200, 700])
def test_the_largest_sums_are_exact(T):
    """-128 * -128 over the longest rows fills 31 bits; every code at its ends."""
    k = 131056
    xq = torch.full((T, k), -128, dtype=i8, device="cuda")
    wq = torch.full((16, k), -128, dtype=i8, device="cuda")
    wq[1] = 127
    wq[2, ::2] = 127
    one = torch.ones(max(T, 16), device="cuda")
    y = run(xq, one[:T], wq, one[:16], "f32").to(f64)
    e = exact(xq, one[:T], wq, one[:16])
    assert float(e.max()) == 2 ** 14 * k and ((y - e).abs() <= HALF * e.abs()).all()


def test_results_do_not_depend_on_the_batch():
    """A token's row is the same bits alone, in a small batch and in a large one (exact sums, the same roundings)."""
    xq, xs = codes(600, 1408, 1)
    wq, ws = codes(2048, 1408, 2)
    whole = run(xq, xs, wq, ws, "f32")
    for a, b in ((0, 1), (3, 11), (40, 53), (7, 38), (3, 60), (100, 190), (0, 256), (300, 599)):
        assert torch.equal(run(xq[a:b].contiguous(), xs[a:b].contiguous(), wq, ws, "f32"), whole[a:b])


def check_swiglu(T, inter, k, scale=1.0):
    xq, xs = codes(T, k, T * 3 + inter)
    wq, ws = codes(2 * inter, k, k + 5)
    ws = ws * (scale / (k ** 0.5 * 73 * 73 * 0.011 * 0.011) * 2)        # products of a few units
    act = torch.full((T + 2, inter), 3.0, dtype=bf, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.spice_swiglu_i8(xq, xs, wq, ws, act[:T], device_status=st)
    torch.cuda.synchronize()
    assert int(st) == 0 and (act[T:] == 3).all()
    y = exact(xq, xs, wq, ws)
    g, u = y[:, :inter], y[:, inter:]
    e = g / (1 + (-g).exp()) * u
    tol = (2.0 ** -8 + (4 * g.abs() + 16) * HALF) * e.abs() + 1e-30
    assert torch.isfinite(act).all() and ((act[:T].to(f64) - e).abs() <= tol).all()


@pytest.mark.parametrize("T,inter,k", [(1, 8, 16), (1, 2816, 2048), (2, 72, 48), (16, 136, 2048), (31, 64, 3584), (100, 200, 528),
                                       (256, 72, 144), (257, 264, 80), (513, 136, 400), (700, 1408, 256),
                                       (9, 264, 2048), (40, 1408, 8192), (256, 520, 8208), (300, 136, 20480), (513, 1000, 6160)])
def test_swiglu_matches_its_definition(T, inter, k):
    check_swiglu(T, inter, k)


def test_swiglu_of_large_gates():
    check_swiglu(20, 128, 512, 40.0)                 # |g| of several hundred: the exponential under- and overflows
    check_swiglu(300, 128, 512, 40.0)


def test_nan_scales_stay_in_their_rows():
    for T in (9, 300):
        xq, xs = codes(T, 256, 3)
        wq, ws = codes(128, 256, 4)
        clean = run(xq, xs, wq, ws, "f32").clone()
        xs[4] = float("nan")
        y = run(xq, xs, wq, ws, "f32")
        assert torch.isnan(y[4]).all()
        clean[4] = y[4] = 0
        assert torch.equal(y, clean)


@pytest.mark.parametrize("T", [16, 400])
def test_other_streams_graphs_and_two_calls_at_once(T):
    """Two captured calls replayed on two streams at the same time, many times over: no workspace to share."""
    data = []
    for i in range(2):
        xq, xs = codes(T, 2048 + 256 * i, 10 + i)
        wq, ws = codes(2816, 2048 + 256 * i, 20 + i)
        data.append((xq, xs, wq, ws, torch.empty(T, 2816, dtype=bf, device="cuda"), torch.empty(T, 1408, dtype=bf, device="cuda")))
    refs = []
    for xq, xs, wq, ws, y, a in data:
        B.spice_gemm_i8(xq, xs, wq, ws, y)
        B.spice_swiglu_i8(xq, xs, wq, ws, a)
        refs.append((y.clone(), a.clone()))
    torch.cuda.synchronize()
    streams, graphs = [torch.cuda.Stream() for _ in data], []
    for (xq, xs, wq, ws, y, a), s in zip(data, streams):
        y.zero_()
        a.zero_()
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            for _ in range(5):
                B.spice_gemm_i8(xq, xs, wq, ws, y)
                B.spice_swiglu_i8(xq, xs, wq, ws, a)
        graphs.append(gr)
    for _ in range(20):
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    for (_, _, _, _, y, a), (ry, ra) in zip(data, refs):
        assert torch.equal(y, ry) and torch.equal(a, ra)


def test_empty_batches_and_refusals_on_tensors():
    xq, xs = codes(4, 64, 1)
    wq, ws = codes(16, 64, 2)
    y = torch.empty(4, 16, dtype=bf, device="cuda")
    B.spice_gemm_i8(xq[:0], xs[:0], wq, ws, y[:0])
    B.spice_swiglu_i8(xq[:0], xs[:0], wq, ws, y[:0, :8].contiguous())
    for args, kw in (((xq, xs, wq, ws, y), dict(accumulate=True)), ((xq, xs[:3], wq, ws, y), {}), ((xq, xs, wq[:, :48], ws, y), {}),
                     ((xq, xs, wq, ws, y[:, :8]), {}), ((xq, xs, wq, ws, y.half()), {}), ((xq[:, :56].contiguous(), xs, wq, ws, y), {}),
                     ((xq.cpu(), xs, wq, ws, y), {}), ((xq, xs, wq, ws.half(), y), {}), ((xq[:, :40].contiguous(), xs, wq[:, :40].contiguous(), ws, y), {})):
        with pytest.raises(B.SpiceError):
            B.spice_gemm_i8(*args, **kw)
    with pytest.raises(B.SpiceError):
        B.spice_swiglu_i8(xq, xs, wq[:15], ws[:15], y[:, :7])
    with pytest.raises(B.SpiceError):
        B.spice_swiglu_i8(xq, xs, wq, ws, y)


# Shapes that the choice of kernel (148 SMs) sends where the ones above do not go: more tiles than CTA pairs (second
# accumulator, ring and barriers carried from tile to tile; 17 and more token tiles: several groups, the last one partial),
# three and four pairs to a tile, token tiles of 128 columns, whole lines of a long reduction per warp.
MORE_SHAPES = [(2600, 2056, 1040), (4100, 2824, 272), (5000, 3592, 144), (257, 3584, 8208), (513, 264, 8208), (1100, 520, 6160),
               (130, 3584, 20480), (128, 3584, 20480), (1, 4096, 11008), (12, 264, 11008), (16, 4096, 11008)]


@pytest.mark.parametrize("T,n,k", MORE_SHAPES)
@pytest.mark.parametrize("out", ["bf16", "f32", "add"])
def test_product_of_more_tiles_and_longer_sums(T, n, k, out):
    check(T, n, k, out)


@pytest.mark.parametrize("T,inter,k", [(2600, 1032, 1040), (4500, 2824, 144), (513, 264, 8208), (513, 520, 12304), (128, 1792, 20480),
                                       (1, 4096, 5504), (5, 1032, 11008), (12, 72, 11008)])
def test_swiglu_of_more_tiles_and_longer_sums(T, inter, k):
    check_swiglu(T, inter, k)


def test_results_of_a_prompt_do_not_depend_on_the_batch():
    """Rows of 4200 tokens through the persistent kernel are the bits of smaller calls."""
    xq, xs = codes(4200, 528, 31)
    wq, ws = codes(2056, 528, 32)
    whole = run(xq, xs, wq, ws, "f32")
    for a, b in ((0, 1), (700, 1300), (2500, 2530), (4090, 4200)):
        assert torch.equal(run(xq[a:b].contiguous(), xs[a:b].contiguous(), wq, ws, "f32"), whole[a:b])


@pytest.mark.parametrize("T,n,k", [(40, 272, 2048), (300, 272, 2048), (700, 2064, 528), (2600, 2064, 528), (513, 272, 8208)])
def test_expired_waits_are_reported(T, n, k):
    """With waits that give up at once, a call ends by itself, reports it, and writes nothing behind its rows; the next call is
    as always.  (Few tokens with a split reduction, pairs, pairs that share tiles.)"""
    xq, xs = codes(T, k, 1)
    wq, ws = codes(n, k, 2)
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    y = torch.full((T + 2, n), 3.0, dtype=f32, device="cuda")
    act = torch.full((T + 2, n // 2), 3.0, dtype=bf, device="cuda")
    torch.cuda.synchronize()
    B.spice_set_option(None, B.OPT_I8_WAIT_LIMIT, 0)
    try:
        B.spice_gemm_i8(xq, xs, wq, ws, y[:T], device_status=st[:1])
        B.spice_swiglu_i8(xq, xs, wq, ws, act[:T], device_status=st[1:])
        torch.cuda.synchronize()
    finally:
        B.spice_set_option(None, B.OPT_I8_WAIT_LIMIT, 1 << 22)
    assert st.tolist() == [6, 6]                     # SPICE_ERR_TIMEOUT
    assert (y[T:] == 3).all() and (act[T:] == 3).all()
    e = exact(xq, xs, wq, ws)
    assert ((run(xq, xs, wq, ws, "f32").to(f64) - e).abs() <= 3 * HALF * e.abs() * (1 + 1e-6)).all()
