"""spice_sort_tokens, spice_combine_tokens and spice_combine_tokens_grad against plain torch in 64 bits.

The sort is exact, and so are gathered rows.  Tolerances, in half steps (2^-24 fp32, 2^-8 bf16, relative): a sum of K products in
fp32 makes K fused roundings, each of a partial sum of at most sum |gate rows| =: A, and one more where y is added to; a row of the
gradient is one product: one fp32 rounding and one of its type; a gate's gradient is d products added by 32 lanes or more and
then across at most 8 warps: d / 32 + 5 + 8 roundings of at most sum |dy rows|."""
import pytest
import torch

from paper_2608_21240_b200 import binding as B

pytestmark = pytest.mark.gpu

bf, f32, f64, i32, u8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
H32, H16 = 2.0 ** -24, 2.0 ** -8


def plain_sort(idx, N):
    flat = idx.reshape(-1).long().cpu()
    keep = (flat >= 0) & (flat < N)
    i = keep.nonzero()[:, 0]
    order = i[flat[i].sort(stable=True).indices]
    pos = torch.full_like(flat, -1)
    pos[order] = torch.arange(order.numel())
    entry = torch.full_like(flat, -1)
    entry[:order.numel()] = order
    offset = torch.zeros(N + 1, dtype=torch.long)
    offset[1:] = torch.bincount(flat[i], minlength=N).cumsum(0)
    return offset.int(), pos.view(idx.shape).int(), entry.int()


def run_sort(idx, N, x=None, xs=None, pad=3):
    T, K = idx.shape
    dev = idx.device
    out = lambda *s: torch.full(s, -77, dtype=i32, device=dev)  # noqa: E731
    offset, pos, entry = out(N + 1 + pad), out(T + pad, K), out(T * K + pad)
    rows = None if x is None else torch.full((T * K + pad, x.shape[1]), 7, dtype=x.dtype, device=dev)
    rs = None if xs is None else torch.full((T * K + pad, xs.shape[1]), 7.0, dtype=f32, device=dev)
    B.spice_sort_tokens(idx, offset[:N + 1], pos[:T], entry[:T * K], x, None if x is None else rows[:T * K], xs, None if xs is None else rs[:T * K])
    torch.cuda.synchronize()
    assert (offset[N + 1:] == -77).all() and (pos[T:] == -77).all() and (entry[T * K:] == -77).all()
    return offset[:N + 1], pos[:T], entry[:T * K], rows, rs


def check_sort(idx, N, x=None, xs=None):
    ref = plain_sort(idx, N)
    offset, pos, entry, rows, rs = run_sort(idx, N, x, xs)
    for got, want in zip((offset, pos, entry), ref):
        assert torch.equal(got.cpu(), want)
    kept = int(ref[0][-1])
    token = (ref[2][:kept].long() // idx.shape[1]).cuda()
    for got, src in ((rows, x), (rs, xs)):
        if src is not None:
            assert torch.equal(got[:kept].view(u8), src[token].view(u8)) and (got[kept:] == 7).all()


def make_idx(T, K, N, seed, drop=0.2, distinct=True):
    g = torch.Generator().manual_seed(seed)
    if distinct and K <= N:
        idx = torch.rand(T, N, generator=g).argsort(1)[:, :K]
    else:
        idx = torch.randint(0, N, (T, K), generator=g)
    bad = torch.tensor([-1, N, -2 ** 31, 2 ** 31 - 1])[torch.randint(0, 4, (T, K), generator=g)]
    return torch.where(torch.rand(T, K, generator=g) < drop, bad, idx).int().cuda()


# (2048 entries and more take the cluster; 341 x 6 = 2046, 342 x 6 = 2052)
@pytest.mark.parametrize("T,K,N", [(1, 1, 1), (1, 6, 64), (2, 32, 1024), (17, 8, 24), (61, 8, 64), (64, 32, 33), (341, 6, 64), (342, 6, 64), (2048, 1, 5),
                                   (2049, 1, 1024), (1000, 3, 7), (4096, 6, 64), (8191, 8, 257), (8192, 32, 1024), (70001, 1, 300)])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_sort_is_the_stable_sort(T, K, N, drop):
    check_sort(make_idx(T, K, N, T + K + N, drop), N)


@pytest.mark.parametrize("T,K,N,d,kind", [(1, 6, 32, 2048, "bf16"), (1, 1, 1, 8, "bf16"), (5, 8, 64, 16, "e4m3"), (33, 6, 64, 2064, "e4m3"),
                                          (129, 8, 24, 3584, "bf16"), (300, 4, 9, 20480, "f32"), (1000, 6, 64, 1040, "e4m3"), (4096, 6, 64, 72, "bf16"),
                                          (3000, 2, 1000, 516, "f32"), (700, 32, 64, 128, "e4m3")])
def test_rows_and_scales_follow(T, K, N, d, kind):
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(T, d, device="cuda", generator=g)
    x = x.to(bf) if kind == "bf16" else (x * 50).to(torch.int8).view(u8) if kind == "e4m3" else x
    xs = torch.rand(T, -(-d // 128), device="cuda", generator=g) if kind == "e4m3" else None
    check_sort(make_idx(T, K, N, d, 0.25), N, x, xs)


@pytest.mark.parametrize("T", [5, 3000])
def test_extreme_routings(T):
    x = torch.randn(T, 64, device="cuda").to(bf)
    for idx in (torch.full((T, 4), -1), torch.full((T, 4), 7), torch.full((T, 4), 8), torch.zeros(T, 4), torch.arange(4).repeat(T, 1),
                torch.tensor([3, 3, 0, 3]).repeat(T, 1)):     # all dropped, one expert, twice the same one in a token's row
        check_sort(idx.int().cuda(), 8, x)
    check_sort(torch.zeros(T, 4, dtype=i32, device="cuda"), 1, x)


def test_empty_batch():
    z = lambda *s: torch.empty(*s, dtype=i32, device="cuda")  # noqa: E731
    offset = torch.full((9,), -5, dtype=i32, device="cuda")
    B.spice_sort_tokens(z(0, 4), offset, z(0, 4), z(0))
    y = torch.empty(0, 64, dtype=bf, device="cuda")
    B.spice_combine_tokens(torch.empty(0, 64, dtype=bf, device="cuda"), z(0, 4), y)
    B.spice_combine_tokens_grad(y, torch.empty(0, 64, dtype=bf, device="cuda"), z(0, 4), None, torch.empty(0, 64, dtype=bf, device="cuda"))
    torch.cuda.synchronize()
    assert (offset == -5).all()


# ------------------------------------------------------------------------------------------------ back
def taken(rows, pos):
    p = pos.long()
    ok = (p >= 0) & (p < rows.shape[0])
    return torch.where(ok[..., None], rows.to(f64)[p.clamp(0, rows.shape[0] - 1)], 0.0)


def make_rows(T, K, N, d, kind, seed, drop=0.2):
    idx = make_idx(T, K, N, seed, drop)
    offset, pos, entry, _, _ = run_sort(idx, N)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.randn(T * K, d, device="cuda", generator=g).to(kind)
    rows[int(offset[-1]):] = float("nan")                       # nobody points there
    return pos.contiguous(), rows, torch.rand(T, K, device="cuda", generator=g) - 0.3, g


SIZES = [(1, 1, 4, 8), (1, 6, 32, 2048), (3, 32, 64, 72), (17, 8, 24, 3584), (61, 8, 64, 1000), (200, 6, 64, 2056), (1025, 5, 16, 520), (2048, 6, 64, 2048),
         (9, 4, 8, 20480)]


@pytest.mark.parametrize("T,K,N,d", SIZES)
@pytest.mark.parametrize("kind", [bf, f32])
@pytest.mark.parametrize("out", ["bf16", "f32", "add"])
def test_combine(T, K, N, d, kind, out):
    pos, rows, gate, _ = make_rows(T, K, N, d, kind, T + d)
    for weights in (gate, None):
        y = torch.full((T + 2, d), 3.0, dtype=bf if out == "bf16" else f32, device="cuda")
        B.spice_combine_tokens(rows, pos, y[:T], weights, accumulate=out == "add")
        torch.cuda.synchronize()
        assert (y[T:] == 3).all()
        parts = taken(rows, pos) * (1 if weights is None else weights.to(f64)[..., None])
        e, A = parts.sum(1), parts.abs().sum(1)
        tol = K * H32 * A
        if out == "bf16":
            tol = tol + H16 * (e.abs() + tol)
        if out == "add":
            e = e + 3
            tol = tol + H32 * (e.abs() + tol)
        assert ((y[:T].to(f64) - e).abs() <= tol * (1 + 1e-6)).all()


@pytest.mark.parametrize("T,K,N,d", SIZES)
@pytest.mark.parametrize("kind", [bf, f32])
@pytest.mark.parametrize("dkind", [bf, f32])
def test_gradient(T, K, N, d, kind, dkind):
    pos, rows, gate, g = make_rows(T, K, N, d, kind, T + d)
    dy = torch.randn(T, d, device="cuda", generator=g).to(dkind)
    d_rows = torch.full((T * K, d), 5.0, dtype=kind, device="cuda")
    d_gate = torch.full((T + 1, K), 5.0, device="cuda")
    B.spice_combine_tokens_grad(dy, rows, pos, gate, d_rows, d_gate[:T])
    torch.cuda.synchronize()
    some = pos >= 0
    want = (gate.to(f64)[..., None] * dy.to(f64)[:, None])[some]
    got = d_rows[pos[some].long()].to(f64)
    assert ((got - want).abs() <= (H32 + (H16 if kind == bf else 0)) * want.abs() * (1 + 1e-2)).all()
    left = torch.ones(T * K, dtype=torch.bool, device="cuda")
    left[pos[some].long()] = False
    assert (d_rows[left] == 5).all() and (d_gate[T:] == 5).all()
    prod = taken(rows, pos) * dy.to(f64)[:, None]
    tol = (d / 32 + 13) * H32 * prod.abs().sum(2)
    assert ((d_gate[:T].to(f64) - prod.sum(2)).abs() <= tol * (1 + 1e-6)).all()
    # parts of it, and weights of 1
    one, only = torch.full_like(d_rows, 5.0), torch.empty_like(gate)
    B.spice_combine_tokens_grad(dy, None, pos, gate, one)
    B.spice_combine_tokens_grad(dy, rows, pos, gate, None, only)
    torch.cuda.synchronize()
    assert torch.equal(one, d_rows) and torch.equal(only, d_gate[:T])
    B.spice_combine_tokens_grad(dy, None, pos, None, one)
    torch.cuda.synchronize()
    assert torch.equal(one[pos[some].long()], dy[:, None].expand(T, K, d)[some].to(kind))


def test_gradient_against_differences():
    """y is linear in the gates and in the rows: a difference over a step of 1 is the derivative, up to the roundings of two values
    of y (K of at most A each) on either side, weighted with |dy|."""
    T, K, N, d = 7, 4, 6, 64
    pos, rows, gate, g = make_rows(T, K, N, d, f32, 3)
    dy = torch.randn(T, d, device="cuda", generator=g)

    def loss(r, w):
        y = torch.empty(T, d, device="cuda")
        B.spice_combine_tokens(r, pos, y, w)
        return float((y.to(f64) * dy.to(f64)).sum())

    d_rows, d_gate = torch.zeros_like(rows), torch.empty_like(gate)
    B.spice_combine_tokens_grad(dy, rows, pos, gate, d_rows, d_gate)
    parts = taken(rows, pos).abs() * (gate.to(f64).abs() + 1)[..., None]
    slack = 2 * K * H32 * float((parts.sum(1) * dy.to(f64).abs()).sum()) + (d / 32 + 13) * H32 * float(parts.sum() * dy.abs().max())
    for t, k in ((0, 0), (3, 2), (6, 3), (5, 1)):
        up = gate.clone()
        up[t, k] += 1
        step = float(up[t, k].to(f64) - gate[t, k].to(f64))
        assert abs(loss(rows, up) - loss(rows, gate) - step * float(d_gate[t, k])) <= slack
    for p, j in ((0, 0), (5, 17), (11, 63)):
        up = rows.clone()
        up[p, j] += 1
        step = float(up[p, j].to(f64) - rows[p, j].to(f64))
        assert abs(loss(up, gate) - loss(rows, gate) - step * float(d_rows[p, j])) <= slack


def test_gather_and_combine_without_gates_are_each_others_gradient():
    """<gather(x), r> = <x, combine(r)>, evaluated in 64 bits from what the calls return."""
    T, K, N, d = 333, 6, 64, 264
    idx = make_idx(T, K, N, 5, 0.3)
    x = torch.randn(T, d, device="cuda")
    offset, pos, entry, rows, _ = run_sort(idx, N, x)
    kept = int(offset[-1])
    r = torch.randn(T * K, d, device="cuda")
    y = torch.empty(T, d, device="cuda")
    B.spice_combine_tokens(r, pos.contiguous(), y)
    left = (rows[:kept].to(f64) * r[:kept].to(f64)).sum()
    right = (x.to(f64) * y.to(f64)).sum()
    assert abs(float(left - right)) <= K * H32 * float((taken(r, pos).abs().sum(1) * x.to(f64).abs()).sum())


def test_nan_and_infinity_stay_with_their_tokens():
    pos, rows, gate, _ = make_rows(50, 4, 8, 128, bf, 9, 0.3)
    y = torch.empty(50, 128, dtype=f32, device="cuda")
    p = pos[7][pos[7] >= 0]
    assert p.numel()
    rows[p[0].long(), 3] = float("inf")
    rows[p[0].long(), 5] = float("nan")
    B.spice_combine_tokens(rows, pos, y, gate)
    torch.cuda.synchronize()
    odd = ~torch.isfinite(y)
    assert odd.sum() == 2 and odd[7, 3] and odd[7, 5]
    # places that are out of range do not count
    wild = pos.clone()
    wild[wild < 0] = 1 << 30
    again = torch.empty_like(y)
    B.spice_combine_tokens(rows, wild, again, gate)
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(y))


def test_more_than_32_bits_of_rows():
    """Rows that lie more than 2^32 bytes into their array."""
    T, K, d = 9, 1, 1 << 20
    n = 4500                                                    # 4500 x 2^20 x 1 byte for the sort, x 2 for the sums
    x = torch.randint(0, 255, (n, d), dtype=u8, device="cuda")
    idx = torch.zeros(n, 1, dtype=i32, device="cuda")
    _, pos, _, rows, _ = run_sort(idx, 1, x, pad=0)
    assert torch.equal(rows[-3:], x[-3:])
    del rows, x
    r = torch.randn(2100, d, device="cuda").to(bf)
    p = torch.tensor([[2099]], dtype=i32, device="cuda")
    y = torch.empty(1, d, dtype=bf, device="cuda")
    B.spice_combine_tokens(r, p, y)
    g = torch.zeros_like(r)
    B.spice_combine_tokens_grad(y, None, p, None, g)
    torch.cuda.synchronize()
    assert torch.equal(y[0], r[2099]) and torch.equal(g[2099], r[2099])


@pytest.mark.parametrize("T", [40, 1200])
def test_captured_calls_on_two_streams(T):
    """Two captured chains (sort, combine, gradient) replayed on two streams at once, many times over."""
    data = []
    for i in range(2):
        idx = make_idx(T, 6, 64, i, 0.2)
        x = torch.randn(T, 512 + 64 * i, device="cuda").to(bf)
        offset, pos, entry, rows, _ = run_sort(idx, 64, x, pad=0)
        gate = torch.rand(T, 6, device="cuda")
        bufs = dict(offset=offset, pos=pos, entry=entry, rows=rows, y=torch.empty_like(x), dr=torch.zeros_like(rows), dg=torch.empty_like(gate))

        def chain(b=bufs, idx=idx, x=x, gate=gate):
            B.spice_sort_tokens(idx, b["offset"], b["pos"], b["entry"], x, b["rows"])
            B.spice_combine_tokens(b["rows"], b["pos"], b["y"], gate)
            B.spice_combine_tokens_grad(b["y"], b["rows"], b["pos"], gate, b["dr"], b["dg"])
        chain()
        torch.cuda.synchronize()
        data.append((chain, bufs, {k: v.clone() for k, v in bufs.items()}))
    graphs = []
    for chain, bufs, _ in data:
        for v in bufs.values():
            v.zero_()
        bufs["rows"].fill_(7)
        torch.cuda.synchronize()
        s, gr = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            for _ in range(5):
                chain()
        graphs.append((s, gr))
    for _ in range(20):
        for s, gr in graphs:
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    for _, bufs, want in data:
        for k, v in bufs.items():
            assert torch.equal(v, want[k]), k
