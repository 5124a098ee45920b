"""Offsets that are not in order, for the products of E4M3 blocks: groups that overlap, more of them than the rows can fill.

What holds: SPICE_ERR_BAD_TABLE is reported; rows of one counted group only (its offsets in order and within 0 .. T) are that group's;
rows of several are, element by element, any of theirs or as they were; all other rows are as they were.  A row's bits depend on T and
the number of groups only, so what group g makes of a row is taken from a call whose table gives all rows to g (that call is compared
with 64 bits elsewhere), and results are compared for equality."""
import pytest
import torch

from paper_2608_21240_b200 import binding as B
from tests.test_gpu_e4m3_blocks import f32, i32, operands, u8

pytestmark = pytest.mark.gpu

KINDS = 3                                                     # different weights: group g has those of g % KINDS
BAD_TABLE = 5


class Calls:
    """A product or SwiGLU over G groups of rows, on fixed operands."""

    def __init__(self, op, T, G, n, k):
        self.op, self.T, self.G, self.n = op, T, G, n
        self.x, self.xs, w, ws = operands(T, 2 * n if op == "swiglu" else n, k, KINDS, T + G + n + k)
        kind = torch.arange(G, device="cuda") % KINDS
        self.w, self.ws = w[kind].contiguous(), ws[kind].contiguous()

    def run(self, bounds, status=0):
        T, n = self.T, self.n
        off = torch.tensor(bounds, dtype=i32, device="cuda")
        st = torch.zeros(1, dtype=i32, device="cuda")
        assert len(bounds) == self.G + 1
        if self.op == "product":
            outs = (torch.full((T + 2, n), 3.0, dtype=f32, device="cuda"),)
            B.spice_gemm_e4m3_blocks(self.x, self.xs, self.w, self.ws, outs[0][:T], off, device_status=st)
        else:
            outs = torch.full((T + 2, n), 0x7e, dtype=u8, device="cuda"), torch.full((T + 2, n // 128), -3.0, device="cuda")
            B.spice_swiglu_e4m3_blocks(self.x, self.xs, self.w, self.ws, outs[0][:T], outs[1][:T], off, st)
        torch.cuda.synchronize()
        assert status is None or int(st) == status
        assert all((o[T:] == o[T, 0]).all() for o in outs)
        return [o[:T] for o in outs]

    def check(self, bounds):
        T, G = self.T, self.G
        status = BAD_TABLE if any(not 0 <= a <= b <= T for a, b in zip(bounds, bounds[1:])) else 0
        untouched = self.run([T] * (G + 1))
        of_kind = [self.run([0] * (g + 1) + [T] * (G - g)) for g in range(min(KINDS, G))]
        assert not torch.equal(of_kind[0][0], untouched[0])
        claims = torch.zeros(T, dtype=torch.long)
        kinds = torch.zeros(T, KINDS, dtype=torch.bool)
        for g in range(G):
            if 0 <= bounds[g] <= bounds[g + 1] <= T:
                claims[bounds[g]:bounds[g + 1]] += 1
                kinds[bounds[g]:bounds[g + 1], g % KINDS] = True
        got = self.run(bounds, status)
        for i, y in enumerate(got):
            fits = torch.zeros_like(y, dtype=torch.bool)
            for kind in range(len(of_kind)):
                fits |= (y == of_kind[kind][i]) & kinds[:, kind, None].cuda()
            fits |= (y == untouched[i]) & (claims != 1)[:, None].cuda()
            assert fits.all(), (i, (~fits).any(1).nonzero().flatten().tolist())


def claimed_over_and_over(T, G):
    """All but the last two rows by half of the groups each, these two by the last group alone."""
    return [0, T - 2] * (G // 2) + [T]


# (reductions shared by the CTAs of a cluster, with more items than clusters: 21 for 9, 13 for 11, 17 for 12, 1025 for 20; then whole
# reductions: too many items for clusters or too short a reduction; then tiles of 256 rows)
STREAMED = [(10, 40, 136, 2064), (26, 8, 136, 528), (64, 8, 136, 528), (18, 1024, 136, 528), (34, 16, 520, 1040), (12, 24, 4104, 528), (33, 8, 72, 144)]


@pytest.mark.parametrize("T,G,n,k", STREAMED + [(900, 8, 264, 272)])
def test_product_of_more_groups_than_rows_can_fill(T, G, n, k):
    Calls("product", T, G, n, k).check(claimed_over_and_over(T, G))


@pytest.mark.parametrize("T,G,n,k", [(8, 40, 128, 2064), (10, 40, 128, 512), (26, 8, 128, 528), (64, 8, 128, 512), (18, 1024, 128, 528), (34, 16, 256, 1040),
                                     (12, 24, 2048, 528), (33, 8, 128, 144), (900, 8, 256, 272)])
def test_swiglu_of_more_groups_than_rows_can_fill(T, G, n, k):
    Calls("swiglu", T, G, n, k).check(claimed_over_and_over(T, G))


@pytest.mark.parametrize("op,T,G,n,k", [("product", 26, 8, 136, 528), ("swiglu", 26, 8, 128, 528), ("product", 900, 8, 264, 272)])
def test_groups_out_of_order_that_do_not_overlap(op, T, G, n, k):
    c = Calls(op, T, G, n, k)
    c.check([T // 2, T, 0, T // 2 - 3, T // 2 - 1, T + 5, -7, 3, T // 2])
    c.check([5, 9, 0, T, 2, 2, 1, 0, T - 1])


# (up to eight tokens: a block for each row, straight from global memory)
@pytest.mark.parametrize("G,n,k", [(18, 136, 528), (40, 72, 272), (1024, 24, 144)])
def test_up_to_eight_tokens_of_more_groups_than_blocks(G, n, k):
    c = Calls("product", 8, G, n, k)
    c.check([0, 1] * (G // 2) + [8])                          # row 0 over and over, then the others
    c.check([7, 8] * (G // 2 - 1) + [0, 8, 3])
    c.check([0, 8] * (G // 2) + [8])
    c.check([3, 5] * (G // 2 - 2) + [0, 2, 1, 4, 8])


@pytest.mark.parametrize("T", [1, 5, 8, 26])
@pytest.mark.parametrize("G", [3, 17, 70])
def test_any_offsets(T, G):
    c = Calls("product", T, G, 72, 400)
    g = torch.Generator().manual_seed(T + G)
    for i in range(12):
        bounds = torch.randint(-1 if i % 2 else 0, T + 1 + i % 2, (G + 1,), generator=g).tolist()
        if i % 3 == 0:                                         # in order but for one offset or two
            bounds = sorted(max(0, min(T, b)) for b in bounds)
            for j in torch.randint(0, G + 1, (2,), generator=g).tolist():
                bounds[j] = int(torch.randint(0, T + 1, (1,), generator=g))
        c.check(bounds)


@pytest.mark.parametrize("op,n", [("product", 136), ("swiglu", 128)])
def test_overlapping_groups_captured_and_between_other_calls(op, n):
    """Replayed over and over beside well-formed calls on another stream, which stay as they are."""
    c = Calls(op, 26, 8, n, 528)
    bounds = [0, 3, 3, 10, 11, 11, 20, 21, 26]
    want = c.run(bounds)
    off = torch.tensor(claimed_over_and_over(26, 8), dtype=i32, device="cuda")
    outs = [torch.empty_like(o) for o in want]
    call = B.spice_gemm_e4m3_blocks if op == "product" else B.spice_swiglu_e4m3_blocks
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(8):
            call(c.x, c.xs, c.w, c.ws, *outs, offset=off)
    for _ in range(10):
        with torch.cuda.stream(side):
            graph.replay()
        for a, b in zip(c.run(bounds), want):
            assert torch.equal(a, b)
    torch.cuda.synchronize()


@pytest.mark.parametrize("op,n", [("product", 136), ("swiglu", 128)])
def test_expired_waits_with_overlapping_groups(op, n):
    """More items than clusters, and waits that give up at once: the call ends by itself and says so."""
    c = Calls(op, 26, 8, n, 528)
    bounds = [0, 3, 3, 10, 11, 11, 20, 21, 26]
    want = c.run(bounds)
    B.spice_set_option(None, B.OPT_E4M3_WAIT_LIMIT, 0)
    try:
        c.run(claimed_over_and_over(26, 8), status=6)         # SPICE_ERR_TIMEOUT, the larger of the two codes
    finally:
        B.spice_set_option(None, B.OPT_E4M3_WAIT_LIMIT, 1 << 22)
    for a, b in zip(c.run(bounds), want):
        assert torch.equal(a, b)
