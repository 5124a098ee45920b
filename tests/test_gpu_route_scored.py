"""spice_route_scored against a row-by-row evaluation in 64 bits: indices equal (ties towards the smaller index, rows that fp32
cannot decide included), gates within the fp32 roundings of their formula.

Gate tolerance: expf is within 2 ulp, its argument off by |x - max| 2^-24 (|x - max| <= 40 here: 40 half steps), a sum over N
adds at most N / 32 + 5 in turn, quotient, product and scale 3 more: (4 + 40 + 37 + 3) 2^-24, in numerator and denominator:
1.1e-5 relative.  Below fp32's range: 1e-37."""
import numpy as np
import pytest
import torch

from paper_2608_21240_b200 import binding as B

pytestmark = pytest.mark.gpu


def reference(logits, bias, K, score, G, top, pair, norm, scale):
    idx, gate = [], []
    N = logits.shape[1]
    for l in logits.astype(np.float64):
        b = np.zeros(N) if bias is None else bias.astype(np.float64)
        there = (l > -np.inf) & (b > -np.inf)          # NaN compares false
        with np.errstate(all="ignore"):
            if score == "softmax":
                m = max(l[there], default=0.0)
                e = np.where(there, np.where(l == m, 1.0, np.exp(l - m)), 0.0)
                every = np.where(l > -np.inf, np.where(l == m, 1.0, np.exp(l - m)), 0.0) if bias is None else e
                s = np.where(there, every / max(every.sum(), 1e-300), 0.0)
            else:
                s = np.where(there, 1 / (1 + np.exp(-l)), 0.0)
        value = np.where(there, s + b, -np.inf)
        key = np.where(there, l, -np.inf) if bias is None else value
        allowed = np.ones(N, bool)
        if G > 1:
            worth = []
            for g in range(G):
                part = slice(g * (N // G), (g + 1) * (N // G))
                if pair:
                    best = np.sort(value[part])[::-1][:2]
                    best = best[best > -np.inf]
                    worth.append(best.sum() if len(best) else -np.inf)
                else:
                    worth.append(key[part].max())
            order = sorted(range(G), key=lambda g: (-worth[g], g))[:top]
            allowed = np.isin(np.arange(N) // (N // G), order)
        win = sorted(np.nonzero(allowed)[0], key=lambda e: (-key[e], e))[:K]
        w = s[win]
        if norm:
            w = w / w.sum() if w.sum() > 0 else np.zeros(K)
        idx.append(win)
        gate.append(scale * w)
    return np.array(idx), np.array(gate)


def call(logits, bias, K, score, G, top, pair, norm, scale):
    T = logits.shape[0]
    lg = torch.from_numpy(logits).cuda()
    bs = None if bias is None else torch.from_numpy(bias).cuda()
    idx = torch.full((T + 2, K), -9, dtype=torch.int32, device="cuda")
    gate = torch.full((T + 2, K), -9.0, device="cuda")
    B.spice_route_scored(lg, idx[:T], gate[:T], bias=bs, score=B.SCORE_SOFTMAX if score == "softmax" else B.SCORE_SIGMOID,
                         n_groups=G, top_groups=top, group_score=B.GROUP_TOP2 if pair else B.GROUP_MAX, norm_topk=norm, scale=scale)
    torch.cuda.synchronize()
    assert (idx[T:] == -9).all() and (gate[T:] == -9).all()
    return idx[:T].cpu().numpy(), gate[:T].cpu().numpy().astype(np.float64)


def check(logits, bias, K, score="sigmoid", G=1, top=1, pair=False, norm=True, scale=1.0):
    ri, rg = reference(logits, bias, K, score, G, top, pair, norm, scale)
    gi, gg = call(logits, bias, K, score, G, top, pair, norm, scale)
    assert np.array_equal(gi, ri), np.nonzero((gi != ri).any(1))
    assert (np.abs(gg - rg) <= 1.1e-5 * np.abs(rg) + 1e-37).all(), np.abs(gg - rg).max()
    return gi, gg


def draw(T, N, seed, bias=True, std=1.5):
    r = np.random.default_rng(seed)
    return (std * r.standard_normal((T, N))).astype(np.float32), (0.1 * r.standard_normal(N)).astype(np.float32) if bias else None


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("N,K,G,top,pair", [(1, 1, 1, 1, False), (8, 2, 1, 1, False), (64, 6, 1, 1, False), (64, 6, 8, 3, False),
                                            (45, 5, 1, 1, False), (45, 5, 9, 2, True), (256, 8, 8, 4, True), (160, 6, 8, 3, False),
                                            (96, 4, 3, 2, True), (1024, 32, 32, 2, True), (1000, 10, 1, 1, False), (32, 32, 32, 32, True),
                                            (30, 7, 30, 7, True), (62, 31, 31, 16, False), (33, 32, 1, 1, False)])
def test_routing_matches_its_definition(score, bias, N, K, G, top, pair):
    for norm, scale, seed in ((True, 1.0, 1), (False, 2.5, 2)):
        check(*draw(37, N, seed + N, bias), K, score, G, top, pair, norm, scale)


def test_order_of_plain_softmax_is_that_of_the_existing_router():
    """Without bias and groups: the selection and the gates of spice_route_topk from its own logits."""
    d, N, K, T = 256, 64, 6, 19
    L = B.SpiceLayer(B.make_cfg(d, N, K, 512, 512, 16, 5, 0.5), T)
    g = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn(T, d, device="cuda", generator=g).bfloat16()
    w = (torch.randn(N, d, device="cuda", generator=g) * 0.1).bfloat16()
    idx, gate, logits = L.route_topk(h, w, want_logits=True)
    i2, g2 = torch.empty_like(idx), torch.empty_like(gate)
    B.spice_route_scored(logits, i2, g2)
    assert torch.equal(i2, idx) and (g2 - gate).abs().max() <= 2e-6
    L.close()


def test_equal_keys_go_to_the_smaller_index():
    z = np.zeros((3, 70), np.float32)
    z[1, 40:] = 1
    z[2, ::2] = -1
    for score in ("softmax", "sigmoid"):
        for bias in (None, np.zeros(70, np.float32), np.where(np.arange(70) % 3 == 0, 0.25, 0).astype(np.float32)):
            gi, _ = check(z, bias, 5, score)
            check(z, bias, 5, score, G=7, top=2, pair=True)
            check(z, bias, 5, score, G=7, top=2)
            if bias is None:
                assert gi[0].tolist() == [0, 1, 2, 3, 4] and gi[1].tolist() == [40, 41, 42, 43, 44] and gi[2].tolist() == [1, 3, 5, 7, 9]


def test_keys_that_fp32_cannot_tell_apart():
    """Scores whose sums with the bias differ by less than fp32 resolves: the order is that of the exact values."""
    r = np.random.default_rng(3)
    T, N = 64, 64
    l = r.standard_normal((T, N)).astype(np.float32)
    bias = (0.5 - 1 / (1 + np.exp(-l[0].astype(np.float64)))).astype(np.float32)    # row 0: every key is 0.5 to within 2^-25
    l[1:8] = l[0]
    l[2] = np.nextafter(l[0], np.float32(9))
    l[3] = np.nextafter(l[0], np.float32(-9))
    check(l, bias, 8)
    check(l, bias, 8, G=8, top=3, pair=True)
    check(l, bias, 8, G=8, top=3)
    m = l[0].astype(np.float64) - l[0].max()
    p = np.exp(m) / np.exp(m).sum()
    check(l, (0.25 - p).astype(np.float32), 8, "softmax")
    check(l, (0.25 - p).astype(np.float32), 8, "softmax", G=4, top=2, pair=True)


def test_groups_whose_sums_nearly_tie_without_a_bias():
    """Group sums decide with scores, winners then go by logits, which tell apart what sigmoid's scores no longer do."""
    l = np.full((2, 16), -3, np.float32)
    l[0, [0, 5, 9, 13]] = [40, 45, 41, 50]
    l[0, [1, 4, 8, 12]] = [38, 39, 37, 60]
    l[1] = np.repeat(np.float32([1, 1, 1, 1]), 4) + np.tile(np.float32([0, -1e-7, 0, 0]), 4)
    # (sigmoid in 64 bits still separates 37 from 40: 1 - 8.5e-17 rounds to the neighbour of 1)
    l[0] = np.minimum(l[0], 30)
    check(l, None, 6, "sigmoid", G=4, top=2, pair=True)
    l[0, [0, 5]] = [60, 70]
    check(l, None, 6, "sigmoid")                       # no groups: 70 before 60, whatever their scores


def test_masked_rows_and_values_that_are_not_finite():
    l, bias = draw(8, 48, 9)
    l[0] = -np.inf                                      # nothing left: valid ids, gates 0
    l[1, 4:] = -np.inf                                  # fewer than K left
    l[2, ::5] = np.nan
    l[3, 7] = np.inf
    l[4, [7, 30]] = np.inf
    l[5] = np.nan
    l[6] = np.finfo(np.float32).min                     # a mask by the lowest value
    l[6, 20] = 0.5
    for score in ("softmax", "sigmoid"):
        for b in (None, bias):
            for norm in (True, False):
                gi, gg = check(l, b, 6, score, norm=norm)
                assert (gg[0] == 0).all() and (gg[5] == 0).all() and (gi >= 0).all() and (gi < 48).all()
                assert (gg[1, 4:] == 0).all()
                check(l, b, 6, score, G=6, top=2, pair=True, norm=norm)
                check(l, b, 6, score, G=6, top=2, norm=norm)
    b2 = bias.copy()
    b2[3] = -np.inf
    b2[11] = np.nan
    b2[17] = np.inf
    r = l[7:]
    check(r, b2, 6)
    check(r, b2, 6, G=6, top=3, pair=True)


def test_gates_of_scores_below_fp32_keep_their_ratios():
    l = np.float32([[-200, -201, -202, -203], [-95, -100, -120, -300]])
    check(l, None, 3)
    check(np.concatenate([l, np.full((2, 4), 20, np.float32)], 1), np.float32([9] * 4 + [0] * 4), 3)


def test_empty_batch_streams_and_graphs():
    l, bias = draw(300, 256, 21)
    e = torch.empty
    B.spice_route_scored(e(0, 64, device="cuda"), e(0, 6, dtype=torch.int32, device="cuda"), e(0, 6, device="cuda"))
    kw = dict(score=B.SCORE_SIGMOID, n_groups=8, top_groups=4, group_score=B.GROUP_TOP2, scale=2.5)
    lg, bs = torch.from_numpy(l).cuda(), torch.from_numpy(bias).cuda()
    ref = e(300, 8, dtype=torch.int32, device="cuda"), e(300, 8, device="cuda")
    B.spice_route_scored(lg, *ref, bias=bs, **kw)
    got = torch.zeros_like(ref[0]), torch.zeros_like(ref[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.spice_route_scored(lg, *got, bias=bs, **kw)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    side = torch.cuda.Stream()
    got[1].zero_()
    torch.cuda.synchronize()
    B.spice_route_scored(lg, *got, bias=bs, stream=side, **kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_refusals_on_tensors():
    e = torch.empty
    lg, idx, gate = e(4, 16, device="cuda"), e(4, 2, dtype=torch.int32, device="cuda"), e(4, 2, device="cuda")
    for args, kw in (((lg, idx[:3], gate), {}), ((lg, idx, gate[:, :1]), {}), ((lg.half(), idx, gate), {}), ((lg, idx.long(), gate), {}),
                     ((lg, idx, gate), dict(bias=e(15, device="cuda"))), ((lg.t(), idx, gate), {}), ((lg, idx, gate), dict(n_groups=3)),
                     ((lg, idx, gate), dict(n_groups=16, top_groups=1)), ((lg, idx, gate), dict(score=2))):
        with pytest.raises(B.SpiceError):
            B.spice_route_scored(*args, **kw)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("big", [4.0, 64.0, 256.0, 1e6])
def test_groups_whose_two_best_keys_cancel(score, big):
    """A group's value is the sum of two keys that may be far larger than it: +-big in every group, sums 1e-7 to 5e-6 apart.
    The keys' own rounding decides how far fp32 can be trusted."""
    r = np.random.default_rng(int(big))
    for N, G, top, spread in ((64, 8, 4, 1e-5), (1024, 32, 8, 1e-3 if score == "softmax" else 1e-5)):
        l = (0.3 + spread * r.standard_normal((200, N))).astype(np.float32)
        bias = np.full(N, -4 * big, np.float32)
        bias[::N // G], bias[1::N // G] = big, np.float32(-big + 0.125)
        check(l, bias, 8, score, G=G, top=top, pair=True)


def test_groups_whose_two_best_keys_sum_beyond_fp32():
    """Biases of the type's lowest value: the sum of two is below fp32's range, but the experts are there, and come before a
    group without an available one."""
    low = np.finfo(np.float32).min
    bias = np.full(24, -np.inf, np.float32)
    bias[8:16] = low
    l = draw(5, 24, 31, False)[0]
    gi, gg = check(l, bias, 2, G=3, pair=True)
    assert (gi >= 8).all() and (gi < 16).all() and (gg > 0).all()
    bias[17] = low                                       # one such expert alone is worth more than two
    gi, _ = check(l, bias, 1, G=3, pair=True)
    assert (gi == 17).all()
    bias[:8], bias[9], bias[10] = -0.8 * low, -low, -0.9 * low   # and the same above it
    gi, _ = check(l, bias, 2, G=3, pair=True)
    assert (gi == [9, 10]).all()
