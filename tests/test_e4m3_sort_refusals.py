"""Host-side checks of the experts' path (tokens sorted by expert and back, E4M3 blocks and their products): every refusal answers
without a device and launches nothing; a call without rows is fine."""
import ctypes as C

import pytest
import torch

from paper_2608_21240_b200 import binding as B

OK, INVALID, SHAPE = 0, 1, 2
P = 4096                   # a 16-byte aligned stand-in for device addresses: no refused call reads it


def sort(idx=P, T=1, K=2, N=8, offset=P, pos=P, entry=P, x=P, row_bytes=64, rows=P, xs=P, cols=1, rs=P):
    return B.lib().spice_sort_tokens(idx, T, K, N, offset, pos, entry, x, row_bytes, rows, xs, cols, rs, None)


def test_sort_refusals():
    assert sort(T=0) == OK and sort(T=0, idx=None, pos=None, entry=None) == OK
    for bad in (dict(T=-1), dict(K=0), dict(N=0), dict(offset=None), dict(idx=None), dict(pos=None), dict(entry=None), dict(idx=P + 2),
                dict(offset=P + 1), dict(pos=P + 2), dict(entry=P + 2), dict(x=None), dict(rows=None), dict(x=P + 8), dict(rows=P + 8),
                dict(row_bytes=0), dict(row_bytes=24), dict(row_bytes=-16), dict(xs=None), dict(rs=None), dict(cols=0), dict(xs=P + 2),
                dict(x=None, rows=None), dict(rs=P + 1)):
        assert sort(**bad) == INVALID, bad
    for bad in (dict(N=1025), dict(K=33), dict(T=1 << 27, K=4)):
        assert sort(**bad) == SHAPE, bad


def combine(rows=P, kind=0, R=4, pos=P, gate=P, T=2, K=2, d=64, out=0, y=P):
    return B.lib().spice_combine_tokens(rows, kind, R, pos, gate, T, K, d, out, y, None)


def grad(dy=P, dk=0, rows=P, rk=0, R=4, pos=P, gate=P, T=2, K=2, d=64, d_rows=P, d_gate=P):
    return B.lib().spice_combine_tokens_grad(dy, dk, rows, rk, R, pos, gate, T, K, d, d_rows, d_gate, None)


def test_combine_and_gradient_refusals():
    assert combine(T=0) == OK and grad(T=0) == OK
    for bad in (dict(T=-1), dict(R=-1), dict(K=0), dict(d=0), dict(d=12), dict(rows=None), dict(pos=None), dict(rows=P + 8), dict(pos=P + 2),
                dict(gate=P + 2)):
        assert combine(**bad) == INVALID, bad
        assert grad(**bad) == INVALID, bad
    for bad in (dict(kind=2), dict(kind=-1), dict(out=3), dict(y=None), dict(y=P + 4)):
        assert combine(**bad) == INVALID, bad
    for bad in (dict(dk=2), dict(rk=-1), dict(dy=None), dict(dy=P + 2), dict(d_rows=P + 4), dict(d_gate=P + 2), dict(d_rows=None, d_gate=None)):
        assert grad(**bad) == INVALID, bad
    for bad in (dict(K=33), dict(d=(1 << 24) + 8), dict(T=1 << 27, K=4)):
        assert combine(**bad) == SHAPE and grad(**bad) == SHAPE, bad


def blocks(w=P, count=1, rows=1, cols=64, tall=1, q=P, scale=P):
    return B.lib().spice_quantize_e4m3_blocks(w, count, rows, cols, tall, q, scale, None)


def test_quantize_blocks_refusals():
    assert blocks(rows=0) == OK and blocks(count=0) == OK
    for bad in (dict(rows=-1), dict(count=-1), dict(cols=0), dict(cols=12), dict(tall=0), dict(tall=64), dict(w=None), dict(q=None),
                dict(scale=None), dict(w=P + 8), dict(q=P + 4), dict(scale=P + 2)):
        assert blocks(**bad) == INVALID, bad
    for bad in (dict(cols=(1 << 24) + 8), dict(rows=1 << 31), dict(count=1 << 31), dict(count=1 << 20, rows=1 << 20),
                dict(count=1 << 20, rows=1 << 20, tall=128), dict(count=(1 << 31) - 1, rows=(1 << 31) - 1, cols=1 << 24)):
        assert blocks(**bad) == SHAPE, bad


def gemm(x=P, xs=P, w=P, ws=P, off=None, G=1, T=1, n=64, k=64, out=0, y=P, status=None):
    return B.lib().spice_gemm_e4m3_blocks(x, xs, w, ws, off, G, T, n, k, out, y, status, None)


def swiglu(x=P, xs=P, w=P, ws=P, off=None, G=1, T=1, n=128, k=64, y=P, ys=P, status=None):
    return B.lib().spice_swiglu_e4m3_blocks(x, xs, w, ws, off, G, T, n, k, y, ys, status, None)


@pytest.mark.parametrize("call", [gemm, swiglu])
def test_product_refusals(call):
    assert call(T=0) == OK and call(T=0, x=None, y=None) == OK
    for bad in (dict(T=-1), dict(n=0), dict(n=12), dict(k=0), dict(k=24), dict(k=8), dict(G=0), dict(G=2), dict(x=None), dict(xs=None),
                dict(w=None), dict(ws=None), dict(y=None), dict(x=P + 8), dict(w=P + 8), dict(ws=P + 2), dict(y=P + 8), dict(xs=P + 2),
                dict(off=P + 2), dict(status=P + 2)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(k=(1 << 24) + 16), dict(n=(1 << 24) + 128), dict(T=(1 << 24) + 1), dict(off=P, G=1025), dict(off=P, G=1024, n=1 << 21)):
        assert call(**bad) == SHAPE, bad
    if call is gemm:
        assert call(out=3) == INVALID and call(out=-1) == INVALID
    else:
        assert call(n=72) == SHAPE and call(ys=None) == INVALID and call(ys=P + 2) == INVALID


def test_wait_limit_of_the_products_is_set_without_a_context():
    assert B.lib().spice_set_option(None, B.OPT_E4M3_WAIT_LIMIT, C.c_int64(1 << 22)) == OK
    for value in (-1, (1 << 30) + 1):
        assert B.lib().spice_set_option(None, B.OPT_E4M3_WAIT_LIMIT, C.c_int64(value)) == INVALID


def test_binding_refuses_host_tensors():
    bf, u8, f32, i32 = torch.bfloat16, torch.uint8, torch.float32, torch.int32
    z = lambda *s, dtype: torch.zeros(*s, dtype=dtype)  # noqa: E731
    for call in (lambda: B.spice_sort_tokens(z(2, 2, dtype=i32), z(9, dtype=i32), z(2, 2, dtype=i32), z(4, dtype=i32)),
                 lambda: B.spice_combine_tokens(z(4, 8, dtype=bf), z(2, 2, dtype=i32), z(2, 8, dtype=bf)),
                 lambda: B.spice_combine_tokens_grad(z(2, 8, dtype=bf), z(4, 8, dtype=bf), z(2, 2, dtype=i32), None, z(4, 8, dtype=bf)),
                 lambda: B.spice_quantize_e4m3_blocks(z(2, 8, dtype=bf), z(2, 8, dtype=u8), z(2, 1, dtype=f32)),
                 lambda: B.spice_gemm_e4m3_blocks(z(2, 16, dtype=u8), z(2, 1, dtype=f32), z(8, 16, dtype=u8), z(1, 1, dtype=f32), z(2, 8, dtype=bf)),
                 lambda: B.spice_swiglu_e4m3_blocks(z(2, 16, dtype=u8), z(2, 1, dtype=f32), z(256, 16, dtype=u8), z(2, 1, dtype=f32),
                                                    z(2, 128, dtype=u8), z(2, 1, dtype=f32))):
        with pytest.raises(B.SpiceError):
            call()


class Stand:
    """What the binding asks of a tensor."""

    def __init__(self, dtype, *shape, dev=0):
        self.dtype, self.shape, self.dev = dtype, torch.Size(shape), dev
        self.is_cuda, self.device = dev >= 0, f"cuda:{dev}" if dev >= 0 else "cpu"

    def get_device(self):
        return self.dev

    def is_pinned(self):
        return self.dev < 0

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def element_size(self):
        return {torch.uint8: 1, torch.bfloat16: 2}.get(self.dtype, 4)

    def data_ptr(self):
        return P


def test_binding_checks_shapes_types_and_devices(monkeypatch):
    calls = []
    monkeypatch.setattr(B, "_call_on", lambda dev, name, stream, *args: calls.append((dev, name, args)))
    bf, u8, f32, i32 = torch.bfloat16, torch.uint8, torch.float32, torch.int32
    S = Stand
    base = dict(idx=S(i32, 3, 2, dev=1), offset=S(i32, 9, dev=1), pos=S(i32, 3, 2, dev=1), entry=S(i32, 6, dev=1))
    with_rows = dict(x=S(u8, 3, 256, dev=1), rows=S(u8, 6, 256, dev=1), x_scale=S(f32, 3, 2, dev=1), rows_scale=S(f32, 6, 2, dev=1))
    B.spice_sort_tokens(**base, **with_rows)
    B.spice_sort_tokens(**base)
    assert calls[0] == (1, "spice_sort_tokens", (P, 3, 2, 8, P, P, P, P, 256, P, P, 2, P))
    assert calls[1][2] == (P, 3, 2, 8, P, P, P, None, 0, None, None, 0, None)
    for bad in (dict(offset=S(i32, 1, dev=1)), dict(entry=S(i32, 5, dev=1)), dict(pos=S(f32, 3, 2, dev=1)), dict(rows=S(u8, 5, 256, dev=1)),
                dict(rows=S(bf, 6, 256, dev=1)), dict(rows=None), dict(x_scale=None), dict(rows_scale=S(f32, 6, 3, dev=1)),
                dict(x=None, rows=None), dict(x=S(u8, 4, 256, dev=1)), dict(rows=S(u8, 6, 256, dev=0))):
        with pytest.raises(B.SpiceError):
            B.spice_sort_tokens(**{**base, **with_rows, **bad})
    rows, pos, gate = S(bf, 6, 64), S(i32, 3, 2), S(f32, 3, 2)
    B.spice_combine_tokens(rows, pos, S(f32, 3, 64), gate, accumulate=True)
    assert calls[-1][2] == (P, 0, 6, P, P, 3, 2, 64, B.OUT_F32_ADD, P)
    for args in ((rows, pos, S(bf, 3, 64), gate, True), (rows, pos, S(torch.float16, 3, 64)), (S(torch.float16, 6, 64), pos, S(bf, 3, 64)),
                 (rows, pos, S(bf, 2, 64)), (rows, pos, S(bf, 3, 64), S(f32, 3, 3)), (rows, S(torch.int64, 3, 2), S(bf, 3, 64))):
        with pytest.raises(B.SpiceError):
            B.spice_combine_tokens(*args)
    dy = S(f32, 3, 64)
    B.spice_combine_tokens_grad(dy, rows, pos, gate, S(bf, 6, 64), gate)
    assert calls[-1][2] == (P, 1, P, 0, 6, P, P, 3, 2, 64, P, P)
    B.spice_combine_tokens_grad(dy, None, pos, None, S(f32, 7, 64))
    assert calls[-1][2] == (P, 1, None, 1, 7, P, None, 3, 2, 64, P, None)
    for args in ((dy, rows, pos, gate), (dy, None, pos, gate, None, gate), (dy, rows, pos, gate, S(f32, 6, 64)), (dy, None, pos, gate, S(bf, 6, 64), gate),
                 (dy, rows, S(i32, 4, 2), gate, S(bf, 6, 64))):
        with pytest.raises(B.SpiceError):
            B.spice_combine_tokens_grad(*args)
    B.spice_quantize_e4m3_blocks(S(bf, 5, 200, 136), S(u8, 5, 200, 136), S(f32, 5, 2, 2), 128)
    assert calls[-1][2] == (P, 5, 200, 136, 128, P, P)
    for args in ((S(bf, 200, 136), S(u8, 200, 136), S(f32, 2, 2), 1), (S(bf, 200, 136), S(u8, 200, 136), S(f32, 2, 2), 64),
                 (S(bf, 136), S(u8, 136), S(f32, 2)), (S(f32, 2, 136), S(u8, 2, 136), S(f32, 2, 2))):
        with pytest.raises(B.SpiceError):
            B.spice_quantize_e4m3_blocks(*args)
    x, xs = S(u8, 3, 144), S(f32, 3, 2)
    B.spice_gemm_e4m3_blocks(x, xs, S(u8, 200, 144), S(f32, 2, 2), S(bf, 3, 200))
    assert calls[-1][2] == (P, P, P, P, None, 1, 3, 200, 144, B.OUT_BF16, P, None)
    B.spice_gemm_e4m3_blocks(x, xs, S(u8, 4, 200, 144), S(f32, 4, 2, 2), S(f32, 3, 200), S(i32, 5))
    assert calls[-1][2] == (P, P, P, P, P, 4, 3, 200, 144, B.OUT_F32, P, None)
    B.spice_swiglu_e4m3_blocks(x, xs, S(u8, 4, 512, 144), S(f32, 4, 4, 2), S(u8, 3, 256), S(f32, 3, 2), S(i32, 5))
    assert calls[-1][2] == (P, P, P, P, P, 4, 3, 256, 144, P, P, None)
    n = len(calls)
    for args in ((x, xs, S(u8, 4, 200, 144), S(f32, 4, 2, 2), S(bf, 3, 200)), (x, xs, S(u8, 200, 144), S(f32, 2, 2), S(bf, 3, 200), S(i32, 2)),
                 (x, S(f32, 3, 1), S(u8, 200, 144), S(f32, 2, 2), S(bf, 3, 200)), (x, xs, S(u8, 200, 144), S(f32, 1, 2), S(bf, 3, 200)),
                 (x, xs, S(u8, 200, 144, dev=-1), S(f32, 2, 2), S(bf, 3, 200)), (x, xs, S(u8, 4, 200, 144), S(f32, 4, 2, 2), S(bf, 3, 200), S(i32, 4)),
                 (x, xs, S(u8, 200, 128), S(f32, 2, 1), S(bf, 3, 200)), (x, xs, S(u8, 144), S(f32, 2, 2), S(bf, 3, 200)),
                 (x, xs, S(u8, 200, 144), S(f32, 2, 2), S(bf, 3, 200), None, True)):
        with pytest.raises(B.SpiceError):
            B.spice_gemm_e4m3_blocks(*args)
    with pytest.raises(B.SpiceError):
        B.spice_swiglu_e4m3_blocks(x, xs, S(u8, 272, 144), S(f32, 3, 2), S(u8, 3, 136), S(f32, 3, 2))
    assert len(calls) == n
