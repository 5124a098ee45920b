"""Host-side checks of the steps next to the layer (residual norm, 8-bit integer rows and products, routing by scores): every
refusal answers without a device and launches nothing; a call without rows is fine."""
import ctypes as C

import pytest
import torch

from paper_2608_21240_b200 import binding as B

OK, INVALID, SHAPE = 0, 1, 2
P, Q = 4096, 8192          # 16-byte aligned stand-ins for device addresses: no refused call reads them
BIG = 1 << 20


def norm(x=P, delta=None, delta32=None, weight=P, eps=1e-6, T=1, d=64, h=P, q=P, scale=P):
    return B.lib().spice_residual_rmsnorm(x, delta, delta32, weight, eps, T, d, h, q, scale, None)


def test_residual_rmsnorm_refusals():
    assert norm(T=0) == OK and norm(T=0, x=None) == OK
    for bad in (dict(T=-1), dict(d=0), dict(d=12), dict(d=-8), dict(eps=-1.0), dict(eps=float("nan")), dict(h=None, q=None),
                dict(scale=None), dict(delta=P, delta32=P), dict(x=None), dict(weight=None), dict(x=P + 8), dict(delta=P + 2),
                dict(delta32=P + 4), dict(weight=P + 2), dict(h=P + 8), dict(q=P + 4), dict(scale=P + 2)):
        assert norm(**bad) == INVALID, bad
    assert norm(d=32776) == SHAPE


def rows(w=P, n=1, cols=64, q=P, scale=P):
    return B.lib().spice_quantize_i8_rows(w, n, cols, q, scale, None)


def test_quantize_i8_rows_refusals():
    assert rows(n=0) == OK
    for bad in (dict(n=-1), dict(cols=0), dict(cols=9), dict(w=None), dict(q=None), dict(scale=None), dict(w=P + 8), dict(q=P + 4),
                dict(scale=P + 1)):
        assert rows(**bad) == INVALID, bad
    assert rows(cols=32776) == SHAPE and rows(n=1 << 31) == SHAPE


def gemm(x=P, xs=P, w=P, ws=P, T=1, n=64, k=64, out=0, y=P, status=None):
    return B.lib().spice_gemm_i8(x, xs, w, ws, T, n, k, out, y, status, None)


def swiglu(x=P, xs=P, w=P, ws=P, T=1, n=64, k=64, y=P, status=None):
    return B.lib().spice_swiglu_i8(x, xs, w, ws, T, n, k, y, status, None)


@pytest.mark.parametrize("call", [gemm, swiglu])
def test_product_refusals(call):
    assert call(T=0) == OK
    for bad in (dict(T=-1), dict(n=0), dict(n=12), dict(k=0), dict(k=24), dict(k=8), dict(x=None), dict(xs=None), dict(w=None),
                dict(ws=None), dict(y=None), dict(x=P + 8), dict(w=P + 8), dict(ws=P + 4), dict(y=P + 8), dict(xs=P + 2),
                dict(status=P + 2)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(k=131072), dict(n=(1 << 24) + 8), dict(T=(1 << 24) + 1)):
        assert call(**bad) == SHAPE, bad
    if call is gemm:
        assert call(out=3) == INVALID and call(out=-1) == INVALID


def route(logits=P, bias=None, T=1, N=64, K=6, score=0, G=1, top=1, pair=0, norm=1, scale=1.0, idx=P, gate=P):
    return B.lib().spice_route_scored(logits, bias, T, N, K, score, G, top, pair, norm, scale, idx, gate, None)


def test_route_scored_refusals():
    assert route(T=0) == OK
    for bad in (dict(T=-1), dict(score=2), dict(score=-1), dict(pair=2), dict(logits=None), dict(idx=None), dict(gate=None),
                dict(logits=P + 2), dict(bias=P + 1), dict(idx=P + 2), dict(gate=P + 3)):
        assert route(**bad) == INVALID, bad
    for bad in (dict(N=0), dict(N=1025), dict(K=0), dict(K=33), dict(N=4), dict(G=0), dict(G=3), dict(N=66, G=33), dict(G=8, top=0),
                dict(G=8, top=9), dict(N=16, G=8, top=2)):
        assert route(**bad) == SHAPE, bad


def test_binding_refuses_host_tensors_and_wrong_shapes():
    bf, i8, f32 = torch.bfloat16, torch.int8, torch.float32
    z = lambda *s, dtype: torch.zeros(*s, dtype=dtype)  # noqa: E731
    with pytest.raises(B.SpiceError):
        B.spice_residual_rmsnorm(z(2, 8, dtype=bf), z(8, dtype=bf), 1e-6, z(2, 8, dtype=i8), z(2, dtype=f32))
    with pytest.raises(B.SpiceError):
        B.spice_quantize_i8_rows(z(2, 8, dtype=bf), z(2, 8, dtype=i8), z(2, dtype=f32))
    with pytest.raises(B.SpiceError):
        B.spice_gemm_i8(z(2, 16, dtype=i8), z(2, dtype=f32), z(8, 16, dtype=i8), z(8, dtype=f32), z(2, 8, dtype=bf))
    with pytest.raises(B.SpiceError):
        B.spice_swiglu_i8(z(2, 16, dtype=i8), z(2, dtype=f32), z(16, 16, dtype=i8), z(16, dtype=f32), z(2, 8, dtype=bf))
    with pytest.raises(B.SpiceError):
        B.spice_route_scored(z(2, 8, dtype=f32), z(2, 2, dtype=torch.int32), z(2, 2, dtype=f32))
    for t, dtype, shape in ((z(2, 8, dtype=bf), bf, (2, 8)), (z(2, 8, dtype=bf), f32, (2, 8)), (z(2, 8, dtype=bf), bf, (2, 4)),
                            (z(8, 2, dtype=bf).t(), bf, (2, 8))):
        with pytest.raises(B.SpiceError, match="f: expected a contiguous"):
            B._addr("f", t, dtype, shape, 0)
    assert B._addr("f", None, bf, (2, 8), 0) is None


def test_calls_go_to_the_tensors_device_and_its_stream(monkeypatch):
    """With the tensors on device 1 while device 0 is current, the entry point runs inside a switch to device 1 and gets that
    device's current stream (or the stream that was given); an error code becomes an exception."""
    log = []

    class Lib:
        def spice_gemm_i8(self, *args):
            log.append(("call", args))
            return 0

        def spice_swiglu_i8(self, *args):
            return 1

        def spice_status_string(self, code):
            return b"invalid argument"

    class On:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            log.append(("enter", self.dev))

        def __exit__(self, *exc):
            log.append(("exit", self.dev))

    class Stream:
        cuda_stream = 4242

    monkeypatch.setattr(B, "_lib", Lib())
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_current_raw_stream", lambda dev: 100 + dev)
    monkeypatch.setattr(torch.cuda, "device", On)
    B._call_on(1, "spice_gemm_i8", None, 7, 8)
    assert log == [("enter", 1), ("call", (7, 8, 101)), ("exit", 1)]
    log.clear()
    B._call_on(0, "spice_gemm_i8", Stream(), 7)
    assert log == [("call", (7, 4242))]
    with pytest.raises(B.SpiceError, match="spice_swiglu_i8: invalid argument"):
        B._call_on(0, "spice_swiglu_i8", None, 7)


def test_wait_limit_of_the_products_is_set_without_a_context():
    assert B.lib().spice_set_option(None, B.OPT_I8_WAIT_LIMIT, C.c_int64(1 << 22)) == OK
    for value in (-1, (1 << 30) + 1):
        assert B.lib().spice_set_option(None, B.OPT_I8_WAIT_LIMIT, C.c_int64(value)) == INVALID
    assert B.lib().spice_set_option(None, B.OPT_TC_WAIT_LIMIT, C.c_int64(5)) == INVALID
    with pytest.raises(B.SpiceError):
        B.spice_set_option(None, B.OPT_PATH, 0)


class Stand:
    """What the binding asks of a tensor."""

    def __init__(self, dtype, shape, dev):
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

    def data_ptr(self):
        return P


def test_operands_of_the_bulk_copies_are_not_taken_from_host_memory(monkeypatch):
    """Pinned host memory may take a product's results and hold its scales; the codes are read by bulk copies and have to be
    on the device."""
    calls = []
    monkeypatch.setattr(B, "_call_on", lambda dev, name, stream, *args: calls.append(name))
    i8, f32, bf = torch.int8, torch.float32, torch.bfloat16
    xq, wq = Stand(i8, (4, 64), 0), Stand(i8, (16, 64), 0)
    xs, ws = Stand(f32, (4,), -1), Stand(f32, (16,), -1)
    B.spice_gemm_i8(xq, xs, wq, ws, Stand(bf, (4, 16), -1))
    B.spice_swiglu_i8(xq, xs, wq, ws, Stand(bf, (4, 8), -1))
    assert calls == ["spice_gemm_i8", "spice_swiglu_i8"]
    for x, w in ((Stand(i8, (4, 64), -1), wq), (xq, Stand(i8, (16, 64), -1))):
        with pytest.raises(B.SpiceError):
            B.spice_gemm_i8(x, xs, w, ws, Stand(bf, (4, 16), 0))
        with pytest.raises(B.SpiceError):
            B.spice_swiglu_i8(x, xs, w, ws, Stand(bf, (4, 8), 0))
    assert len(calls) == 2
