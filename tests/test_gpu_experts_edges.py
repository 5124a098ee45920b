"""Tokens sorted by expert and E4M3 blocks where several threads call at once, and at the ends of the ranges that the calls take."""
import threading

import pytest
import torch

from paper_2608_21240_b200 import binding as B
from tests.test_gpu_e4m3_blocks import plain_quantiser
from tests.test_gpu_sort_tokens import make_idx, plain_sort

pytestmark = pytest.mark.gpu

bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def test_sorts_of_different_numbers_of_experts_from_several_threads():
    """Kernels that need different amounts of shared memory, launched from host threads at once on streams of their own (the entry point
    itself, called as fast as it goes: another thread has to come in between two steps of a call)."""
    T, K = 1025, 2
    failed, gate, call = [], threading.Barrier(4), B.lib().spice_sort_tokens

    def work(N, seed):
        try:
            idx = make_idx(T, K, N, seed)
            want = [w.cuda() for w in plain_sort(idx, N)]
            stream = torch.cuda.Stream()
            got = [torch.empty(N + 1, dtype=i32, device="cuda"), torch.empty_like(idx), torch.empty(T * K, dtype=i32, device="cuda")]
            torch.cuda.synchronize()
            args = (idx.data_ptr(), T, K, N, *(g.data_ptr() for g in got), None, 0, None, None, 0, None, stream.cuda_stream)
            gate.wait()
            codes = set(call(*args) for _ in range(20000))
            stream.synchronize()
            assert codes == {0}, codes
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        except Exception as e:   # noqa: BLE001 (reported by the test's own thread)
            failed.append((N, repr(e)))

    threads = [threading.Thread(target=work, args=(N, i)) for i, N in enumerate((1024, 400, 1000, 512))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


def test_quantiser_of_the_most_rows():
    """2^31 - 1 rows: the places of blocks and rows fill 32 bits.  All zeros but for some blocks at the ends and in the middle."""
    rows = 2 ** 31 - 1
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 52 GB of device memory")
    w = torch.zeros(rows, 8, dtype=bf, device="cuda")
    q = torch.full((rows, 8), 0x55, dtype=u8, device="cuda")
    blocks = 2 ** 24
    scale = torch.full((blocks, 1), -3.0, device="cuda")
    filled = [0, 1, blocks // 2, blocks - 2, blocks - 1]
    for i in filled:
        part = w[i * 128:(i + 1) * 128]
        part.copy_(torch.randn(part.shape, device="cuda"))
    B.spice_quantize_e4m3_blocks(w, q, scale, 128)
    torch.cuda.synchronize()
    for i in filled:
        want_q, want_s = plain_quantiser(w[i * 128:(i + 1) * 128], 128)
        assert torch.equal(q[i * 128:(i + 1) * 128].view(torch.float8_e4m3fn).double(), want_q)
        assert abs(float(scale[i]) - float(want_s)) <= 2.0 ** -24 * float(want_s)
        q[i * 128:(i + 1) * 128] = 0
        scale[i] = 1
    assert (scale == 1).all()
    flat = q.view(-1)
    for a in range(0, flat.numel(), 1 << 32):
        assert not flat[a:a + (1 << 32)].any()
    del w, q, scale, flat
    torch.cuda.empty_cache()


def test_sort_with_the_widest_scales():
    """2^31 - 1 scales a row: the columns behind the last one do not fit 32 bits with a sign."""
    n = 2 ** 31 - 1
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 18 GB of device memory")
    xs = torch.zeros(1, n, device="cuda")
    xs[0, -300:] = torch.arange(300.0, device="cuda")
    xs[0, ::1 << 20] = 5.0
    rs = torch.full((1, n), -1.0, device="cuda")
    x = torch.randn(1, 8, device="cuda").to(bf)
    rows = torch.zeros(1, 8, dtype=bf, device="cuda")
    off, pos, entry = (torch.full(s, -7, dtype=i32, device="cuda") for s in ((4,), (1, 1), (1,)))
    B.spice_sort_tokens(torch.full((1, 1), 2, dtype=i32, device="cuda"), off, pos, entry, x, rows, xs, rs)
    torch.cuda.synchronize()
    assert off.tolist() == [0, 0, 0, 1] and pos.tolist() == [[0]] and entry.tolist() == [0]
    assert torch.equal(rows, x) and torch.equal(rs, xs)
    del xs, rs
    torch.cuda.empty_cache()
