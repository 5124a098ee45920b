"""Tokens sorted by expert and E4M3 blocks where several threads call at once, and at the ends of the ranges that the calls take."""
import threading

import pytest
import torch

from paper_2608_21240_b200 import binding as B
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
