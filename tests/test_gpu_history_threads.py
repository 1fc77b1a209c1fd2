"""The history entry points are stateless: calls from several host threads at once do not meet, whatever each asks of the device."""
import ctypes as C
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


class _Backward:
    """Arguments of one tgnn_slot_attend_backward call through ctypes, which lets other threads run meanwhile."""

    def __init__(self, lib, n, slots, heads, dim, buckets):
        g = torch.Generator(device="cuda").manual_seed(heads)
        mk = lambda *s: torch.randn(*s, generator=g, device="cuda")
        q, do, k, v = mk(n, heads, dim), mk(n, heads, dim), mk(n, slots, heads, dim), mk(n, slots, heads, dim)
        cnt = torch.full((n,), slots, dtype=torch.int32, device="cuda")
        bias = [None] * 4 if not buckets else [mk(heads, buckets), torch.arange(1.0, buckets, dtype=torch.float64, device="cuda"),
                                               torch.full((n,), float(buckets), dtype=torch.float64, device="cuda"),
                                               buckets * torch.rand(n, slots, generator=g, device="cuda", dtype=torch.float64)]
        self.out = [torch.empty_like(t) for t in (q, k, v)] + ([torch.empty_like(bias[0])] if buckets else [None])
        scratch = torch.empty(lib.tgnn_slot_attend_scratch(n, heads, buckets), device="cuda") if buckets else None
        p = lambda t: None if t is None else t.data_ptr()
        self.keep = (q, k, v, cnt, bias, do, scratch)
        self.err = C.create_string_buffer(256)
        self.stream = torch.cuda.Stream()
        self.lib = lib
        self.args = (p(q), p(k), p(v), 0, n, slots, heads, heads, dim, p(cnt), p(bias[0]), buckets, p(bias[1]), p(bias[2]), p(bias[3]), dim ** -0.5,
                     p(do), *map(p, self.out), p(scratch), self.stream.cuda_stream, C.addressof(self.err), len(self.err))

    def call(self):
        rc = self.lib.tgnn_slot_attend_backward(*self.args)
        return None if rc == 0 else (rc, self.err.value.decode())


def test_calls_of_two_threads_that_need_different_amounts_of_shared_memory():
    """Two threads run the backward pass of one kernel, one with a small row of slots per block (49 KB of shared memory), one with a wide table of
    the bias (77 KB): neither's launch may depend on what the other has asked for since."""
    from paper_2608_16305_b200 import binding
    lib = binding.load_library()
    jobs = [_Backward(lib, 2400, 192, 8, 16, 0), _Backward(lib, 24, 30, 64, 16, 128)]
    torch.cuda.synchronize()
    want = []
    for j in jobs:
        assert j.call() is None
        torch.cuda.synchronize()
        want.append([None if t is None else t.clone() for t in j.out])
    failed, start = [], threading.Barrier(2)

    def work(j):
        torch.cuda.set_device(0)
        start.wait()
        for i in range(4000):
            bad = j.call()
            if bad is not None:
                failed.append((i, bad))
                return
            if i % 200 == 199:
                j.stream.synchronize()
    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for j, w in zip(jobs, want):
        for a, b in zip(j.out, w):
            assert a is None or torch.equal(a, b)
