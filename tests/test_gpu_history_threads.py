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


def test_python_threads_that_score_and_train_at_once():
    """Two Python threads on streams of their own through the public operators (the interpreter is free during a call): each gets what it gets alone."""
    from paper_2608_16305_b200 import history as H
    from paper_2608_16305_b200 import workload as wl
    import numpy as np
    cfg = wl.scaled(wl.CONFIGS["tiny"], num_events=2000)
    s = wl.make_stream(cfg)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    h = H.EventHistory(dev(s.indptr), dev(s.nbr), dev(s.eid), dev(s.ts), 2, 50, 1000, 2, 4)
    g = torch.Generator(device="cuda").manual_seed(5)
    mk = lambda *sh: torch.randn(*sh, generator=g, device="cuda")
    P, R, S = h.ts.numel(), 300, 30
    h.append(torch.arange(P, device="cuda"), mk(P, 2, 50), mk(P, 2, 50))
    nodes = torch.randint(0, cfg.num_nodes, (R,), generator=g, device="cuda", dtype=torch.int32)
    times = torch.full((R,), 1e9, dtype=torch.float64, device="cuda")
    bias = H.TimeBias.logarithmic(2, 16, 1.0, 3000.0)
    bias.table.normal_(generator=g)
    q, k, v = mk(R, 2, 50), mk(R, S, 2, 50).requires_grad_(), mk(R, S, 2, 50).requires_grad_()
    cnt = torch.full((R,), S, dtype=torch.int32, device="cuda")
    ts = 1e9 * torch.rand(R, S, generator=g, device="cuda", dtype=torch.float64)
    score = lambda: [h.attend(q, nodes, times, bias), h.attend(q[:3].contiguous(), nodes[:3], times[:3], bias)]
    train = lambda: list(torch.autograd.grad(H.slot_attention(q, k, v, cnt, bias, times, ts).square().sum(), (k, v)))
    want = [score(), train()]
    torch.cuda.synchronize()
    got, start = [[], []], threading.Barrier(2)

    def work(i, f):
        torch.cuda.set_device(0)
        start.wait()
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(100):
                got[i].append(f())
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=a) for a in ((0, score), (1, train))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for res, w in zip(got, want):
        assert len(res) == 100
        for r in res:
            assert all(torch.equal(a, b) for a, b in zip(r, w))


@pytest.mark.parametrize("roots,length", [(3, 40000), (3, 300), (200, 9000), (5000, 100)])
def test_every_launch_shape_captured(roots, length):
    """Clusters of 16 blocks and fewer, blocks and warps per unit, in a graph: what is asked of the device before a launch is allowed there."""
    from paper_2608_16305_b200 import binding as B
    P, st = length + 50, torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = B.RowCache(P, 1, 50, 4), B.RowCache(P, 1, 50, 4)
    g = torch.Generator(device="cuda").manual_seed(roots)
    B.cache_write(k, torch.randn(P, 1, 50, generator=g, device="cuda"), st)
    B.cache_write(v, torch.randn(P, 1, 50, generator=g, device="cuda"), st)
    q = torch.randn(roots, 1, 50, generator=g, device="cuda")
    first = torch.randint(0, 50, (roots,), generator=g, device="cuda")
    n = torch.full((roots,), length, dtype=torch.int32, device="cuda")
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        B.cached_attend(q, k, v, first, n, length, 0, out, st)
    for _ in range(2):
        q.normal_(generator=g)
        graph.replay()
        B.cached_attend(q, k, v, first, n, length, 0, again, st)
        assert torch.equal(out, again) and out.abs().sum() > 0
    assert int(st.item()) == 0
