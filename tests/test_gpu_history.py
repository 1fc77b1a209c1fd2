"""The history operators together, as a program uses them: a stream whose keys and values are appended batch by batch and read by
later roots, training over the same slots, and the boundary refresh in 8 and 4 bits."""
import numpy as np
import pytest
import torch

from oracle import history as oh
from oracle import refresh as orf
from paper_2608_16305_b200 import workload as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    from paper_2608_16305_b200 import binding, history
    binding.load_library()
    return history


def _stream(events=3000):
    cfg = wl.scaled(wl.CONFIGS["tiny"], num_events=events)
    s = wl.make_stream(cfg)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return cfg, s, dev(s.indptr), dev(s.nbr), dev(s.eid), dev(s.ts)


@pytest.mark.parametrize("bits,window,sinks,dt", [(4, 10, 2, torch.float32), (8, 20, 0, torch.bfloat16), (4, 200, 4, torch.float16)])
def test_stream_scored_from_the_cache_as_it_grows(H, bits, window, sinks, dt):
    """Batch after batch: score its roots on what came before, then append its own entries.  Rows of later batches hold NaN scales
    until they are written: nothing reads them."""
    cfg, s, indptr, nbr, eid, ts = _stream()
    KV, heads, D = 2, 4, 25
    h = H.EventHistory(indptr, nbr, eid, ts, KV, D, window, sinks, bits)
    h.k.scales.fill_(float("nan"))
    h.v.scales.fill_(float("nan"))
    rng = np.random.default_rng(bits)
    P = ts.numel()
    k, v = (rng.standard_normal((P, KV, D)).astype(np.float32) for _ in range(2))
    kq, vq = (oh.dequantise(*oh.quantise(x, bits)) for x in (k, v))
    bias = H.TimeBias.logarithmic(heads, 12, 1.0, 3000.0)
    bias.table.normal_()
    kd, vd = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    table, bounds = bias.table.double().cpu().numpy(), bias.bounds.cpu().numpy()
    checked = 0
    for b in range(cfg.num_batches):
        e0, e1 = b * cfg.batch, min((b + 1) * cfg.batch, cfg.num_events)
        nodes_h = np.concatenate([s.src[e0:e1], s.dst[e0:e1], s.neg[e0:e1]])
        # all roots of a batch ask at the time of its first event: they see earlier batches only
        times_h = np.full(len(nodes_h), s.t[e0])
        nodes, times = torch.from_numpy(nodes_h).int().cuda(), torch.from_numpy(times_h).cuda()
        q = torch.randn(len(nodes_h), heads, D, generator=torch.Generator().manual_seed(b)).to(dt).cuda()
        out = h.attend(q, nodes, times, bias)
        assert out.isfinite().all()
        if b % 5 == 4:
            qd, od = q.double().cpu().numpy(), out.double().cpu().numpy()
            for i in rng.integers(0, len(nodes_h), 12):
                a = int(s.indptr[nodes_h[i]])
                _, recent, first = oh.visible(s.ts, a, int(s.indptr[nodes_h[i] + 1]), times_h[i], window, sinks)
                at = [a + j for j in recent + first]
                bk = [oh.bucket(bounds, times_h[i] - s.ts[j]) for j in at]
                ref = oh.attend(qd[i:i + 1], kq, vq, [at], table, [bk], D ** -0.5)[0]
                # fp32 sums of a few hundred terms (2^-15 of the largest value) and half a step of the output
                tol = 2.0 ** -15 * (np.abs(vq[at]).max() if at else 0) + torch.finfo(dt).eps / 2 * np.abs(ref)
                assert (np.abs(od[i] - ref) <= tol).all()
                checked += len(at)
        places = h.places(e0, e1)
        assert sorted(eid[places].cpu().tolist()) == sorted(list(range(e0, e1)) * 2)
        h.append(places, kd[places], vd[places])
    assert h.status() == 0 and checked > 100 and not h.k.scales.isnan().any()


def test_training_form_agrees_with_the_scoring_form(H):
    """Slots gathered from rows that the cache holds exactly: both forms see the same entries, keys and values."""
    cfg, s, indptr, nbr, eid, ts = _stream()
    KV, heads, D, window, sinks = 2, 2, 50, 12, 3
    h = H.EventHistory(indptr, nbr, eid, ts, KV, D, window, sinks, 8)
    P = ts.numel()
    g = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randint(-127, 128, (P, KV, D), generator=g, device="cuda").float() for _ in range(2))
    k[..., 0] = v[..., 0] = 127                                # scale 1: integers are held exactly
    every = torch.arange(P, device="cuda")
    h.append(every, k, v)
    R = 900
    nodes = torch.randint(0, cfg.num_nodes, (R,), generator=g, device="cuda", dtype=torch.int32)
    times = torch.rand(R, generator=g, device="cuda", dtype=torch.float64) * float(s.t[-1]) * 1.1
    q = 0.01 * torch.randn(R, heads, D, generator=g, device="cuda")
    bias = H.TimeBias.logarithmic(heads, 9, 2.0, 2000.0)
    bias.table.normal_(generator=g)
    served = h.attend(q, nodes, times, bias)
    sl = h.slots(nodes, times)
    # places of the slots: the entry of that event in the root's own slice
    at = torch.zeros_like(sl.eid, dtype=torch.int64)
    ptr, ev = s.indptr, s.eid
    for r in range(R):
        n = int(nodes[r])
        of = {}
        for p in range(int(ptr[n]), int(ptr[n + 1])):
            of.setdefault(int(ev[p]), []).append(p)
        for j in range(int(sl.cnt[r])):
            at[r, j] = of[int(sl.eid[r, j])].pop(0)
    trained = H.slot_attention(q, k[at], v[at], sl.cnt, bias, times, sl.ts)
    # both in fp32 on values up to 127: 2^-15 of them covers sums of 15 slots and 50 columns on either side
    assert (served - trained).abs().max() <= 2 * 127 * 2.0 ** -15
    assert h.status() == 0 and served[sl.cnt == 0].abs().sum() == 0


def test_gradients_through_autograd(H):
    """slot_attention inside a torch program: gradients of all four leaves equal those of the formula in 64 bits, also when the leaves are
    views, gradients are accumulated, and an eager graph lives while the step is captured."""
    R, S, heads, KV, D = 20, 6, 4, 2, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda")
    q, k, v = mk(heads, R, D).transpose(0, 1).requires_grad_(), mk(R, S, KV, D).requires_grad_(), mk(R, KV, S, D).transpose(1, 2).requires_grad_()
    bias = H.TimeBias(mk(heads, 5).requires_grad_(), torch.tensor([1.0, 5.0, 20.0, 80.0], dtype=torch.float64, device="cuda"))
    cnt = torch.randint(0, S + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    times = torch.full((R,), 200.0, dtype=torch.float64, device="cuda")
    ts = 200.0 * torch.rand(R, S, generator=g, device="cuda", dtype=torch.float64)
    w = mk(R, heads, D)
    out = H.slot_attention(q, k, v, cnt, bias, times, ts)
    (out * w).sum().backward()
    bk = np.searchsorted(bias.bounds.cpu().numpy(), (times[:, None] - ts).cpu().numpy(), side="right")
    d = lambda t: t.detach().double().cpu().numpy()
    ref = oh.slot_attend_backward(d(q), d(k), d(v), cnt.cpu().numpy(), d(bias.table), bk, D ** -0.5, d(w))
    for t, r in zip((q, k, v, bias.table), ref):
        assert np.abs(d(t.grad) - r).max() <= 2.0 ** -17 * max(1.0, np.abs(r).max())      # fp32 sums of under a hundred terms
    first = [t.grad.clone() for t in (q, k, v, bias.table)]
    (H.slot_attention(q, k, v, cnt, bias, times, ts) * w).sum().backward()
    for t, f in zip((q, k, v, bias.table), first):
        assert torch.equal(t.grad, 2 * f)
    # no bias, and leaves that need no gradient
    out = H.slot_attention(q.detach().contiguous(), k, v.detach(), cnt)
    assert torch.autograd.grad(out.sum(), k)[0].abs().sum() == 0 or out.requires_grad


def test_training_step_in_a_graph(H):
    """Forward and backward captured on leaves of their own, replayed while eager graphs of other leaves live."""
    R, S, heads, KV, D = 30, 8, 2, 2, 50
    g = torch.Generator(device="cuda").manual_seed(4)
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda")
    q, k, v = (t.requires_grad_() for t in (mk(R, heads, D), mk(R, S, KV, D), mk(R, S, KV, D)))
    bias = H.TimeBias(mk(heads, 4).requires_grad_(), torch.tensor([1.0, 5.0, 20.0], dtype=torch.float64, device="cuda"))
    cnt = torch.full((R,), S, dtype=torch.int32, device="cuda")
    times, ts = torch.full((R,), 50.0, dtype=torch.float64, device="cuda"), 50 * torch.rand(R, S, generator=g, device="cuda", dtype=torch.float64)
    leaves = (q, k, v, bias.table)
    step = lambda: torch.autograd.grad(H.slot_attention(q, k, v, cnt, bias, times, ts).square().sum(), leaves)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        static = step()
    with torch.no_grad():
        for t in leaves:
            t.copy_(mk(*t.shape))
    graph.replay()
    for a, b in zip(static, step()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("d", [100, 172, 256])
def test_quantised_refresh_between_emulated_workers(H, bits, d):
    """Three workers' refreshes run one after the other on one device, the all-to-all written out as segment copies."""
    from paper_2608_16305_b200 import distributed as D
    rng = np.random.default_rng(d)
    P, N, Q = 3, 400, 2
    owner = rng.integers(0, P, N).astype(np.int32)
    sets = [[sorted(rng.choice(np.nonzero(owner != p)[0], 60, replace=False).tolist()) for p in range(P)] for _ in range(Q)]
    sync = np.zeros((P, Q, N), np.uint8)
    for q in range(Q):
        for p in range(P):
            sync[p, q, sets[q][p]] = 1
    n_sync = sync.sum(2).astype(np.int32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    plans = [D.RefreshPlan(dev(sync), dev(owner), n_sync, P, me) for me in range(P)]
    ref = [D.QuantisedRefresh(pl, d, bits) for pl in plans]
    mem_h = [rng.standard_normal((N, d)).astype(np.float32) for _ in range(P)]
    lu_h = [rng.random(N) * 1e9 for _ in range(P)]
    mem, lu = [dev(m) for m in mem_h], [dev(t) for t in lu_h]
    heads = ref[0].send.heads
    for q in range(Q):
        for me in range(P):
            ref[me].pack(q, mem[me], lu[me])
        for me in range(P):
            for o in range(P):
                seg = ref[o].send.data[int(plans[o].send_off[q, me]):int(plans[o].send_off[q, me + 1])]
                ref[me].recv.data[int(plans[me].recv_off[q, o]):int(plans[me].recv_off[q, o + 1])] = seg
        for me in range(P):
            assert ref[me].unpack(q, mem[me], lu[me]) == len(sets[q][me])
        # the oracle's refresh on rows that went through the quantiser
        sent = [oh.dequantise(*oh.quantise(m.reshape(N, heads, -1), bits)).reshape(N, d).astype(np.float32) for m in mem_h]
        new_m, new_t = orf.boundary_refresh([s.copy() for s in sent], [t.copy() for t in lu_h], sets[q], owner)
        for me in range(P):
            got = np.zeros(N, bool)
            got[sets[q][me]] = True
            mem_h[me] = np.where(got[:, None], new_m[me], mem_h[me]).astype(np.float32)
            lu_h[me] = np.where(got, new_t[me], lu_h[me])
            assert np.array_equal(mem[me].cpu().numpy(), mem_h[me]) and np.array_equal(lu[me].cpu().numpy(), lu_h[me])
            assert int(ref[me].status.item()) == 0
    if d == 100:
        assert ref[0].send.record_bytes == (144 if bits == 8 else 80)


def test_calls_on_a_side_stream(H):
    """The operators follow torch's current stream."""
    cfg, s, indptr, nbr, eid, ts = _stream(800)
    h = H.EventHistory(indptr, nbr, eid, ts, 2, 50, 10, 2, 4)
    P = ts.numel()
    k, v = torch.randn(P, 2, 50, device="cuda"), torch.randn(P, 2, 50, device="cuda")
    nodes = torch.arange(300, dtype=torch.int32, device="cuda")
    times = torch.full((300,), 1e9, dtype=torch.float64, device="cuda")
    q = torch.randn(300, 2, 50, device="cuda")
    every = torch.arange(P, device="cuda")
    h.append(every, k, v)
    want = h.attend(q, nodes, times)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h2 = H.EventHistory(indptr, nbr, eid, ts, 2, 50, 10, 2, 4)
        torch.cuda._sleep(20_000_000)                          # work of this stream that the calls have to stay behind
        k2, v2 = k.clone(), v.clone()
        h2.append(every, k2, v2)
        got = h2.attend(q, nodes, times)
    side.synchronize()
    assert torch.equal(got, want)


def test_calls_that_overlap_on_two_streams(H):
    """The same caches and inputs read by calls on two streams at once, each with outputs (and scratch) of its own."""
    from paper_2608_16305_b200 import binding as B
    cfg, s, indptr, nbr, eid, ts = _stream()
    h = H.EventHistory(indptr, nbr, eid, ts, 2, 50, 300, 2, 4)
    P, R, S = ts.numel(), 700, 40
    g = torch.Generator(device="cuda").manual_seed(9)
    mk = lambda *sh: torch.randn(*sh, generator=g, device="cuda")
    h.append(torch.arange(P, device="cuda"), mk(P, 2, 50), mk(P, 2, 50))
    nodes = torch.randint(0, cfg.num_nodes, (R,), generator=g, device="cuda", dtype=torch.int32)
    times = torch.full((R,), 1e9, dtype=torch.float64, device="cuda")
    bias = H.TimeBias.logarithmic(2, 16, 1.0, 3000.0)
    bias.table.normal_(generator=g)
    q, k, v, do = mk(R, 2, 50), mk(R, S, 2, 50), mk(R, S, 2, 50), mk(R, 2, 50)
    cnt = torch.full((R,), S, dtype=torch.int32, device="cuda")
    slot_ts = 1e9 - torch.cumsum(10 * torch.rand(R, S, generator=g, device="cuda", dtype=torch.float64), 1)

    def run():
        out = h.attend(q, nodes, times, bias)
        grads = [torch.empty_like(t) for t in (q, k, v, bias.table)]
        scratch = torch.empty(B.slot_attend_scratch(R, 2, 16), device="cuda")
        B.slot_attend_backward(q, k, v, cnt, do, *grads[:3], bias=bias.table, bounds=bias.bounds, times=times, ts=slot_ts, dbias=grads[3],
                               scratch=scratch)
        return [out] + grads + [scratch]
    want = run()[:5]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(10):
        for st in streams:
            with torch.cuda.stream(st):
                got.append(run())
    torch.cuda.synchronize()
    for res in got:
        for a, b in zip(res, want):
            assert torch.equal(a, b)


def test_empty_batches_and_histories(H):
    cfg, s, indptr, nbr, eid, ts = _stream(400)
    h = H.EventHistory(indptr, nbr, eid, ts, 2, 50, 10, 2, 8)
    e = lambda *sh, **kw: torch.empty(*sh, device="cuda", **kw)
    assert h.attend(e(0, 2, 50), e(0, dtype=torch.int32), e(0, dtype=torch.float64)).shape == (0, 2, 50)
    assert h.slots(e(0, dtype=torch.int32), e(0, dtype=torch.float64)).nbr.shape == (0, 12)
    h.append(e(0, dtype=torch.int64), e(0, 2, 50), e(0, 2, 50))
    # a graph without entries, and one without nodes
    for ptr in (torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")):
        none = H.EventHistory(ptr, e(0, dtype=torch.int32), e(0, dtype=torch.int32), e(0, dtype=torch.float64), 2, 50, 10, 2, 4)
        nodes, times = torch.arange(3, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.float64, device="cuda")
        bias = H.TimeBias.logarithmic(2, 4, 1.0, 9.0)
        assert not none.attend(torch.ones(3, 2, 50, device="cuda"), nodes, times, bias).any()
        assert none.slots(nodes, times).cnt.tolist() == [0, 0, 0] and none.status() == (0 if ptr.numel() > 1 else 4)
    assert h.status() == 0


def test_one_source_for_several_places_and_roots_that_share_a_history(H):
    from paper_2608_16305_b200 import binding as B
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = torch.randn(5, 2, 50, device="cuda")
    k, v = B.RowCache(40, 2, 50, 8), B.RowCache(40, 2, 50, 8)
    src = torch.tensor([3, 3, 3, 1] * 10, device="cuda")
    B.cache_write(k, x, st, src=src)
    B.cache_write(v, x, st, src=src)
    assert torch.equal(k.codes[0], k.codes[1]) and torch.equal(k.codes[0], k.codes[36])
    q = torch.randn(1, 2, 50, device="cuda").expand(64, 2, 50).contiguous()
    first, length = torch.full((64,), 4, dtype=torch.int64, device="cuda"), torch.full((64,), 33, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    B.cached_attend(q, k, v, first, length, 20, 3, out, st)
    assert torch.equal(out, out[:1].expand_as(out)) and int(st.item()) == 0
    rows = torch.empty(6, 100, device="cuda")
    B.cache_read(k, rows, st, src=torch.tensor([0, 0, 4, 4, 3, 3], device="cuda"))
    assert torch.equal(rows[0], rows[1]) and torch.equal(rows[0], rows[2]) and torch.equal(rows[4], rows[5])


def test_quantised_refresh_over_a_one_rank_communicator():
    """The all-to-all of records on a real NCCL communicator (one rank: rows sent to itself) between the cache's kernels."""
    import os
    import socket
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = r"""
import os, sys, numpy as np, torch, torch.distributed as dist
sys.path.insert(0, %r)
from oracle import history as oh
from paper_2608_16305_b200 import distributed as D
torch.cuda.set_device(0)
dist.init_process_group("nccl", rank=0, world_size=1, init_method="tcp://127.0.0.1:" + os.environ["PORT"],
                        device_id=torch.device("cuda", 0))
N, n = 5000, 1200
rng = np.random.default_rng(0)
perm = rng.permutation(N)
src, dst = perm[:n].astype(np.int32), perm[n:2 * n].astype(np.int32)
for d, bits in ((100, 8), (100, 4), (344, 4)):
    mem_h, lu_h = rng.standard_normal((N, d)).astype(np.float32), rng.random(N) * 1e5
    mem, lu = torch.from_numpy(mem_h).cuda(), torch.from_numpy(lu_h).cuda()
    plan = D.RefreshPlan.from_lists(torch.from_numpy(dst[None]).cuda(), np.array([[0, n]]), torch.from_numpy(src[None]).cuda(),
                                    np.array([[0, n]]), 1, 0)
    ref = D.QuantisedRefresh(plan, d, bits)
    ref.run(0, mem, lu)
    want, t = mem_h.copy(), lu_h.copy()
    want[dst] = oh.dequantise(*oh.quantise(mem_h[src].reshape(n, ref.send.heads, -1), bits)).reshape(n, d)
    t[dst] = lu_h[src]
    assert int(ref.status.item()) == 0 and ref.rows_sent == n and ref.rows_received == n
    assert np.array_equal(mem.cpu().numpy(), want) and np.array_equal(lu.cpu().numpy(), t)
dist.destroy_process_group()
print("ok")
""" % root
    sock = socket.socket()
    sock.bind(("127.0.0.1", 0))
    port = sock.getsockname()[1]
    sock.close()
    p = subprocess.run([sys.executable, "-c", code], env=dict(os.environ, PORT=str(port), NCCL_NVLS_ENABLE="0"), capture_output=True, timeout=240)
    assert p.returncode == 0 and b"ok" in p.stdout, p.stderr.decode()[-3000:]
