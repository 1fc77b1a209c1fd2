"""Sampling with sinks and the quantised row cache on the GPU, bit for bit against the plain form."""
import numpy as np
import pytest
import torch

from oracle import history as oh

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def B():
    from paper_2608_16305_b200 import binding
    binding.load_library()
    return binding


def _dev(a, dt):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).cuda()


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def csr(rng, lens, ties=True):
    indptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    P = int(indptr[-1])
    ts = np.concatenate([np.sort(rng.integers(0, max(2 * n, 3), n).astype(np.float64) if ties else rng.random(n) * 1e6) for n in lens] or [[]])
    return indptr, rng.integers(0, len(lens), P).astype(np.int32), rng.integers(0, 1 << 30, P).astype(np.int32), ts


@pytest.mark.parametrize("window,sinks", [(10, 0), (0, 3), (1, 1), (5, 40), (64, 4), (33, 2), (4096, 7)])
def test_sample_window_bit_exact(B, window, sinks):
    """Slices of no, one, 31 to 34 and thousands of entries, equal times, roots before, on and behind all entries."""
    rng = np.random.default_rng(window * 100 + sinks)
    lens = [0, 1, 2, 31, 32, 33, 34, 65, 1056, 1057, 5000, 0]
    indptr, nbr, eid, ts = csr(rng, lens)
    nodes, times = [], []
    for n, m in enumerate(lens):
        s = ts[indptr[n]:indptr[n + 1]]
        for t in [-1.0, 0.0, np.inf, np.nan] + ([s[0], s[-1], s[m // 2], np.nextafter(s[m // 2], 1e9)] if m else []):
            nodes.append(n)
            times.append(t)
    ref = oh.sample_window(indptr, nbr, eid, ts, nodes, times, window, sinks)
    R, S = len(nodes), window + sinks
    out = [torch.full((R, S), -7, dtype=torch.int32, device="cuda"), torch.full((R, S), -7, dtype=torch.int32, device="cuda"),
           torch.full((R, S), -7.0, dtype=torch.float64, device="cuda"), torch.full((R,), -7, dtype=torch.int32, device="cuda"),
           torch.full((R,), -7, dtype=torch.int64, device="cuda"), torch.full((R,), -7, dtype=torch.int32, device="cuda")]
    g = [_dev(indptr, np.int64), _dev(nbr, np.int32), _dev(eid, np.int32), _dev(ts, np.float64)]
    nd, tm, st = _dev(nodes, np.int32), _dev(times, np.float64), _status()
    B.sample_window(*g, nd, tm, window, sinks, *out, st)
    for o, name in zip(out, ("nbr", "eid", "ts", "cnt", "first", "len")):
        assert np.array_equal(o.cpu().numpy(), ref[name]), name
    assert int(st.item()) == 0
    first, length = torch.empty_like(out[4]), torch.empty_like(out[5])
    B.sample_window(g[0], None, None, g[3], nd, tm, window, sinks, None, None, None, None, first, length, st)
    assert torch.equal(first, out[4]) and torch.equal(length, out[5])


def test_sample_window_agrees_with_most_recent_search(B):
    """Without sinks, the slots of tgnn_sample_recent."""
    rng = np.random.default_rng(5)
    N, k = 50, 12
    indptr, nbr, eid, ts = csr(rng, rng.integers(0, 200, N))
    g = [_dev(indptr, np.int64), _dev(nbr, np.int32), _dev(eid, np.int32), _dev(ts, np.float64)]
    R = 300
    nodes, times = _dev(rng.integers(0, N, R), np.int32), _dev(rng.integers(0, 400, R), np.float64)
    i32 = dict(dtype=torch.int32, device="cuda")
    a, b = ([torch.empty((R, k), **i32), torch.empty((R, k), **i32), torch.empty((R, k), dtype=torch.float64, device="cuda"),
             torch.empty(R, **i32)] for _ in range(2))
    lib = B.Tgnn(B.make_config(N, 32, 16, k, 2, max_events=100, max_roots=R))
    lib.set_graph(*g)
    lib.sample_recent(nodes, times, *a)
    B.sample_window(*g, nodes, times, k, 0, *b, None, None, _status())
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_sample_window_reports_what_lies_outside(B):
    indptr, nbr, eid, ts = csr(np.random.default_rng(1), [5, 6])
    g = [_dev(indptr, np.int64), _dev(nbr, np.int32), _dev(eid, np.int32), _dev(ts, np.float64)]
    first, length = torch.empty(4, dtype=torch.int64, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    for ptr, nodes, want in ((indptr, [0, -1, 2, 1], [5, 0, 0, 6]), ([0, 5, 99], [0, 1, 1, 0], [5, 0, 0, 5]),
                             ([0, 5, 2], [0, 1, 1, 0], [5, 0, 0, 5]), ([-3, 5, 11], [0, 1, 1, 0], [0, 6, 6, 0])):
        st = _status()
        B.sample_window(_dev(ptr, np.int64), None, None, g[3], _dev(nodes, np.int32), _dev([1e9] * 4, np.float64), 3, 1, None, None, None,
                        None, first, length, st)
        assert int(st.item()) == 4 and length.cpu().tolist() == want


def _plain_rows(rng, n, heads, dim, dt):
    x = rng.standard_normal((n, heads, dim)) * np.exp(rng.standard_normal((n, heads, 1)) * 3)
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[dt])


def _unpack(cache, dim):
    """Codes of the cache as integers, from its documented layout."""
    c = cache.codes.cpu().numpy()
    if cache.bits == 4:
        c = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:2], -1).astype(np.int64) - 8
    else:
        c = c.astype(np.int64) - 128
    return c[..., :dim], c[..., dim:]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,dim", [(1, 1), (2, 50), (1, 100), (4, 64), (3, 43), (2, 25), (1, 128), (2, 33), (5, 8), (2, 32), (1, 2)])
def test_cache_bit_exact(B, bits, dt, heads, dim):
    rng = np.random.default_rng(bits * 1000 + heads * 130 + dim)
    N, C, n = 517, 600, 211
    x = _plain_rows(rng, N, heads, dim, dt)
    times = torch.from_numpy(rng.random(N) * 1e9)
    src, dst = rng.permutation(N)[:n], rng.permutation(C)[:n]
    cache = B.RowCache(C, heads, dim, bits)
    before = cache.codes.random_(0, 256).cpu().numpy().copy()
    cache.scales.fill_(3.0)
    cache.times.fill_(-1.0)
    st = _status()
    B.cache_write(cache, x.cuda(), st, src=_dev(src, np.int64), dst=_dev(dst, np.int64), times=times.cuda())
    codes, s = oh.quantise(x.float().numpy()[src], bits)
    got, pad = _unpack(cache, dim)
    assert np.array_equal(got[dst], codes) and not pad[dst].any()
    assert np.array_equal(cache.scales.float().cpu().numpy()[dst], s, equal_nan=True)   # (wide fp16 rows hold infinities)
    assert np.array_equal(cache.times.cpu().numpy()[dst], times.numpy()[src])
    others = np.setdiff1d(np.arange(C), dst)
    assert np.array_equal(cache.codes.cpu().numpy()[others], before[others])            # rows that were not named stay
    assert (cache.scales.float().cpu().numpy()[others] == 3).all() and (cache.times.cpu().numpy()[others] == -1).all()
    for out in TYPES:
        rows = torch.full((N, heads, dim), 7.0, dtype=TYPES[out], device="cuda")
        t = torch.full((N,), 7.0, dtype=torch.float64, device="cuda")
        B.cache_read(cache, rows, st, src=_dev(dst, np.int32), dst=_dev(src, np.int32), times=t)
        want = torch.full((N, heads, dim), 7.0, dtype=TYPES[out])
        want[src] = torch.from_numpy(oh.dequantise(codes, s).astype(np.float32)).to(TYPES[out])
        torch.testing.assert_close(rows.cpu(), want, rtol=0, atol=0, equal_nan=True)
        tw = torch.full((N,), 7.0, dtype=torch.float64)
        tw[src] = times[src]
        assert torch.equal(t.cpu(), tw)
    assert int(st.item()) == 0


@pytest.mark.parametrize("bits", [4, 8])
def test_cache_ties_and_extremes(B, bits):
    """Halves between codes, groups at the ends of the range, zeros, infinities and NaN beside ordinary groups."""
    L = 7 if bits == 4 else 127
    D = 16
    rows = np.zeros((12, D), np.float32)
    rows[0, :6] = [L, 0.5, 1.5, 2.5, -0.5, -1.5]
    rows[1] = 3.4e38 * np.linspace(-1, 1, D)
    rows[2] = 2.0 ** -99 * np.linspace(-1, 1, D)
    rows[3] = 2.0 ** -101
    rows[4] = 1e-45
    rows[5] = 1.0
    rows[5, 3] = np.inf
    rows[6] = 1.0
    rows[6, 9] = np.nan
    rows[7, 15] = -np.inf
    rows[8] = -0.0
    rows[9] = np.nextafter(np.float32(1), np.float32(2))
    rows[10] = np.random.default_rng(0).integers(-2 * L, 2 * L + 1, D) / 2
    rows[10, 0] = L
    rows[11] = 65504.0
    cache, st = B.RowCache(12, 1, D, bits), _status()
    x = torch.from_numpy(rows).cuda()
    B.cache_write(cache, x, st)
    codes, s = oh.quantise(rows[:, None], bits)
    assert np.array_equal(_unpack(cache, D)[0], codes)
    assert np.array_equal(cache.scales.float().cpu().numpy(), s, equal_nan=True)
    out = torch.zeros_like(x)
    B.cache_read(cache, out, st)
    want = oh.dequantise(codes, s)[:, 0].astype(np.float32)
    assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)
    assert np.isnan(want[5:8]).all() and not want[3:5].any()


def test_cache_indices_outside_are_reported_and_skipped(B):
    x = torch.randn(10, 2, 50, device="cuda")
    t = torch.arange(10.0, dtype=torch.float64, device="cuda") + 1
    for idt in (np.int32, np.int64):
        cache, st = B.RowCache(8, 2, 50, 8), _status()
        cache.codes.fill_(9)
        cache.scales.fill_(2.0)
        B.cache_write(cache, x, st, src=_dev([0, 10, -1, 3], idt), dst=_dev([7, 5, 6, 8], idt), times=t)
        assert int(st.item()) == 4
        sc = cache.scales.float().cpu()
        assert (sc[:5] == 2).all() and not sc[5:7].any() and cache.times[7].item() == 1.0 and not cache.times[5:7].any()
        assert (cache.codes[:5] == 9).all() and (cache.codes[5:7] == 128).all()
        rows = torch.full((10, 100), 5.0, device="cuda")
        st.zero_()
        B.cache_read(cache, rows, st, src=_dev([7, 8, -2, 7], idt), dst=_dev([1, 2, 3, 10], idt))
        assert int(st.item()) == 4 and not rows[2:4].any() and (rows[[0, 4, 5, 6, 7, 8, 9]] == 5).all()
        assert (rows[1].view(2, 50) - x[0]).abs().max() <= x[0].abs().max() / 127
    big = 1 << 40
    st.zero_()
    B.cache_read(cache, rows, st, src=_dev([big, -big], np.int64), dst=_dev([0, 1], np.int64))
    assert int(st.item()) == 4 and not rows[:2].any()


@pytest.mark.parametrize("bits,dt", [(4, "f32"), (8, "bf16")])
def test_cache_strided_rows_and_records(B, bits, dt):
    """Rows inside wider ones, on unaligned bases, and caches kept as records of one byte tensor."""
    rng = np.random.default_rng(7)
    N, heads, dim = 300, 2, 50
    wide = _plain_rows(rng, N, 1, 3 * heads * dim + 5, dt)[:, 0].cuda()
    times = torch.rand(N, dtype=torch.float64, device="cuda")
    for off in (0, 1, 2, 8, 100):
        rows = wide[:, off:off + heads * dim]
        st = _status()
        a, b = B.RowCache(N, heads, dim, bits), B.RowCache(N, heads, dim, bits, record=True)
        assert b.data.shape[1] % 16 == 0
        B.cache_write(a, rows, st, times=times)
        B.cache_write(b, rows, st, times=times)
        codes, s = oh.quantise(rows.float().cpu().numpy().reshape(N, heads, dim), bits)
        assert np.array_equal(_unpack(a, dim)[0], codes)
        o1, o2, t2 = torch.zeros_like(wide), torch.zeros_like(wide), torch.zeros_like(times)
        B.cache_read(a, o1[:, off:off + heads * dim], st)
        B.cache_read(b, o2[:, off:off + heads * dim], st, times=t2)
        assert torch.equal(o1, o2) and torch.equal(t2, times) and int(st.item()) == 0
        want = torch.zeros_like(wide)
        want[:, off:off + heads * dim] = torch.from_numpy(oh.dequantise(codes, s).astype(np.float32)).to(TYPES[dt]).reshape(N, -1).cuda()
        assert torch.equal(o1, want)


def test_cache_beyond_32_bit_offsets(B):
    """A cache of more than 4 GB of codes: rows at its ends and around every 2^31 bytes."""
    rows, heads, dim = 17_000_000, 2, 128
    cache, st = B.RowCache(rows, heads, dim, 8, times=False), _status()
    assert cache.codes.numel() > 2 ** 32
    at = torch.tensor([0, 2 ** 31 // 256 - 1, 2 ** 31 // 256, 2 ** 32 // 256 - 1, 2 ** 32 // 256, rows - 1], device="cuda")
    x = torch.randn(len(at), heads, dim, device="cuda")
    B.cache_write(cache, x, st, dst=at)
    out = torch.zeros_like(x)
    B.cache_read(cache, out, st, src=at)
    codes, s = oh.quantise(x.cpu().numpy(), 8)
    assert np.array_equal(out.cpu().numpy(), oh.dequantise(codes, s).astype(np.float32)) and int(st.item()) == 0
    touched = torch.zeros(rows, dtype=torch.bool, device="cuda")
    touched[at] = True
    assert torch.equal(cache.scales.float().amax(1) > 0, touched)


def test_cache_calls_captured_and_on_another_stream(B):
    cache, st = B.RowCache(64, 1, 100, 4), _status()
    x, out = torch.randn(64, 100, device="cuda"), torch.zeros(64, 100, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.cache_write(cache, x, st)
        B.cache_read(cache, out, st)
    for seed in (1, 2):
        x.copy_(torch.randn(64, 100, generator=torch.Generator().manual_seed(seed)).cuda())
        g.replay()
        codes, sc = oh.quantise(x.cpu().numpy()[:, None], 4)
        assert np.array_equal(out.cpu().numpy(), oh.dequantise(codes, sc)[:, 0].astype(np.float32))


def test_cache_of_no_rows(B):
    cache, st = B.RowCache(0, 2, 50, 4), _status()
    empty = torch.empty(0, 100, device="cuda")
    B.cache_write(cache, empty, st)
    B.cache_read(cache, empty, st)
    idx = torch.empty(0, dtype=torch.int64, device="cuda")
    B.cache_write(cache, torch.ones(3, 100, device="cuda"), st, src=idx, dst=idx)
    assert int(st.item()) == 0
