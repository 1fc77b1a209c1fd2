"""Attention over the quantised history cache on the GPU against the plain form in 64 bits.

Tolerance of an output, from the arithmetic: the query is held in 22 bits and both products are summed in fp32 over at most 128 terms,
so a logit is off by at most d = 2^-18 * scale * sum |q k| + 2^-21 * (|z| + |bias|) (three roundings of the scaled logit, one of its
difference to the maximum, the exponential's own 2^-22); weights are then off by a factor of 1 +- 2 d, and the weighted sum by
(2 d + 2^-17) * sum p |v|, where 2^-17 covers 22-bit weights, fp32 sums over all tiles and the final quotient.  Weights below 2^-36 of
the largest p * scale are lost to fp16's range: 2^-20 * max(p * scale) * L for thousands of them.  Then half a step of the output type."""
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


class Case:
    """Caches of P rows with random values, histories of the given lengths, one root per history (or roots_per of them)."""

    def __init__(self, B, lens, H, KV, D, bits, dt, buckets=8, seed=0, spread=1.0, roots_per=1, record=False):
        rng = np.random.default_rng(seed)
        self.B, self.rng, self.H, self.KV, self.D, self.bits, self.dt = B, rng, H, KV, D, bits, dt
        lens = np.asarray(lens)
        first = np.concatenate([[0], np.cumsum(lens)[:-1]]) + 3
        self.P = int(lens.sum()) + 7
        self.first, self.len = np.repeat(first, roots_per), np.repeat(lens, roots_per).astype(np.int32)
        self.R = len(self.len)
        self.k, self.v = (self._rows(rng, spread) for _ in range(2))
        self.kc, self.vc = (B.RowCache(self.P, KV, D, bits, record=record) for _ in range(2))
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.cache_write(self.kc, torch.from_numpy(self.k).cuda(), self.status)
        B.cache_write(self.vc, torch.from_numpy(self.v).cuda(), self.status)
        self.ks, self.vs = oh.quantise(self.k, bits), oh.quantise(self.v, bits)
        self.q = torch.from_numpy((rng.standard_normal((self.R, H, D)) * np.exp(rng.standard_normal((self.R, H, 1)))).astype(np.float32)).to(TYPES[dt])
        self.ts = np.sort(rng.integers(0, 10 * self.P, self.P).astype(np.float64))
        self.times = np.array([self.ts[min(f + n, self.P - 1)] + 1.0 for f, n in zip(self.first, self.len)])
        self.bounds = np.concatenate([[0.0], np.geomspace(1, 10 * self.P, max(buckets - 2, 0))])[:buckets - 1]
        self.bias = rng.standard_normal((H, buckets)).astype(np.float32) if buckets else None

    def _rows(self, rng, spread):
        x = rng.standard_normal((self.P, self.KV, self.D)) * np.exp(spread * rng.standard_normal((self.P, self.KV, 1)))
        return x.astype(np.float32)

    def run(self, window, sinks, scale=None, q=None, out=None, **kw):
        q = self.q.cuda() if q is None else q
        out = torch.full_like(q, 77.0) if out is None else out
        b = {} if self.bias is None else dict(bias=_dev(self.bias, np.float32), bounds=_dev(self.bounds, np.float64),
                                              times=_dev(self.times, np.float64), ts=_dev(self.ts, np.float64))
        self.B.cached_attend(q, self.kc, self.vc, _dev(self.first, np.int64), _dev(self.len, np.int32), window, sinks, out, self.status,
                             scale=scale, **b, **kw)
        return out

    def seen(self, r, window, sinks):
        n = int(self.len[r])
        lo = max(n - window, 0)
        return [int(self.first[r]) + j for j in list(range(min(sinks, lo))) + list(range(lo, n))]

    def check(self, out, window, sinks, scale=None, roots=None):
        scale = self.D ** -0.5 if scale is None else scale
        out = out.float().cpu().numpy().astype(np.float64)
        q = self.q.double().numpy()
        half = torch.finfo(TYPES[self.dt]).eps / 2
        L = 7 if self.bits == 4 else 127
        worst = 0.0
        for r in (range(self.R) if roots is None else roots):
            at = self.seen(r, window, sinks)
            bk = np.searchsorted(self.bounds, self.times[r] - self.ts[at], side="right") if self.bias is not None else None
            for h in range(self.H):
                kv = h // (self.H // self.KV)
                k = oh.dequantise(self.ks[0][at, kv], self.ks[1][at, kv])
                v = oh.dequantise(self.vs[0][at, kv], self.vs[1][at, kv])
                b = 0.0 if bk is None else self.bias[h][bk].astype(np.float64)
                z = scale * (k @ q[r, h]) + b
                p = oh.softmax(z)
                ref = p @ v if len(at) else np.zeros(self.D)
                if len(at) == 0 or not p.any():
                    assert not out[r, h].any(), (r, h)
                    continue
                live = p > 0
                d = 2.0 ** -18 * scale * (np.abs(k[live]) @ np.abs(q[r, h])).max() + 2.0 ** -21 * np.max(np.abs(z[live]) + np.abs(np.broadcast_to(b, z.shape)[live]))
                tol = (2 * d + 2.0 ** -17) * (p @ np.abs(v)) + 2.0 ** -20 * (p * self.vs[1][at, kv]).max() * L + half * np.abs(ref) + 2.0 ** -25 * (self.dt == "f16")
                err = np.abs(out[r, h] - ref)
                worst = max(worst, float((err / tol).max()))
                assert (err <= tol).all(), (r, h, len(at), float((err / tol).max()))
        return worst


LENS = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 100, 0, 130]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H,KV,D", [(2, 2, 50), (1, 1, 100), (8, 2, 64), (4, 4, 32), (3, 1, 25), (16, 1, 128), (1, 1, 1), (9, 1, 33), (6, 3, 127)])
def test_attend_all_lengths(B, bits, dt, H, KV, D):
    """A warp per unit (short windows) and a block per unit (long ones); groups of 1 to 16 query heads; every tile boundary."""
    c = Case(B, LENS, H, KV, D, bits, dt, seed=bits + 10 * D)
    for window, sinks in ((20, 0), (1, 0), (0, 2), (30, 2), (60, 4), (500, 0), (90, 7), (16, 64)):
        c.check(c.run(window, sinks), window, sinks)
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("bits,H,KV,D,dt", [(4, 2, 2, 50, "f32"), (8, 2, 2, 50, "f32"), (8, 4, 1, 128, "bf16"), (4, 1, 1, 20, "f16")])
def test_attend_long_windows_over_clusters(B, bits, H, KV, D, dt):
    """One to three roots with windows that take clusters of 2, 4 and 8 blocks; histories shorter than the launch expects."""
    c = Case(B, [5000, 3, 1700], H, KV, D, bits, dt, seed=bits, buckets=32)
    for window, sinks in ((520, 4), (1100, 1), (2200, 16), (4096, 4), (1 << 30, 0), (2 ** 31 - 1, 2 ** 31 - 1)):
        c.check(c.run(window, sinks), window, sinks)
        c.check(c.run(window, sinks, max_len=5000), window, sinks)
        c.check(c.run(window, sinks, max_len=1), window, sinks)                # a hint that is wrong changes nothing but the launch


def test_attend_many_roots_with_long_windows(B):
    """More units than the machine has warps, each of many tiles: a warp walks them alone."""
    c = Case(B, [300, 700, 50, 0], 2, 2, 50, 4, "f32", roots_per=600)
    out = c.run(600, 3)
    c.check(out, 600, 3, roots=list(range(0, c.R, 97)))
    assert torch.equal(out, c.run(600, 3))                                     # the same bits again


def test_attend_without_bias_one_bucket_and_many(B):
    for buckets in (0, 1, 2, 33, 128):
        c = Case(B, LENS, 4, 2, 50, 8, "f32", buckets=buckets, seed=buckets)
        for window, sinks in ((20, 1), (200, 1)):
            c.check(c.run(window, sinks, scale=0.37), window, sinks, scale=0.37)


def test_attend_records_and_strides(B):
    c = Case(B, LENS, 4, 2, 50, 4, "f32", record=True)
    c.check(c.run(40, 2), 40, 2)
    c.check(c.run(300, 2), 300, 2)


def test_attend_values_of_very_different_size(B):
    """Value rows over 26 decades, key rows that make logits of hundreds."""
    for bits in (4, 8):
        c = Case(B, LENS, 2, 1, 64, bits, "f32", spread=8.0, seed=3)
        c.k[:] = 0.05 * np.random.default_rng(1).standard_normal(c.k.shape)
        B.cache_write(c.kc, torch.from_numpy(c.k).cuda(), c.status)
        c.ks = oh.quantise(c.k, bits)
        c.check(c.run(20, 2), 20, 2)
        c.check(c.run(100, 2), 100, 2)
        c.q = c.q * 1e4
        c.check(c.run(100, 2), 100, 2)


def test_attend_does_not_touch_what_a_root_does_not_see(B):
    """NaN scales in every row outside the windows and sinks; a visible one spoils its own head only."""
    c = Case(B, [40, 100, 0, 33], 2, 2, 50, 4, "f32")
    for window, sinks in ((20, 3), (5, 0), (70, 1)):
        want = c.run(window, sinks)
        hidden = torch.ones(c.P, dtype=torch.bool)
        for r in range(c.R):
            hidden[c.seen(r, window, sinks)] = False
        k, v = c.kc.scales.clone(), c.vc.scales.clone()
        c.kc.scales[hidden.cuda()] = float("nan")
        c.vc.scales[hidden.cuda()] = float("nan")
        assert torch.equal(c.run(window, sinks), want)
        c.kc.scales.copy_(k)
        c.vc.scales.copy_(v)
        for cache, row, head in ((c.kc, c.seen(1, window, sinks)[-1], 1), (c.vc, c.seen(0, window, sinks)[0], 0)):
            keep = cache.scales.clone()
            cache.scales[row, head] = float("nan")
            got = c.run(window, sinks)
            r = 1 if cache is c.kc else 0
            assert got[r, head].isnan().all()
            got[r, head] = want[r, head]
            assert torch.equal(got, want)
            cache.scales.copy_(keep)


def test_attend_masked_buckets(B):
    """Buckets at minus infinity and at the type's lowest value; roots that are left with nothing get zeros."""
    c = Case(B, LENS, 2, 2, 50, 8, "f32", buckets=6)
    for low in (-np.inf, float(np.finfo(np.float32).min)):
        c.bias[:, 2:4] = low
        for window in (20, 200):
            c.check(c.run(window, 1), window, 1)
    c.bias[:] = -np.inf
    for window in (20, 200, 5000):
        assert not c.run(window, 1).any()
    c.bias[:] = float(np.finfo(np.float32).min)
    out = c.run(200, 1)
    assert out.isfinite().all() and out[1].any()
    assert not Case(B, LENS, 2, 2, 50, 8, "f32", buckets=0).run(20, 0)[[0, 17]].any()


def test_attend_zero_and_tiny_operands(B):
    c = Case(B, LENS, 2, 2, 50, 4, "f32", buckets=0)
    c.q.zero_()
    c.check(c.run(20, 1), 20, 1)                                               # uniform weights
    c.q += 1e-30
    c.check(c.run(200, 1), 200, 1)
    c.q.fill_(1e30)
    assert c.run(200, 1)[1].isfinite().all()                                   # one entry: its value, whatever the logit
    c.v[:] = 0
    B.cache_write(c.vc, torch.from_numpy(c.v).cuda(), c.status)
    c.q.fill_(1.0)
    assert not c.run(20, 1).any() and not c.run(200, 1).any()


def test_attend_histories_outside_the_cache_are_reported(B):
    c = Case(B, [10, 10, 10, 10, 10], 2, 2, 50, 4, "f32")
    want = c.run(20, 1)
    good = c.first.copy(), c.len.copy()
    for first, length in ((-1, 5), (0, -1), (c.P - 4, 5), (c.P + 1, 0), (1 << 40, 3), (-(1 << 40), 3), (0, 2 ** 31 - 1)):
        c.first, c.len = good[0].copy(), good[1].copy()
        c.first[2], c.len[2] = first, length
        c.status.zero_()
        got = c.run(20, 1)
        assert int(c.status.item()) == 4 and not got[2].any()
        assert torch.equal(got[[0, 1, 3, 4]], want[[0, 1, 3, 4]])
    c.first, c.len = good
    c.first[2], c.len[2] = c.P, 0                                              # empty at the end: fine
    c.status.zero_()
    assert not c.run(20, 1)[2].any() and int(c.status.item()) == 0


def test_attend_unaligned_queries_and_outputs(B):
    """q and out on any element, as a slice of a larger buffer starts."""
    for dt in TYPES:
        c = Case(B, LENS, 2, 2, 25, 4, dt)
        n = c.q.numel()
        want = c.run(40, 2)
        for off in (1, 2, 3):
            q = torch.zeros(n + 8, dtype=TYPES[dt], device="cuda")[off:off + n].view(c.q.shape).copy_(c.q)
            buf = torch.full((n + 8,), 5.0, dtype=TYPES[dt], device="cuda")
            out = buf[off:off + n].view(c.q.shape)
            assert torch.equal(c.run(40, 2, q=q, out=out), want)
            assert (buf[:off] == 5).all() and (buf[off + n:] == 5).all()       # nothing beside the output


def test_attend_captured_and_replayed_on_new_inputs(B):
    c = Case(B, [3000, 5], 2, 2, 50, 4, "f32")
    args = [_dev(c.first, np.int64), _dev(c.len, np.int32)]
    b = dict(bias=_dev(c.bias, np.float32), bounds=_dev(c.bounds, np.float64), times=_dev(c.times, np.float64), ts=_dev(c.ts, np.float64))
    q = c.q.cuda()
    outs, graphs = [torch.zeros_like(q), torch.zeros_like(q)], []
    for window, out in zip((20, 4096), outs):                                  # a warp per unit; clusters
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.cached_attend(q, c.kc, c.vc, *args, window, 2, out, c.status, **b)
        graphs.append(g)
    c.q = c.q.flip(0).contiguous()
    q.copy_(c.q)
    for g in graphs:
        g.replay()
    for window, out in zip((20, 4096), outs):
        c.check(out, window, 2)


def test_attend_rows_beyond_32_bit_offsets(B):
    """Histories at the far end of a cache whose codes pass 4 GB."""
    rows, KV, D = 34_000_000, 2, 50
    k = B.RowCache(rows, KV, D, 8, times=False)
    assert k.codes.numel() > 2 ** 32
    c = Case(B, [100, 40], KV, KV, D, 8, "f32", buckets=0)
    want = c.run(64, 2)
    st = c.status
    at = torch.arange(c.P, device="cuda")
    far = rows - c.P
    v = B.RowCache(rows, KV, D, 8, times=False)
    B.cache_write(k, torch.from_numpy(c.k).cuda(), st, dst=at + far)
    B.cache_write(v, torch.from_numpy(c.v).cuda(), st, dst=at + far)
    c.kc, c.vc, c.first = k, v, c.first + far
    assert torch.equal(c.run(64, 2), want) and int(st.item()) == 0
