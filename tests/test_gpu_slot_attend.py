"""Slot attention and its backward pass on the GPU against the plain forms in 64 bits.

Tolerances, from the arithmetic (u = 2^-24): a dot product of D terms in fp32 is off by at most D u sum|.|, so a logit by
d = (D + 4) u scale sum|q k| + 4 u (|z| + |bias|); the weights by a factor of 1 +- w, w = 2 d + (n + 16) u over n slots (the exponential's
2^-22, the sum, the quotient); dp = do.v by e = D u sum|do v|; dz = p (dp - delta) by p (w (|dp| + |delta|) + e + sum p (w |dp| + e)).  These go
through the last sums with their own n u, and the output type adds half a step."""
import numpy as np
import pytest
import torch

from oracle import history as oh

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2608_16305_b200 import binding
    binding.load_library()
    return binding


class Case:
    def __init__(self, B, R, S, H, KV, D, dt, buckets=8, seed=0, cnt=None):
        rng = np.random.default_rng(seed)
        self.B, self.shape, self.dt = B, (R, S, H, KV, D), dt
        mk = lambda *s: torch.from_numpy((rng.standard_normal(s) * np.exp(0.5 * rng.standard_normal(s[:-1] + (1,)))).astype(np.float32)).to(TYPES[dt]).cuda()
        self.q, self.do, self.k, self.v = mk(R, H, D), mk(R, H, D), mk(R, S, KV, D), mk(R, S, KV, D)
        if cnt is None:
            cnt = rng.integers(0, S + 1, R)
            cnt[rng.random(R) < 0.5] = S
        self.cnt = torch.tensor(np.asarray(cnt), dtype=torch.int32, device="cuda")
        self.bias = self.b = {}
        if buckets:
            times = rng.random(R) * 100 + 1000
            ts = times[:, None] - np.cumsum(rng.integers(0, 50, (R, S)), 1)
            bounds = np.concatenate([[0.0], np.geomspace(1, 50 * S, max(buckets - 2, 0))])[:buckets - 1]
            dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, t)).cuda()
            self.b = dict(bias=dev(rng.standard_normal((H, buckets)), np.float32), bounds=dev(bounds, np.float64),
                          times=dev(times, np.float64), ts=dev(ts, np.float64))
        self.buckets = buckets

    def forward(self, scale=None, **kw):
        out = torch.full_like(self.q, 77.0)
        self.B.slot_attend(self.q, self.k, self.v, self.cnt, out, scale=scale, **self.b, **kw)
        return out

    def backward(self, scale=None):
        R, S, H, KV, D = self.shape
        g = [torch.full_like(t, 77.0) for t in (self.q, self.k, self.v)]
        extra = {}
        if self.buckets:
            g.append(torch.full_like(self.b["bias"], 77.0))
            extra = dict(dbias=g[3], scratch=torch.full((self.B.slot_attend_scratch(R, H, self.buckets),), float("nan"), device="cuda"))
        self.B.slot_attend_backward(self.q, self.k, self.v, self.cnt, self.do, *g[:3], scale=scale, **self.b, **extra)
        return g

    def check(self, scale=None):
        R, S, H, KV, D = self.shape
        out, grads = self.forward(scale), self.backward(scale)
        scale = D ** -0.5 if scale is None else scale
        G = H // KV
        q, do, k, v = (t.double().cpu().numpy() for t in (self.q, self.do, self.k, self.v))
        cnt = self.cnt.clamp(0, S).cpu().numpy()
        bias = bk = None
        if self.buckets:
            bias = self.b["bias"].double().cpu().numpy()
            bk = np.searchsorted(self.b["bounds"].cpu().numpy(), (self.b["times"][:, None] - self.b["ts"]).cpu().numpy(), side="right")
        ref = oh.slot_attend(q, k, v, cnt, bias, bk, scale)
        dq, dk, dv, db, _ = oh.slot_attend_backward(q, k, v, cnt, bias, bk, scale, do)
        # bounds, as at the head of this file: [R, KV, G, S]
        ok = (np.arange(S)[None] < cnt[:, None])[:, None, None]
        qg, dog = q.reshape(R, KV, G, D), do.reshape(R, KV, G, D)
        b4 = np.zeros((R, KV, G, S)) if bias is None else bias[:, bk].reshape(KV, G, R, S).transpose(2, 0, 1, 3)
        fin = np.isfinite(b4)
        qk = scale * np.einsum("rkgd,rskd->rkgs", np.abs(qg), np.abs(k))
        z = scale * np.einsum("rkgd,rskd->rkgs", qg, k) + b4
        z = np.where(ok, z, -np.inf)
        m = z.max(-1, keepdims=True)
        p = np.where(z > -np.inf, np.exp(z - np.where(np.isfinite(m), m, 0)), 0.0)
        p = p / np.maximum(p.sum(-1, keepdims=True), 1e-300)
        d = np.where(ok & fin, (D + 4) * U * qk + 4 * U * (np.where(fin, np.abs(z), 0) + np.where(fin, np.abs(b4), 0)), 0)
        d = np.where(np.isfinite(d), d, 0).max(-1, keepdims=True)
        w = 2 * d + (S + 16) * U
        av, ak = np.abs(v), np.abs(k)
        dp = np.einsum("rkgd,rskd->rkgs", dog, v)
        e = (D + 2) * U * np.einsum("rkgd,rskd->rkgs", np.abs(dog), av)
        delta = (p * dp).sum(-1, keepdims=True)
        e_dz = p * (w * (np.abs(dp) + np.abs(delta)) + e + (p * (w * np.abs(dp) + e)).sum(-1, keepdims=True) + (S + 4) * U * (p * np.abs(dp)).sum(-1, keepdims=True))
        dz = np.abs(p * (dp - delta))
        half = torch.finfo(TYPES[self.dt]).eps / 2
        tiny = 2.0 ** -25 if self.dt == "f16" else 1e-37
        n = (S + 4) * U
        bounds = [(np.einsum("rkgs,rskd->rkgd", p * (w + n), av).reshape(R, H, D), ref, out),
                  (scale * np.einsum("rkgs,rskd->rkgd", e_dz + n * dz, ak).reshape(R, H, D), dq, grads[0]),
                  (scale * np.einsum("rkgs,rkgd->rskd", e_dz + (G + 4) * U * dz, np.abs(qg)), dk, grads[1]),
                  (np.einsum("rkgs,rkgd->rskd", p * (w + (G + 4) * U), np.abs(dog)), dv, grads[2])]
        worst = []
        for tol, want, got in bounds:
            tol = tol + half * np.abs(want) + tiny
            err = np.abs(got.double().cpu().numpy() - want)
            assert (err <= tol).all(), (len(worst), float((err / tol).max()))
            worst.append(float((err / tol).max()))
        if self.buckets:
            tol = np.zeros((H, self.buckets))
            eh = (e_dz * ok).reshape(R, H, S)
            for h in range(H):
                np.add.at(tol[h], bk, eh[:, h])
            err = np.abs(grads[3].double().cpu().numpy() - db)
            assert (err <= tol + U * np.abs(db) + 1e-37).all(), float((err / (tol + 1e-37)).max())
        return out, grads


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,S,H,KV,D", [(40, 10, 2, 2, 50), (33, 20, 2, 2, 16), (7, 64, 4, 4, 32), (5, 130, 2, 1, 64), (9, 1, 1, 1, 1), (3, 3, 8, 2, 25),
                                        (4, 33, 16, 4, 128), (6, 17, 3, 3, 43), (2, 7, 32, 32, 2), (2, 5, 64, 16, 8), (1, 9, 1, 1, 128)])
def test_slots_forward_and_backward(B, dt, R, S, H, KV, D):
    Case(B, R, S, H, KV, D, dt, seed=S + D).check()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("S,H,KV,D", [(1000, 2, 2, 50), (700, 1, 1, 33), (301, 8, 2, 128), (129, 16, 16, 128)])
def test_slots_in_several_chunks(B, dt, S, H, KV, D):
    """More slots than a warp holds: two sweeps of the backward pass; counts at, before and behind every chunk's end."""
    c = Case(B, 12, S, H, KV, D, dt, seed=S, cnt=[S, 0, 1, S // 2, S - 1, 7, 8, 9, 28, 29, 64, S])
    c.check()
    c.check(scale=0.01)


def test_slots_many_roots_and_the_same_bits_again(B):
    """More roots than warps that run at once; the bias's gradient over all of them."""
    c = Case(B, 9000, 6, 2, 1, 10, "f32", buckets=5)
    out, grads = c.check()
    assert torch.equal(out, c.forward())
    for a, b in zip(grads, c.backward()):
        assert torch.equal(a, b)


def test_slots_buckets(B):
    for buckets in (0, 1, 2, 33, 128):
        Case(B, 50, 12, 4, 2, 20, "f32", buckets=buckets, seed=buckets).check()


def test_slots_wide_tables_and_heads(B):
    Case(B, 30, 6, 128, 64, 16, "f32", buckets=128).check()
    Case(B, 5, 3, 256, 256, 8, "bf16", buckets=64).check()
    Case(B, 5, 3, 16, 1, 128, "f32", buckets=3).check()


def test_slots_gradients_against_differences(B):
    """Central differences of the forward kernel itself, in fp32, along random directions."""
    c = Case(B, 64, 10, 2, 2, 16, "f32", buckets=6)
    grads = c.backward()
    rng = torch.Generator(device="cuda").manual_seed(1)
    for name, g in zip(("q", "k", "v", "bias"), grads):
        t = c.b["bias"] if name == "bias" else getattr(c, name)
        dirn = torch.randn(t.shape, generator=rng, device="cuda")
        keep, f = t.clone(), []
        for e in (1e-2, -1e-2):
            t.copy_(keep + e * dirn)
            f.append((c.forward().double() * c.do.double()).sum().item())
        t.copy_(keep)
        num, ana = (f[0] - f[1]) / 2e-2, (g.double() * dirn.double()).sum().item()
        mag = (g.double() * dirn.double()).abs().sum().item()
        # second-order remainder e^2 / 6 f''' and fp32 sums: a thousandth of the terms' magnitudes
        assert abs(num - ana) <= 1e-3 * mag, (name, num, ana, mag)


def test_slots_hidden_rows_and_counts(B):
    """NaN and infinities behind the counted slots change nothing; counts out of range are cut; gradients there are zero."""
    c = Case(B, 40, 9, 2, 2, 50, "f32")
    out, grads = c.forward(), c.backward()
    for r in range(40):
        n = int(c.cnt[r])
        c.k[r, n:] = float("nan")
        c.v[r, n:] = float("inf")
        c.b["ts"][r, n:] = float("nan")
        assert not grads[1][r, n:].any() and not grads[2][r, n:].any()
    assert torch.equal(c.forward(), out)
    for a, b in zip(grads, c.backward()):
        assert torch.equal(a, b)
    c = Case(B, 40, 9, 2, 2, 50, "bf16", cnt=[-5, 0, 9, 100] * 10)
    out, _ = c.check()
    assert not out[0::4].any() and not out[1::4].any()


def test_slots_masked_buckets(B):
    for S in (9, 600):
        c = Case(B, 20, S, 2, 2, 50, "f32", buckets=6)
        c.b["bias"][:, 2:4] = float("-inf")
        c.check()
        c.b["bias"][:, 2:4] = torch.finfo(torch.float32).min
        assert all(t.isfinite().all() for t in [c.forward()] + c.backward())
        c.b["bias"][:] = torch.finfo(torch.float32).min
        assert c.forward()[c.cnt > 0].any()
        c.b["bias"][:] = float("-inf")
        assert not c.forward().any() and not any(g.any() for g in c.backward())


def test_slots_of_one_have_no_gradient_of_logits(B):
    """One counted slot: its weight is 1 whatever the logit, exactly."""
    c = Case(B, 100, 5, 2, 2, 50, "f32", cnt=[1] * 100)
    dq, dk, dv, db = c.backward()
    assert not dq.any() and not dk.any() and not db.any()
    assert torch.equal(dv[:, 0], c.do) and torch.equal(c.forward(), c.v[:, 0])


def test_slots_on_unaligned_bases(B):
    for dt, D in (("f32", 50), ("bf16", 50), ("f16", 25)):
        c = Case(B, 11, 7, 2, 2, D, dt, seed=D)
        out, grads = c.check()
        for off in (1, 2, 4):
            move = lambda t: torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")[off:off + t.numel()].view(t.shape).copy_(t)
            c.q, c.k, c.v, c.do = move(c.q), move(c.k), move(c.v), move(c.do)
            o2, g2 = c.check()
            buf = torch.full((c.k.numel() + 8,), 5.0, dtype=c.k.dtype, device="cuda")
            dk = buf[off:off + c.k.numel()].view(c.k.shape)
            R, S, H, KV, _ = c.shape
            B.slot_attend_backward(c.q, c.k, c.v, c.cnt, c.do, g2[0], dk, g2[2], **c.b, dbias=g2[3],
                                   scratch=torch.empty(B.slot_attend_scratch(R, H, 8), device="cuda"))
            assert torch.equal(dk, g2[1]) and (buf[:off] == 5).all() and (buf[off + dk.numel():] == 5).all()


def test_slots_captured_and_replayed(B):
    """Forward and backward in one graph, replayed on new inputs; an eager call between."""
    c = Case(B, 30, 12, 2, 2, 50, "f32")
    out = torch.zeros_like(c.q)
    g = [torch.zeros_like(t) for t in (c.q, c.k, c.v, c.b["bias"])]
    scratch = torch.empty(B.slot_attend_scratch(30, 2, 8), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.slot_attend(c.q, c.k, c.v, c.cnt, out, **c.b)
        B.slot_attend_backward(c.q, c.k, c.v, c.cnt, c.do, *g[:3], **c.b, dbias=g[3], scratch=scratch)
    for seed in (5, 6):
        n = Case(B, 30, 12, 2, 2, 50, "f32", seed=seed)
        for a in ("q", "k", "v", "do", "cnt"):
            getattr(c, a).copy_(getattr(n, a))
        for a in c.b:
            c.b[a].copy_(n.b[a])
        want = [n.forward()] + n.backward()
        graph.replay()
        for x, y in zip([out] + g, want):
            assert torch.equal(x, y)


def test_slots_without_roots(B):
    c = Case(B, 0, 5, 2, 2, 50, "f32", cnt=[])
    assert c.forward().numel() == 0
    assert not c.backward()[3].any()


@pytest.mark.parametrize("R,H,KV,D,buckets", [(1, 2, 2, 50, 8), (11, 2, 2, 50, 8), (3, 64, 64, 20, 100), (600, 16, 16, 33, 7), (2000, 4, 4, 50, 5)])
def test_slots_scratch_is_not_written_beyond_its_size(B, R, H, KV, D, buckets):
    """Fewer roots than units of work, and more: the documented scratch suffices, and what lies behind it stays."""
    c = Case(B, R, 4, H, KV, D, "f32", buckets=buckets)
    n = B.slot_attend_scratch(R, H, buckets)
    buf = torch.full((n + 4096,), 5.0, device="cuda")
    g = [torch.empty_like(t) for t in (c.q, c.k, c.v, c.b["bias"])]
    B.slot_attend_backward(c.q, c.k, c.v, c.cnt, c.do, *g[:3], **c.b, dbias=g[3], scratch=buf[:n])
    assert (buf[n:] == 5).all()
    for a, b in zip(g, c.backward()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("S,H,KV,D", [(40, 2, 2, 16), (33, 8, 2, 16), (7, 1, 1, 16), (128, 4, 4, 32)])
def test_slots_bias_gradient_sums_to_zero_over_the_buckets(B, dt, S, H, KV, D):
    """A root's dz sum to 0, so a head's gradients of all buckets do.  Here dp is near 1000 and differs by a fraction, so that a delta rounded
    to fp32 shows on every slot with one sign (U 1000 a root).  Allowed are the roundings of each dz (its weight, two differences, a
    product) and five of a scan: 9 U sum |dz|, and those of the results."""
    R = 64
    c = Case(B, R, S, H, KV, D, dt, buckets=5, seed=S)
    c.do.fill_(1.0)
    c.v.normal_(generator=torch.Generator("cuda").manual_seed(S)).mul_(1.0 / 16).add_(1000.0 / D)
    q, do, k, v = (t.double().cpu().numpy() for t in (c.q, c.do, c.k, c.v))
    cnt, G = c.cnt.cpu().numpy(), H // KV
    bias = c.b["bias"].double().cpu().numpy()
    bk = np.searchsorted(c.b["bounds"].cpu().numpy(), (c.b["times"][:, None] - c.b["ts"]).cpu().numpy(), side="right")
    z = D ** -0.5 * np.einsum("rkgd,rskd->rkgs", q.reshape(R, KV, G, D), k) + bias[:, bk].reshape(KV, G, R, S).transpose(2, 0, 1, 3)
    z = np.where((np.arange(S)[None] < cnt[:, None])[:, None, None], z, -1e30)
    p = np.exp(z - z.max(-1, keepdims=True)) * (z > -1e29)
    p /= np.maximum(p.sum(-1, keepdims=True), 1e-300)
    dp = np.einsum("rkgd,rskd->rkgs", do.reshape(R, KV, G, D), v)
    dz = p * (np.abs(dp - (p * dp).sum(-1, keepdims=True)) + 2 * (D + 2) * U * np.abs(dp))
    tol = 9 * U * dz.sum((0, 3)).reshape(H)
    db = c.backward()[3].double().cpu().numpy()
    assert (np.abs(db.sum(1)) <= tol + U * np.abs(db).sum(1)).all(), (db.sum(1), tol)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("H,KV,D", [(2, 2, 50), (4, 2, 33), (8, 2, 64), (3, 1, 16), (6, 3, 100), (8, 1, 128), (12, 3, 25), (24, 2, 8), (4, 4, 5)])
@pytest.mark.parametrize("R,S", [(3, 100), (60, 37), (1000, 20)])
def test_slots_query_heads_together_and_warps_together(B, dt, R, S, H, KV, D):
    """Query heads of a cached head by ones, twos and fours, several times over; a root by four warps, by two, by one."""
    c = Case(B, R, S, H, KV, D, dt, seed=R + H)
    out, grads = c.check()
    assert torch.equal(out, c.forward())
    for a, b in zip(grads, c.backward()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("R,S,H,KV,D", [(1300, 30, 128, 64, 4), (1300, 70, 64, 16, 3), (3, 5000, 1, 1, 2), (1200, 4200, 1, 1, 2), (5, 4101, 4, 2, 20),
                                        (590, 400, 8, 2, 6), (1024, 200, 8, 8, 4), (1025, 200, 8, 8, 4)])
def test_slots_in_several_chunks_by_one_and_more_warps(B, R, S, H, KV, D):
    Case(B, R, S, H, KV, D, "f32", seed=S).check()


def test_slots_masked_buckets_by_more_warps(B):
    """Buckets at -infinity and at the type's lowest value, rows without a slot, where warps share a root and heads are taken together."""
    for R, S, H, KV in ((20, 150, 8, 2), (20, 150, 2, 2), (900, 40, 4, 2)):
        c = Case(B, R, S, H, KV, 32, "f32", seed=R + H, cnt=[0] + [S] * (R - 1))
        c.b["bias"][:, 1::2] = float("-inf")
        c.check()
        c.b["bias"][:] = torch.finfo(torch.float32).min
        out, grads = c.forward(), c.backward()
        assert all(bool(torch.isfinite(t).all()) for t in (out, *grads)) and not out[0].any()
        c.b["bias"][:] = float("-inf")
        assert not c.forward().any() and not any(g.any() for g in c.backward())
