"""Attention over the cache on inputs whose sums are exact: what is left is the roundings that the arithmetic cannot do without, so these
bounds are far below those of random inputs, and an operand form that keeps fewer bits does not pass.

Exact sums of the outputs: with a query of zeros every weight is 1; values are integers at scale 1, so that all products (codes times 1/2, the weight in
units of the running bound 2) and their sums, below 2^24 halves, are exact in any order.  Left: 1 / l by an instruction of relative error 2^-23 or one
division, and one product: 2^-22 of the output in all, 2^-21 with the margin of a merge of several warps (exact products with 1).

Exact logits: integer queries of 21 bits and a sign in [2^20, 2^21), integer keys at scale 1, a power of two as scale.  The upper term of a query is
a multiple of 2^-10 (of 2^20), its products' sums over 64 columns stay below 2^14: 24 bits; the lower term, times 2^11, is a multiple of 2^-9 of at
most 1: 22 bits.  The pairs of a query cancel: sums are 2^12 times smaller than their terms, and the logits, multiples of scale * ks of a few bits, are
exact.  The values are one-hot: an output column has one weight.  In units of 2^-24: exponent's argument |z - m| (1 + 1/2) (log2(e) and the product
rounded, times ln 2), 4 for the instruction; twice, for the weight and for the sum l; 12 for the sum's roundings of 64 keys; 4 for the
weight's two terms, 1 for putting them together, 3 for the quotient."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_16305_b200 import binding
    binding.load_library()
    return binding


def _caches(B, k, v, bits):
    P, KV, D = k.shape
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    kc, vc = B.RowCache(P, KV, D, bits), B.RowCache(P, KV, D, bits)
    B.cache_write(kc, torch.from_numpy(k.astype(np.float32)).cuda(), st)
    B.cache_write(vc, torch.from_numpy(v.astype(np.float32)).cuda(), st)
    assert (kc.scales == 1).all() and (vc.scales == 1).all()
    return kc, vc, st


def _integers(rng, shape, L):
    x = rng.integers(-L, L + 1, shape)
    x[..., 0] = L                                                  # the group's largest magnitude: scale 1
    return x


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("H,KV,D", [(2, 2, 50), (4, 2, 64), (8, 1, 128), (3, 1, 20), (1, 1, 100)])
@pytest.mark.parametrize("window", [40, 64, 500, 5000])
def test_equal_weights(B, bits, H, KV, D, window):
    rng = np.random.default_rng(D + window)
    L = 7 if bits == 4 else 127
    P = 5000
    k, v = (_integers(rng, (P, KV, D), L) for _ in range(2))
    kc, vc, st = _caches(B, k, v, bits)
    first, length = np.array([0, 10, 300, 7]), np.array([5000, 33, 1, 1700])
    q = torch.zeros(4, H, D, device="cuda")
    out = torch.zeros_like(q)
    B.cached_attend(q, kc, vc, torch.from_numpy(first).cuda(), torch.from_numpy(length.astype(np.int32)).cuda(), window, 0, out, st)
    out = out.cpu().numpy().astype(np.float64)
    for r in range(4):
        a, b = first[r] + max(0, length[r] - window), first[r] + length[r]
        want = np.repeat(v[a:b].sum(0) / (b - a), H // KV, 0)
        assert (np.abs(out[r] - want) <= 2.0 ** -21 * np.abs(want)).all()
    assert int(st.item()) == 0


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("H,KV,D", [(2, 2, 64), (4, 1, 64), (3, 1, 50), (8, 1, 64), (1, 1, 32)])
@pytest.mark.parametrize("roots", [3, 4000])
def test_exact_logits(B, bits, H, KV, D, roots):
    rng = np.random.default_rng(D + H)
    L = 7 if bits == 4 else 127
    n = D                                                          # keys of a history, one column of the values each
    k = _integers(rng, (n, KV, D), L)
    k[..., 1::2] = k[..., 0::2]
    v = np.zeros((n, KV, D), np.int64)
    v[np.arange(n), :, np.arange(n)] = L
    # pairs x, r - x of either sign: the logit is the sum of r k over the pairs, terms 2^12 and more times larger than r
    x = rng.integers(2 ** 20 + 16, 2 ** 21 - 16, (roots, H, D // 2)) * rng.choice([-1, 1], (roots, H, D // 2))
    r = rng.integers(-3, 4, x.shape)
    q = np.stack([x, r - x], -1).reshape(roots, H, D)
    scale = 2.0 ** -9 if bits == 8 else 2.0 ** -5
    kc, vc, st = _caches(B, k, v, bits)
    out = torch.zeros(roots, H, D, device="cuda")
    qd = torch.from_numpy(q.astype(np.float32)).cuda()
    assert np.array_equal(qd.cpu().numpy().astype(np.int64), q)
    B.cached_attend(qd, kc, vc, torch.zeros(roots, dtype=torch.int64, device="cuda"), torch.full((roots,), n, dtype=torch.int32, device="cuda"),
                    n, 0, out, st, scale=scale)
    out = out.cpu().numpy().astype(np.float64)
    z = scale * np.einsum("rhd,jhd->rhj", q, np.repeat(k, H // KV, 1)).astype(np.float64)
    z -= z.max(-1, keepdims=True)
    p = np.exp(z)
    want = L * p / p.sum(-1, keepdims=True)
    # weights below 2^-14 of the largest have fewer than 22 bits in their two terms: 2^-36 of the largest at least
    tol = want * (1.5 * np.abs(z) + 1.5 * np.abs(z).max(-1, keepdims=True) + 4 + 4 + 12 + 4 + 1 + 3) * 2.0 ** -24 + 2.0 ** -34 * want.max(-1, keepdims=True)
    err = np.abs(out - want)
    assert (err <= tol).all(), float((err / tol).max())
    assert int(st.item()) == 0
