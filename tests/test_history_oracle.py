"""Pins of the history operators' fp64 forms: closed forms, the library's attention, finite differences."""
import numpy as np
import pytest
import torch

from oracle import history as oh


def test_visible_set_of_window_and_sinks():
    ts = np.array([1.0, 2.0, 2.0, 5.0, 9.0])
    assert oh.visible(ts, 0, 5, 2.0, 3, 2) == (1, [0], [])              # strictly earlier only
    assert oh.visible(ts, 0, 5, 9.0, 2, 1) == (4, [3, 2], [0])
    assert oh.visible(ts, 0, 5, 99.0, 2, 9) == (5, [4, 3], [0, 1, 2])   # sinks stop at the window
    assert oh.visible(ts, 0, 5, 99.0, 0, 2) == (5, [], [0, 1])
    assert oh.visible(ts, 0, 5, 0.5, 3, 2) == (0, [], [])
    assert oh.visible(ts, 2, 2, 9.0, 3, 2) == (0, [], [])


@pytest.mark.parametrize("bits", [4, 8])
def test_quantiser_closed_forms(bits):
    L = 7 if bits == 4 else 127
    x = np.arange(-L, L + 1, dtype=np.float64)
    codes, s = oh.quantise(x, bits)
    assert s == 1.0 and codes.tolist() == x.tolist()                    # integers up to L are held exactly
    codes, s = oh.quantise(np.array([L, 0.5, 1.5, 2.5, -0.5, -1.5]), bits)
    assert codes.tolist() == [L, 0, 2, 2, 0, -2]                        # ties to even
    assert oh.quantise(np.zeros(5), bits)[1] == 0.0
    assert np.isnan(oh.quantise(np.array([1.0, np.inf]), bits)[1])
    assert oh.quantise(np.array([2.0 ** -101]), bits)[1] == 0.0
    assert oh.quantise(np.array([2.0 ** -100]), bits)[1] > 0.0
    x = np.random.default_rng(bits).standard_normal((2000, 50)).astype(np.float32)
    codes, s = oh.quantise(x, bits)
    assert np.abs(codes).max() <= L
    # half a step from the value, and the bf16 scale at most 2^-7 above amax / L
    assert (np.abs(oh.dequantise(codes, s) - x) <= s[:, None] * (0.5 + 1e-5)).all()
    amax = np.abs(x).max(1)
    assert (s * L >= amax * (1 - 2.0 ** -22)).all() and (s * L <= amax * (1 + 2.0 ** -7) * (1 + 2.0 ** -22)).all()


def test_bf16_up_is_the_next_number_above():
    x = np.random.default_rng(0).lognormal(0, 20, 4000).astype(np.float32)
    up = oh.bf16_up(x)
    t = torch.from_numpy(up)
    assert torch.equal(t.bfloat16().float(), t) and (up >= x).all()
    below = (up.view(np.uint32) - 0x10000).view(np.float32)
    assert (below < x).all()


def test_bucket_counts_bounds_not_above():
    b = [0.0, 1.0, 1.0, 4.0]
    assert [oh.bucket(b, x) for x in (-1.0, 0.0, 0.5, 1.0, 3.9, 4.0, 1e9, float("nan"))] == [0, 1, 1, 3, 3, 4, 4, 0]


def test_attention_against_the_library():
    rng = np.random.default_rng(3)
    R, S, H, KV, D, B = 4, 7, 4, 2, 6, 5
    q, k, v = rng.standard_normal((R, H, D)), rng.standard_normal((R, S, KV, D)), rng.standard_normal((R, S, KV, D))
    bias, bk = rng.standard_normal((H, B)), rng.integers(0, B, (R, S))
    out = oh.slot_attend(q, k, v, [S] * R, bias, bk, 0.3)
    tk = torch.from_numpy(k).permute(0, 2, 1, 3).repeat_interleave(2, 1)
    tv = torch.from_numpy(v).permute(0, 2, 1, 3).repeat_interleave(2, 1)
    mask = torch.from_numpy(bias[:, bk]).permute(1, 0, 2)[:, :, None]
    ref = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q)[:, :, None], tk, tv, attn_mask=mask, scale=0.3)
    assert np.allclose(out, ref[:, :, 0].numpy(), atol=1e-12)
    rows = k.reshape(R * S, KV, D)
    seen = [np.arange(r * S, (r + 1) * S)[::-1].copy() for r in range(R)]
    assert np.allclose(out, oh.attend(q, rows, v.reshape(R * S, KV, D), seen, bias, [b[::-1] for b in bk], 0.3), atol=1e-12)
    assert not oh.slot_attend(q, k, v, [0] * R, bias, bk, 0.3).any()
    assert not oh.slot_attend(q, k, v, [S] * R, np.full((H, B), -np.inf), bk, 0.3).any()


def test_gradients_against_differences():
    rng = np.random.default_rng(4)
    R, S, H, KV, D, B = 2, 4, 4, 2, 3, 3
    x = dict(q=rng.standard_normal((R, H, D)), k=rng.standard_normal((R, S, KV, D)), v=rng.standard_normal((R, S, KV, D)),
             bias=rng.standard_normal((H, B)))
    bk, cnt, w = rng.integers(0, B, (R, S)), [S, 2], rng.standard_normal((R, H, D))
    grads = oh.slot_attend_backward(x["q"], x["k"], x["v"], cnt, x["bias"], bk, 0.7, w)
    for name, g in zip(("q", "k", "v", "bias"), grads):
        for i in np.ndindex(g.shape):
            f = []
            for e in (1e-6, -1e-6):
                y = {n: a.copy() for n, a in x.items()}
                y[name][i] += e
                f.append((oh.slot_attend(y["q"], y["k"], y["v"], cnt, y["bias"], bk, 0.7) * w).sum())
            assert abs((f[0] - f[1]) / 2e-6 - g[i]) < 1e-7, (name, i)
    assert not grads[1][1, 2:].any() and not grads[2][1, 2:].any()
