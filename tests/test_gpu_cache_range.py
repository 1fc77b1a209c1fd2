"""Row cache at the ends of the row types' ranges: a finite row reads back finite, in the type that it was written in.

The scale is rounded up to bf16, so that the largest code times the scale may pass the row type's largest finite value M by up to 2^-7 of it.
Tolerance of a value that is read back: half a step of the codes (half the stored scale; 2^-20 of it for the fp32 product that is
rounded to the code) and half a step of the row type."""
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


def _rows(dt, heads, dim):
    """Rows whose largest magnitude lies at and just below the type's largest value."""
    top = torch.finfo(TYPES[dt]).max
    rng = np.random.default_rng(dim)
    x = rng.uniform(-1, 1, (40, heads, dim))
    x[np.arange(40)[:, None], np.arange(heads)[None], rng.integers(0, dim, (40, heads))] = rng.choice([-1.0, 1.0], (40, heads))
    x *= (1 - np.arange(40) / 40 * 0.02)[:, None, None]
    return torch.from_numpy(x * top).clamp(-top, top).to(TYPES[dt])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,dim", [(2, 64), (2, 50), (3, 43), (1, 1), (1, 128)])
def test_finite_rows_read_back_finite(B, bits, dt, heads, dim):
    x = _rows(dt, heads, dim)
    assert x.isfinite().all()
    cache, st = B.RowCache(len(x), heads, dim, bits), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cache_write(cache, x.cuda(), st)
    out = torch.zeros_like(x, device="cuda")
    B.cache_read(cache, out, st)
    out = out.cpu()
    assert out.isfinite().all()
    xd, od = x.double().numpy(), out.double().numpy()
    codes, s = oh.quantise(x.float().numpy(), bits)
    tol = s[..., None].astype(np.float64) * (0.5 + 2.0 ** -20) + torch.finfo(TYPES[dt]).eps / 2 * np.abs(od)
    assert (np.abs(od - xd) <= tol).all()
    want = oh.dequantise(codes, s, torch.finfo(TYPES[dt]).max)
    assert np.array_equal(out.float().numpy(), torch.from_numpy(want.astype(np.float32)).to(TYPES[dt]).float().numpy())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 43])
def test_rows_of_a_wider_type_convert_as_they_do_elsewhere(B, bits, dim):
    """A row beyond fp16's range is infinity there, as by any conversion; a group that is not finite is NaN."""
    x = torch.ones(6, 1, dim)
    x[0] *= 1e5
    x[1] *= -7e4
    x[2, 0, 0] = float("inf")
    x[3, 0, 0] = float("nan")
    x[4] *= 60000.0
    cache, st = B.RowCache(6, 1, dim, bits), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cache_write(cache, x.cuda(), st)
    out = torch.zeros(6, dim, dtype=torch.float16, device="cuda")
    B.cache_read(cache, out, st)
    assert (out[0] == float("inf")).all() and (out[1] == -float("inf")).all() and out[2:4].isnan().all() and out[4:].isfinite().all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("heads,D", [(1, 64), (2, 50), (4, 43), (8, 128)])
def test_attention_over_such_rows_is_finite(B, bits, heads, D):
    """fp16 values at the type's end through the attention: every weighted mean of them is finite in fp16."""
    P = 600
    v = torch.full((P, 1, D), 65504.0, dtype=torch.float16)
    v[:, :, 1::2] *= -1
    kc, vc = B.RowCache(P, 1, D, bits), B.RowCache(P, 1, D, bits)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.cache_write(kc, torch.randn(P, 1, D, generator=torch.Generator().manual_seed(1)).cuda(), st)
    B.cache_write(vc, v.cuda(), st)
    q = torch.randn(3, heads, D, generator=torch.Generator().manual_seed(2)).half().cuda()
    first = torch.tensor([0, 5, 0], device="cuda")
    length = torch.tensor([600, 1, 40], dtype=torch.int32, device="cuda")
    for window in (20, 600):
        out = torch.zeros_like(q)
        B.cached_attend(q, kc, vc, first, length, window, 0, out, st)
        # every value is the same but for its sign: the mean is within the sums' roundings (2^-17) and a half step of it
        assert (out.abs().float() - 65504.0).abs().max() <= 65504.0 * (2.0 ** -17 + 2.0 ** -11)
        assert (out[..., 0::2] > 0).all() and (out[..., 1::2] < 0).all()
