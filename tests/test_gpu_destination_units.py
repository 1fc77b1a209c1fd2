"""fp32 rows of very different magnitude in the destination loss: what a single large row or root leaves to the others."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_destination import F32, call, check, make
from tests.test_gpu_destination_reference import check_seen

pytestmark = pytest.mark.gpu
SHAPES = [(60, 400, 48), (300, 2000, 100), (40, 900, 200)]


@pytest.mark.parametrize("power", [20, 30, 45, 100])
@pytest.mark.parametrize("n,rows,dim", SHAPES)
def test_a_large_row_that_is_hidden(n, rows, dim, power):
    x = make(n, rows, dim, F32, masked=0.1)
    big = torch.zeros(rows, dtype=torch.bool, device="cuda")
    big[[3, rows // 2]] = True
    x["table"][big] *= 2.0 ** power
    x["bias"][big] = -math.inf
    x["target"] = torch.where((x["target"] >= 0) & big[x["target"].long().clamp(min=0)], torch.full_like(x["target"], 5), x["target"])
    check_seen(x, call(x), ~big)


@pytest.mark.parametrize("power", [20, 30, 45, 100])
@pytest.mark.parametrize("n,rows,dim", SHAPES)
def test_a_large_row_far_below_the_others(n, rows, dim, power):
    """Its logits are below -10^5: no weight at all."""
    x = make(n, rows, dim, F32, masked=0.1)
    x["q"][:, 0] = x["q"][:, 0].abs() + 1.0
    big = torch.zeros(rows, dtype=torch.bool, device="cuda")
    big[rows // 2] = True
    x["table"][big] = 0.0
    x["table"][big, 0] = -(2.0 ** power) * 8
    x["target"] = torch.where((x["target"] >= 0) & big[x["target"].long().clamp(min=0)], torch.full_like(x["target"], 5), x["target"])
    check_seen(x, call(x), ~big)


@pytest.mark.parametrize("power", [20, 30, 45])
@pytest.mark.parametrize("n,rows,dim", SHAPES)
def test_a_large_root(n, rows, dim, power):
    """All of its softmax lies on one node, which is its target: it adds nothing to the others' gradients."""
    x = make(n, rows, dim, F32, masked=0.1)
    x["table"][7] = 0.0
    x["table"][7, 0] = 40.0
    x["q"][5] = 0.0
    x["q"][5, 0] = 2.0 ** power * 8
    x["target"][5] = 7
    out = call(x)
    assert float(out["loss"][5]) == 0.0 and bool((out["dq"][5] == 0).all())
    some = torch.arange(n, device="cuda") != 5
    check(x | dict(q=x["q"][some], target=x["target"][some], g=x["g"][some]),
          {k: v[some] if k in ("loss", "alone", "dq") else v for k, v in out.items()})


@pytest.mark.parametrize("power", [20, 35])
@pytest.mark.parametrize("n,rows,dim", SHAPES)
def test_gradients_of_very_different_size(n, rows, dim, power):
    """What the small ones add is exact to 2^-40 of the largest; dq goes by the root's own."""
    x = make(n, rows, dim, F32, masked=0.1)
    x["g"][::3] *= 2.0 ** power
    check(x, call(x))


@pytest.mark.parametrize("top", [1e-30, 3e38])
def test_the_ends_of_the_range(top):
    """Rows up to the largest finite number, and all of them tiny."""
    x = make(50, 300, 40, F32, masked=0.1)
    x["table"] = x["table"] / x["table"].abs().max() * top
    x["scale"] = float(np.float32(x["scale"] / top * 4))                       # what the call takes (a subnormal number beside 3e38)
    check(x, call(x))


def test_a_root_without_numbers_is_alone_with_them():
    x = make(50, 300, 40, F32, masked=0.0)
    clean = call(x)
    for bad in (math.inf, math.nan):
        x["q"][7, 3] = bad
        out = call(x)
        some = torch.arange(50, device="cuda") != 7
        assert not any(bool(torch.isfinite(out[k][7])) for k in ("loss", "alone"))     # infinite where the target's product alone is -infinity
        check(x | dict(q=x["q"][some], target=x["target"][some], g=x["g"][some]), {k: out[k][some] for k in ("loss", "alone", "dq")})
    assert bool(torch.isfinite(clean["loss"]).all())


def test_logits_beyond_fp32_beside_others():
    """A root whose logits are infinite has no numbers; one of zeros, beside it, has all nodes alike."""
    x = make(20, 100, 16, F32, bias=False, masked=0.0)
    x["q"] *= 2.0 ** 120
    x["table"] *= 2.0 ** 110
    x["q"][4:] = 0.0
    x["scale"] = 1.0
    out = call(x, ())
    for k in ("loss", "alone"):
        assert not bool(torch.isfinite(out[k][:4]).any()) and float((out[k][4:] - math.log(100)).abs().max()) < 1e-5
