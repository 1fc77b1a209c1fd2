"""Logits that rise inside a thread block's share of the tiles, by as much as the types hold and by more."""
import pytest
import torch

from tests.test_gpu_destination import BF16, F32, call, check, make
from tests.test_gpu_destination_reference import LONG, steer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rise", [30.0, 70.0, 82.0, 87.5, 100.0, 300.0])
@pytest.mark.parametrize("n,rows,dim", LONG)
def test_a_few_nodes_far_above_the_others(n, rows, dim, rise, dtype):
    """One node of 1000, so that a share's first nodes lie far below the others; rows of magnitude 8 to 60, gradients of 10^-11."""
    high = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda") < 1e-3
    x = make(n, rows, dim, dtype, bias=False, masked=0.0)
    x = steer(x | dict(q=x["q"] / 8, table=x["table"] * 8, g=x["g"] * 1e-8), torch.where(high, rise, 0.0))
    near = torch.nonzero(high)[:, 0]
    x["target"] = torch.where(torch.arange(n, device="cuda") % 2 == 0, x["target"], near[x["target"] % near.numel()].int())
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,rows,dim", LONG)
def test_logits_that_climb_through_every_share(n, rows, dim, dtype):
    """By 400 in 5 tiles, over and over, by rows and by biases."""
    x = make(n, rows, dim, dtype, masked=0.1)
    up = torch.arange(rows, device="cuda") % 640 / 1.6 - 200.0
    check(x | dict(bias=x["bias"] + up), call(x | dict(bias=x["bias"] + up)))
    x = steer(x, up)
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,rows,dim", LONG)
def test_sums_of_rows_beyond_what_fp32_holds(n, rows, dim, dtype):
    """Rows of 2^90: their sums pass 2^128 beside a reference that weights rise above by no more than 2^40."""
    high = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda") < 1e-3
    x = steer(make(n, rows, dim, dtype, bias=False, masked=0.0), torch.where(high, 28.0, 0.0))
    x = x | dict(q=x["q"] * 2.0 ** -90, table=x["table"] * 2.0 ** 90)
    check(x, call(x))
