"""The destination loss where the reference of a row's weights may lie far above all of its logits: products far below zero, and hidden nodes with
products above all others.  Against the formulas in 64 bits, with the bounds of test_gpu_destination.py; shares of one tile and of ten and more, in
every form of the kernels (rows to 128 values and above, few and many roots)."""
import math

import pytest
import torch

from tests.test_gpu_destination import BF16, F32, call, check, make

pytestmark = pytest.mark.gpu

# Few roots (a block joins four of them) and many (a warp does), over so many nodes that 148 blocks have ten tiles of 128 (or 64) nodes each and more.
LONG = [(200, 190_000, 40), (120, 190_000, 160), (2600, 17_500, 40), (1400, 17_500, 160)]


def steer(x, add):
    """Products of every root raised by add[j] (natural units): one more column that all roots share, and nothing else of it in the table."""
    q, t = x["q"].float(), x["table"].float()
    q[:, 0], t[:, 0] = 16.0, torch.as_tensor(add, device="cuda", dtype=torch.float32) / (16.0 * x["scale"])
    return x | dict(q=q.to(x["q"].dtype), table=t.to(x["table"].dtype))


def check_seen(x, out, seen):
    """The nodes that are not seen get nothing, and all else is as without them."""
    for k in ("dtable", "dbias"):
        if out.get(k) is not None:
            assert bool((out[k][~seen] == 0).all()), k
    place = torch.cumsum(seen, 0) - 1
    y = x["target"].long()
    y = torch.where(y >= 0, place[y.clamp(min=0)], y)
    check(x | dict(table=x["table"][seen].contiguous(), bias=x["bias"][seen].contiguous(), target=y),
          {k: v[seen] if k in ("dtable", "dbias") else v for k, v in out.items()})


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dim", [40, 160])
@pytest.mark.parametrize("n,rows", [(7, 10), (20, 130), (20, 900), (300, 2001)])
def test_all_products_far_below_zero(n, rows, dim, bias, dtype):
    """Nothing but a shift of all logits, which the softmax does not mind; behind the table's end there are products of 0."""
    x = steer(make(n, rows, dim, dtype, bias, masked=0.0), [-150.0] * rows)
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("low", [-math.inf, -1e4, torch.finfo(F32).min])
@pytest.mark.parametrize("above", [60.0, 86.0, 150.0])
@pytest.mark.parametrize("n,rows,dim", [(20, 200, 40), (300, 1500, 40), (100, 900, 160)] + LONG)
def test_hidden_nodes_with_the_largest_products(n, rows, dim, above, low, dtype):
    hidden = torch.arange(rows, device="cuda") % 61 == 0                     # in every 64 nodes
    x = steer(make(n, rows, dim, dtype, masked=0.0), torch.where(hidden, above, 0.0))
    x["bias"] = torch.where(hidden, torch.full_like(x["bias"], low), x["bias"])
    y = x["target"].long()
    x["target"] = torch.where(hidden[y], (y + 1) % 60 + 1, y)
    check_seen(x, call(x), ~hidden)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("low", [-math.inf, -1e9])
@pytest.mark.parametrize("n,rows,dim", LONG)
def test_hidden_tiles_at_the_start_of_shares(n, rows, dim, low, dtype):
    """Two tiles of three hide nodes only, with products above and below the others'."""
    at = torch.arange(rows, device="cuda")
    hidden = at // 128 % 3 != 1
    x = steer(make(n, rows, dim, dtype, masked=0.1), torch.where(hidden, (at // 128 % 2 * 2 - 1) * 50.0, 0.0))
    x["bias"] = torch.where(hidden, torch.full_like(x["bias"], low), x["bias"])
    y = x["target"].long()
    x["target"] = torch.where(y >= 0, 128 + y % 128, y)
    check_seen(x, call(x), ~hidden)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("low", [-math.inf, -1e9])
@pytest.mark.parametrize("n,rows,dim", [(9, 300, 40), (300, 4000, 160)])
def test_a_single_node_in_sight(n, rows, dim, low, dtype):
    """It is certain: no loss and no gradient, however large the hidden products are."""
    for above in (-150.0, 0.0, 150.0):
        x = steer(make(n, rows, dim, dtype, masked=0.0), [above] * rows)
        x["bias"][:] = low
        x["bias"][70] = 0.25
        x["target"][:] = 70
        out = call(x)
        assert all(bool((v == 0).all()) for v in out.values()), above


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("low", [-math.inf, -1e4, -1e9, torch.finfo(F32).min])
@pytest.mark.parametrize("n,rows,dim", [(20, 131, 40), (300, 900, 100), (90, 1000, 200)])
def test_a_target_among_hidden_nodes(n, rows, dim, low, dtype):
    """The only node in sight of its tile, beside masks of any size: its logit is not lost in theirs."""
    x = make(n, rows, dim, dtype, masked=0.0)
    seen = torch.arange(rows, device="cuda") % 128 >= 64
    seen[rows - 2] = True
    seen[256:384] = False
    seen[300:301] = True
    x["bias"][~seen] = low
    x["target"][:] = rows - 2
    if rows > 300:
        x["target"][::2] = 300
    check_seen(x, call(x), seen)
