"""The loss of a destination among all nodes and its gradients, against the formulas in 64 bits.

Tolerances.  A logit is a sum of dim products in fp32, where the tensor cores may cut each of the additions (2^-23 of the partial sum); fp32 operands
are held in 22 bits and lo x lo is left out (3 * 2^-22 of a product's magnitude); z then passes three fp32 roundings (factor, sum, difference).
A weight is 2^x to 2^-22.  Sums over nodes (roots) have chains of 34 additions in a tile and one per tile.  Products with weights round them to bf16 (half a step: 2^-8), or
to 22 bits, and add one step of 16 after the other (2^-23 each).  All of it is bounded by the sum of the terms' magnitudes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def make(n, rows, dim, dtype, bias=True, masked=0.2, seed=0, spread=1.0, sure=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * n + rows)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    table = (spread * r(rows, dim)).to(dtype)
    target = torch.randint(0, rows, (n,), generator=g, device="cuda", dtype=torch.int32)
    q = (spread * r(n, dim) + sure * table[target.long()].float()).to(dtype)
    target = torch.where(torch.rand(n, generator=g, device="cuda") < masked, torch.full_like(target, -1), target)
    return dict(q=q, table=table, target=target, bias=r(rows) if bias else None, g=r(n) / n, scale=1.0 / math.sqrt(dim))


def call(x, want=("dq", "dtable", "dbias"), scratch=None, status=None):
    from paper_2608_16305_b200 import binding as B
    q, table = x["q"], x["table"]
    (n, dim), rows = q.shape, table.shape[0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda") if status is None else status
    size = B.destination_loss_scratch(n, rows, dim, q.dtype)
    scratch = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if scratch is None else scratch      # NaN wherever nothing was written
    out = dict(loss=torch.full((n,), 7.0, device="cuda"), alone=torch.full((n,), 7.0, device="cuda"))
    kept = torch.full((B.destination_loss_kept(n, dim),), float("nan"), device="cuda")
    B.destination_loss(q, table, x["target"], out["alone"], scratch, status, bias=x["bias"], scale=x["scale"])
    B.destination_loss(q, table, x["target"], out["loss"], scratch, status, bias=x["bias"], kept=kept, scale=x["scale"])
    like = dict(dq=q, dtable=table, dbias=x["bias"])
    for k in want:
        out[k] = None if like[k] is None else torch.full_like(like[k], float("nan"))
    scratch.fill_(0xFF)
    B.destination_loss_backward(q, table, x["target"], kept, x["g"], out.get("dq"), out.get("dtable"), scratch, status, bias=x["bias"],
                                dbias=out.get("dbias"), scale=x["scale"])
    assert int(status.item()) == 0
    return out


def check(x, out):
    q, t, y, g, c = x["q"].double(), x["table"].double(), x["target"].long(), x["g"].double(), float(x["scale"])
    dtype = x["q"].dtype
    n, dim = q.shape
    rows = t.shape[0]
    live = y >= 0
    q = torch.where(live[:, None], q, torch.zeros_like(q))
    g = torch.where(live, g, torch.zeros_like(g))
    at = y.clamp(min=0)
    z = c * q @ t.T
    mag = abs(c) * q.abs() @ t.abs().T
    if x["bias"] is not None:
        z = z + x["bias"].double()
        mag = mag + torch.where(torch.isfinite(x["bias"]), x["bias"], torch.zeros_like(x["bias"])).double().abs()
    others = z.clone()
    others[torch.arange(n), at] = -math.inf
    zt = z.gather(1, at[:, None])[:, 0]
    top = torch.maximum(others.amax(1), zt)
    e = torch.exp(others - top[:, None])
    total = e.sum(1) + torch.exp(zt - top)
    p = e / total[:, None]                                                   # 0 at the target
    miss = p.sum(1)
    loss = torch.where(live, torch.where(miss < 0.5, -torch.log1p(-miss), torch.log(total) + top - zt), torch.zeros_like(zt))
    # what a logit may be off by, per row (natural units), and what a weight may, relative to itself
    per = (dim + 8) * 2.0 ** -23 + (3 * 2.0 ** -22 if dtype == F32 else 0.0)
    ez = mag.amax(1) * per
    ep = 2 * ez + 2.0 ** -21 + (42 + rows / 64) * 2.0 ** -24
    lim = ep * torch.minimum(torch.ones_like(loss), 2 * loss) + (loss + 1e-30) * 2.0 ** -21
    # the log itself: of a sum that is ep off, no more than ep, and where it is small no more than its own part
    for k in ("alone", "loss"):
        err = (out[k].double() - loss).abs()
        assert bool((err <= lim).all()), (k, float((err / lim).max()))
        assert bool((out[k][~live] == 0).all())
    weight = 2.0 ** -8 if dtype == BF16 else 2.0 ** -21
    half = torch.finfo(dtype).eps / 2 * 1.01
    if out.get("dq") is not None:
        ref = (g * c)[:, None] * (p @ t - miss[:, None] * t[at])
        size = (g * c).abs()[:, None] * (p @ t.abs() + miss[:, None] * t[at].abs())
        lim = size * (ep[:, None] + weight + rows / 16 * 2.0 ** -23 + 2.0 ** -20) + (ref.abs() + size * 2.0 ** -7) * half + 1e-37       # the value rounded is not quite ref
        err = (out["dq"].double() - ref).abs()
        assert bool((err <= lim).all()), ("dq", float((err / lim).max()))
        assert bool((out["dq"][~live] == 0).all())
    dz = p * g[:, None]
    dz[torch.arange(n), at] = -g * miss
    rel = ep[:, None] + 2.0 ** -21
    if out.get("dtable") is not None:
        ref = c * dz.T @ q
        size = abs(c) * (dz.abs() * (rel + weight + n / 16 * 2.0 ** -23)).T @ q.abs()
        if dtype == F32:                                                     # weights in fp16 pairs: 2^-40 of the largest gradient at least
            size = size + abs(c) * 2.0 ** -39 * g.abs().max() * q.abs().sum(0)[None]
        lim = size * (1 + half) + ref.abs() * half + 1e-37
        err = (out["dtable"].double() - ref).abs()
        assert bool((err <= lim).all()), ("dtable", float((err / lim).max()))
    if out.get("dbias") is not None:
        ref = dz.sum(0)
        lim = (dz.abs() * (rel + (36 + n / 64) * 2.0 ** -24)).sum(0) + 1e-37
        err = (out["dbias"].double() - ref).abs()
        assert bool((err <= lim).all()), ("dbias", float((err / lim).max()))


SIZES = [(1, 1, 1), (1, 2, 8), (3, 5, 16), (127, 129, 32), (128, 128, 64), (129, 1000, 100), (256, 256, 128), (257, 300, 128), (300, 513, 129),
         (64, 2000, 172), (200, 700, 256), (1000, 130, 50), (40, 5000, 25), (2000, 3000, 101), (513, 20_001, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("n,rows,dim", SIZES)
def test_against_64_bits(n, rows, dim, dtype, bias):
    x = make(n, rows, dim, dtype, bias, masked=0.2 if n > 3 else 0.0)
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", list(range(1, 33)) + [48, 63, 65, 80, 96, 111, 112, 113, 127, 130, 192, 208, 240, 255])
def test_widths(dim, dtype):
    x = make(150, 260, dim, dtype, seed=dim)
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("sure", [0.5, 1.0, 2.0, 4.0, 8.0])
def test_destinations_that_are_nearly_certain(sure, dtype):
    """Losses far below 1 and their gradients keep their relative accuracy."""
    x = make(400, 900, 100, dtype, bias=True, masked=0.0, sure=sure)
    out = call(x)
    check(x, out)
    if sure >= 4:
        assert float(out["loss"].median()) < 1e-6


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_that_rise_along_the_table(dtype):
    """The reference of the weights has to move many times, by more than any type holds."""
    x = make(300, 3000, 64, dtype, bias=False, masked=0.0, spread=0.2)
    x["bias"] = torch.linspace(-400, 400, 3000, device="cuda")
    check(x, call(x))
    x["bias"] = x["bias"].flip(0).contiguous()
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [5, 400])
def test_products_that_rise_along_the_table(n, dtype):
    """The same by the rows themselves: logits of 0 to 600."""
    x = make(n, 2000, 64, dtype, bias=True, masked=0.0, spread=0.2)
    x["table"] = (x["table"].float() * 0.02 + torch.linspace(0, 1, 2000, device="cuda")[:, None]).to(dtype)
    x["q"] = (x["q"].float() * 0.02 + 75.0).to(dtype)
    out = call(x)
    check(x, out)
    assert float(out["loss"].max()) > 300
    x["table"] = x["table"].flip(0).contiguous()
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("low", [-1e4, -1e9, torch.finfo(F32).min, -math.inf])
def test_masks_over_the_first_nodes(low, dtype):
    x = make(100, 1500, 32, dtype, masked=0.1)
    x["bias"][:700] = low
    x["target"] = torch.where(x["target"] >= 0, 700 + x["target"] % 800, x["target"])
    out = call(x)
    assert bool(torch.isfinite(out["loss"]).all()) and bool((out["dtable"][:700] == 0).all()) and bool((out["dbias"][:700] == 0).all())
    check(x | dict(table=x["table"][700:].contiguous(), bias=x["bias"][700:].contiguous(), target=torch.where(x["target"] >= 0, x["target"] - 700, x["target"])),
          {k: v[700:] if k in ("dtable", "dbias") else v for k, v in out.items()})


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_hidden_nodes(dtype):
    x = make(200, 700, 40, dtype, masked=0.1)
    hidden = torch.rand(700, device="cuda") < 0.5
    hidden[x["target"][x["target"] >= 0].long()] = False
    x["bias"] = torch.where(hidden, torch.full_like(x["bias"], -math.inf), x["bias"])
    out = call(x)
    check(x, out)
    assert bool((out["dtable"][hidden] == 0).all()) and bool((out["dbias"][hidden] == 0).all())
    # a whole tile of hidden nodes first
    x["bias"][:256] = -math.inf
    x["target"] = torch.where(x["target"] < 256, torch.full_like(x["target"], -1), x["target"])
    check(x, call(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_targets_that_are_hidden(dtype):
    x = make(6, 300, 24, dtype, masked=0.0)
    y = int(x["target"][0])
    x["bias"][y] = -math.inf
    hit = x["target"] == y
    out = call(x)
    assert bool(torch.isinf(out["loss"][hit]).all()) and bool((out["loss"][hit] > 0).all()) and bool(torch.isfinite(out["loss"][~hit]).all())
    for k in ("dq", "dtable", "dbias"):
        assert bool(torch.isfinite(out[k]).all())
    p = torch.softmax(x["scale"] * x["q"].double() @ x["table"].double().T + x["bias"].double(), 1)
    ref = (x["g"].double() * x["scale"])[:, None] * (p @ x["table"].double() - x["table"].double()[x["target"].long()])
    assert float((out["dq"].double() - ref).abs().max()) <= 2.0 ** -8 * float(ref.abs().max()) * (1 if dtype == BF16 else 2.0 ** -9)
    x["bias"][:] = -math.inf                                                  # nothing in sight: no gradient
    out = call(x)
    assert bool(torch.isinf(out["loss"]).all())
    for k in ("dq", "dtable", "dbias"):
        assert bool((out[k] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masks_of_the_lowest_value(dtype):
    """All nodes at the type's lowest value are all alike: the loss is log(rows)."""
    low = torch.finfo(F32).min
    x = make(10, 500, 32, dtype, masked=0.0)
    x["bias"][:] = low
    out = call(x)
    assert float((out["loss"] - math.log(500)).abs().max()) < 1e-5
    p = 1 / 500
    want = torch.zeros(500, dtype=torch.float64, device="cuda").index_add_(0, x["target"].long(), -x["g"].double()) + p * x["g"].double().sum()
    assert float((out["dbias"].double() - want).abs().max()) <= 2.0 ** -20 * float(x["g"].abs().sum())
    x["bias"][100:300] = 0.5                                                  # beside finite ones it hides
    x["target"] = torch.randint(100, 300, (10,), device="cuda", dtype=torch.int32)
    out = call(x)
    hidden = x["bias"] == low
    assert bool((out["dtable"][hidden] == 0).all()) and bool(torch.isfinite(out["loss"]).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masked_roots_touch_nothing(dtype):
    x = make(300, 400, 64, dtype, masked=0.5)
    off = x["target"] < 0
    clean = call(x)
    x["q"][off] = float("nan")
    x["g"][off] = float("inf")
    out = call(x)
    for k in clean:
        assert torch.equal(clean[k], out[k]), k
    x["target"][:] = -5                                                       # nobody takes part
    out = call(x)
    for k in out:
        assert bool((out[k] == 0).all()), k


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_targets_beyond_the_table_are_reported(dtype):
    from paper_2608_16305_b200 import binding as B
    x = make(20, 30, 16, dtype, masked=0.0)
    y = x["target"].long()
    y[3], y[4] = 30, 2**40
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss = torch.empty(20, device="cuda")
    scratch = torch.empty(B.destination_loss_scratch(20, 30, 16, dtype), dtype=torch.uint8, device="cuda")
    B.destination_loss(x["q"], x["table"], y, loss, scratch, status, bias=x["bias"])
    assert int(status.item()) == 4 and loss[3] == 0 and loss[4] == 0
    y[3] = y[4] = -1
    again = torch.empty(20, device="cuda")
    B.destination_loss(x["q"], x["table"], y, again, scratch, status, bias=x["bias"])
    assert torch.equal(loss, again)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shift", [-60, -20, 20, 40])
def test_rows_of_any_size(dtype, shift):
    x = make(140, 300, 48, dtype, bias=True)
    x["q"], x["table"] = x["q"] * 2.0 ** shift, x["table"] * 2.0 ** (shift / 2)
    x["scale"] = 2.0 ** (-1.5 * shift) / 7
    out = call(x)
    check(x, out)


@pytest.mark.parametrize("dtype,dim", [(BF16, 64), (BF16, 128), (BF16, 100), (F32, 64)])
@pytest.mark.parametrize("offset", [1, 3])
def test_addresses_between_words(dtype, dim, offset):
    x = make(70, 200, dim, dtype)
    plain = call(x)
    for k in ("q", "table"):
        buf = torch.zeros(x[k].numel() + 8, dtype=dtype, device="cuda")
        buf[offset:offset + x[k].numel()] = x[k].reshape(-1)
        x[k] = buf[offset:offset + x[k].numel()].view(x[k].shape)
    out = call(x)
    for k in plain:
        assert torch.equal(plain[k], out[k]), k


@pytest.mark.parametrize("want", [("dq",), ("dtable",), ("dbias",), ()])
def test_parts_of_the_gradients(want):
    x = make(300, 900, 64, BF16)
    whole, part = call(x), call(x, want)
    for k in part:
        assert torch.equal(whole[k], part[k]), k


def test_many_roots_and_few_nodes():
    """Groups of rows that a block has to itself, in both directions."""
    for dtype in (BF16, F32):
        x = make(60_000, 200, 24, dtype)
        check(x, call(x))
        x = make(30, 60_000, 24, dtype, masked=0.0)
        check(x, call(x))


@pytest.mark.parametrize("dtype,dim", [(BF16, 100), (BF16, 172), (F32, 100), (F32, 172)])
def test_long_walks_without_a_backward_pass(dtype, dim):
    """Groups of rows run ahead of one another; the loss alone is the loss beside the gradients, and always the same."""
    from paper_2608_16305_b200 import binding as B
    x = make(3000, 40_000, dim, dtype, masked=0.0)
    out = call(x, ())
    assert float((out["alone"] - out["loss"]).abs().max()) <= 2.0 ** -21 * float(out["loss"].abs().max())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    scratch = torch.empty(B.destination_loss_scratch(3000, 40_000, dim, dtype), dtype=torch.uint8, device="cuda")
    again = torch.empty(3000, device="cuda")
    for _ in range(30):
        B.destination_loss(x["q"], x["table"], x["target"], again, scratch, status, bias=x["bias"], scale=x["scale"])
        assert torch.equal(again, out["alone"])
    assert int(status.item()) == 0


def test_the_same_bits_from_a_graph_and_beside_another_call():
    from paper_2608_16305_b200 import binding as B
    x, other = make(700, 5000, 100, BF16), make(500, 3000, 64, F32)
    first, first_other = call(x), call(other)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mine = torch.empty(B.destination_loss_scratch(700, 5000, 100, BF16), dtype=torch.uint8, device="cuda")
    loss, kept = torch.empty(700, device="cuda"), torch.empty(B.destination_loss_kept(700, 100), device="cuda")
    dq, dt, db = torch.empty_like(x["q"]), torch.empty_like(x["table"]), torch.empty_like(x["bias"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.destination_loss(x["q"], x["table"], x["target"], loss, mine, status, bias=x["bias"], kept=kept, scale=x["scale"])
        B.destination_loss_backward(x["q"], x["table"], x["target"], kept, x["g"], dq, dt, mine, status, bias=x["bias"], dbias=db, scale=x["scale"])
    for _ in range(3):
        with torch.cuda.stream(s):
            graph.replay()
        again = call(other)
        torch.cuda.synchronize()
        for k, v in (("loss", loss), ("dq", dq), ("dtable", dt), ("dbias", db)):
            assert torch.equal(first[k], v), k
        for k in again:
            assert torch.equal(first_other[k], again[k]), k
    assert int(status.item()) == 0


def test_gradients_under_autograd_and_by_differences():
    from paper_2608_16305_b200 import destinations as D
    x = make(30, 50, 20, F32, masked=0.2)
    q, t, b = (x[k].clone().requires_grad_() for k in ("q", "table", "bias"))
    loss = D.destination_loss(q, t, x["target"], bias=b, scale=x["scale"])
    (loss * x["g"]).sum().backward()
    check(x, dict(alone=loss.detach(), loss=loss.detach(), dq=q.grad, dtable=t.grad, dbias=b.grad))
    at = lambda **kw: float((D.destination_loss(*[kw.get(k, x[k]) for k in ("q", "table")], x["target"], bias=kw.get("bias", x["bias"]),
                                                scale=x["scale"]).double() * x["g"].double()).sum())
    h = 2.0 ** -6
    size = float(x["g"].abs().sum())
    for k, grad in (("q", q.grad), ("table", t.grad), ("bias", b.grad)):
        d = torch.randn_like(x[k])
        d /= d.norm()
        slope = (at(**{k: x[k] + h * d}) - at(**{k: x[k] - h * d})) / (2 * h)
        # central differences: h^2 / 6 of the third derivative, which is below 8 (scale |t|)^3 per unit of loss, and the losses' own 2^-20 over h
        reach = float(max(x["table"].double().norm(dim=1).max(), x["q"].double().norm(dim=1).max())) * x["scale"] if k != "bias" else 1.0
        assert abs(slope - float((grad * d).sum())) <= size * (h * h / 6 * 8 * reach ** 3 + 2.0 ** -19 / h)


def test_only_some_leaves_and_an_eager_step_beside_a_captured_one():
    """A captured backward pass while an eager graph of the same leaves lives: leaves of their own, gradients by autograd.grad."""
    from paper_2608_16305_b200 import destinations as D
    x = make(100, 300, 32, BF16)
    t = x["table"].clone().requires_grad_()
    eager = D.destination_loss(x["q"], t, x["target"], scale=x["scale"])
    (g,) = torch.autograd.grad((eager * x["g"]).sum(), t)
    mine = x["table"].clone().requires_grad_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        (warm,) = torch.autograd.grad((D.destination_loss(x["q"], mine, x["target"], scale=x["scale"]) * x["g"]).sum(), mine)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        (captured,) = torch.autograd.grad((D.destination_loss(x["q"], mine, x["target"], scale=x["scale"]) * x["g"]).sum(), mine)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g, captured) and torch.equal(g, warm)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,rows,masked", [(61_000, 600, 0.999), (61_000, 600, 0.5), (1300, 40_000, 0.2), (1300, 40_000, 0.99)])
def test_uneven_shares(n, rows, masked, dtype):
    """Walks long enough that a change of groups counts in the blocks' shares, and so few roots that some shares are nothing else."""
    x = make(n, rows, 40, dtype, masked=masked)
    check(x, call(x))
