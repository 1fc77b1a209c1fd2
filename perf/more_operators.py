"""Cases of the node-table operators for timing: rows of a learned table of nodes looked up, the loss of a destination among
all nodes, and the step that trains them.

A case names one call pattern (`kind`):

  lookup   lookup and its backward pass: rows of a table by node id, scaled; an id below 0 (an unused neighbor slot) gives
           zeros; the gradient of the whole table from that of the rows
  loss     destination_loss and (grad) its backward pass: every root scored against all rows of the table, softmax cross
           entropy with its target, and the gradients of the root, the table and the bias
  adam     one AdamW step over many tensors, with states in 32 or 8 bits; in 8 bits the states are read back as values, as a
           checkpoint does

Definitions (both forms, and the 64-bit one):

  lookup                 out[i] = scale * table[ids[i]], 0 where ids[i] < 0;  dtable[r] = scale * sum of dout[i] with ids[i] = r
  loss                   z[i, j] = scale * q[i].table[j] + bias[j];  loss[i] = log(sum_j exp(z[i, j])) - z[i, target[i]], 0 where
                         target[i] < 0 (a masked event);  dz[i, j] = g[i] * (p[i, j] - [j = target[i]]), 0 for masked events
  AdamW                  g = grad * grad_scale;  m' = b1 m + (1 - b1) g;  v' = b2 v + ((1 - b2) g) g;  t = steps so far + 1
                         p' = p - lr * (decay * p + (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps))
  states in 8 bits       blocks of 256 values with one scale each for m and for u = sqrt(v), every operation in fp32 and rounded:
                         top = largest magnitude of the block, L = 127 (m) or 255 (u), scale = top * fp32(1 / L^2), y = |x| * (1 / scale),
                         c = floor(sqrt(y)), at most L;  one up where y - c^2 > a * (2 c + 1) and c < L;  c = 1 where u > 0 had 0;
                         value c^2 * scale, with m's sign;  v = u * u;  a block with top < 2^-60 holds zeros, its scale too
                         a = (16 bits of a hash + 0.5) / 65536: the hash is SplitMix64's finaliser of
                         seed ^ t * 0x9E3779B97F4A7C15 ^ (tensor * 2^40 + element // 2) * 0xC2B2AE3D27D4EB4F, its bits 0-15 (m) and
                         16-31 (u) for even elements, 32-47 and 48-63 for odd ones
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
LR, B1, B2, EPS, DECAY, GRAD_SCALE, STEPS = 1e-3, 0.9, 0.999, 1e-8, 0.01, 0.5, 100
BLOCK = 256


# ------------------------------------------------------------------------------------------------- the cases --
def _lookup(name, rows, dim, n, zipf, bits, dtype, out):
    return dict(name=name, kind="lookup", rows=rows, dim=dim, n=n, zipf=zipf, bits=bits, dtype=dtype, out=out)


def _loss(name, n, rows, dim, dtype, bias, masked, grad):
    return dict(name=name, kind="loss", n=n, rows=rows, dim=dim, dtype=dtype, bias=bias, masked=masked, grad=grad)


def _adam(name, table, tensors, most, bits, grads, copy):
    return dict(name=name, kind="adam", table=table, tensors=tensors, most=most, bits=bits, grads=grads, copy=copy)


def listed():
    return [
        # the neighbor slots of the smallest configuration's batch
        _lookup("lookup_tiny_f32", 1000, 32, 6000, 1.1, 32, "f32", "f32"),
        # the slots of a Wikipedia-shaped batch, rows of 100
        _lookup("lookup_wiki_f32", 9000, 100, 36_000, 1.2, 32, "f32", "f32"),
        # the slots of large batches with wide windows: few nodes, very many ids, hubs
        _lookup("lookup_hubs_bf16", 17_000, 128, 921_600, 1.2, 32, "bf16", "bf16"),
        # a table of very many nodes of which a batch touches a few: the gradient is mostly zeros
        _lookup("lookup_sparse_f32", 1_000_000, 64, 100_000, 0.7, 64, "f32", "f32"),
        # one batch of the smallest configuration against its nodes
        _loss("loss_tiny_f32", 200, 1000, 32, "f32", True, 0.0, True),
        # a Wikipedia-shaped batch in full precision
        _loss("loss_wiki_f32", 600, 9000, 100, "f32", True, 0.0, True),
        # a large batch with replay events (masked) in 16 bits, rows of 100
        _loss("loss_replay_bf16", 4800, 17_000, 100, "bf16", True, 0.17, True),
        # the same batch over very many nodes, no bias
        _loss("loss_many_bf16", 4800, 200_000, 128, "bf16", False, 0.0, True),
        # an evaluation pass: the loss alone
        _loss("loss_eval_bf16", 4000, 17_000, 100, "bf16", True, 0.0, False),
        # the tensors of the smallest configuration's model and its table
        _adam("adam_tiny_32", 32_000, 18, 12_000, 32, "f32", False),
        # the tensors of a Wikipedia-shaped model with states in 8 bits
        _adam("adam_wiki_8", 900_000, 18, 142_000, 8, "f32", False),
        # a table of very many nodes with 16-bit gradients and a 16-bit copy, states in 8 bits
        _adam("adam_many_8", 25_600_000, 18, 142_000, 8, "bf16", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "loss", "adam"])
    dims = [8, 16, 25, 32, 50, 64, 100, 101, 128, 172, 200, 256]
    most = {m: max(work(c)[m] for c in listed() if c["kind"] == kind) for m in ("bytes", "flops")}
    if kind == "lookup":
        c = _lookup("", _log(rng, 10, 1_000_000), rng.choice(dims), _log(rng, 1, 1_000_000), rng.choice([0.0, 0.7, 1.1, 1.5]),
                    rng.choice([32, 64]), rng.choice(list(DTYPES)), rng.choice(list(DTYPES)))
        smaller = "n" if rng.random() < 0.5 else "rows"
    elif kind == "loss":
        c = _loss("", _log(rng, 1, 5000), _log(rng, 10, 200_000), rng.choice(dims), rng.choice(["f32", "bf16"]), rng.random() < 0.5,
                  rng.choice([0.0, 0.2, 0.9]), rng.random() < 0.8)
        smaller = "n" if rng.random() < 0.5 else "rows"
    else:
        c = _adam("", _log(rng, 1, 25_000_000), rng.randint(1, 20), _log(rng, 1, 300_000), rng.choice([8, 32]),
                  rng.choice(["f32", "bf16"]), rng.random() < 0.3)
        smaller = "table"
    while any(work(c)[m] > most[m] for m in most) or (kind == "loss" and c["n"] * c["rows"] > 9.6e8):
        if c[smaller] <= 16:
            smaller = {"n": "rows", "rows": "n", "table": "most"}[smaller]
        c[smaller] = max(1, c[smaller] * 2 // 3)
    del c["name"]
    return c


def _sizes(case):
    """Elements of the tensors: the table, then weights and biases of many sizes up to `most`."""
    return [case["table"]] + [max(1, case["most"] * (37 * k % 101) // 101 if k % 3 else 1 + 13 * k) for k in range(1, case["tensors"])]


def work(case):
    k = case["kind"]
    if k == "lookup":
        n, d = case["n"], case["dim"]
        seen = min(n, case["rows"])
        return {"bytes": 2.0 * n * case["bits"] / 8 + seen * d * SIZE[case["dtype"]] + 2.0 * n * d * SIZE[case["out"]]
                + case["rows"] * d * SIZE[case["dtype"]], "flops": 3.0 * n * d}
    if k == "loss":
        n, N, d = case["n"] * (1.0 - case["masked"]), case["rows"], case["dim"]
        values = (case["n"] + N) * d * SIZE[case["dtype"]]
        return {"bytes": values * (2 if case["grad"] else 1) + case["n"] * 12 + (N * 8 if case["bias"] else 0),
                "flops": (6.0 if case["grad"] else 2.0) * n * N * d}
    n = sum(_sizes(case))
    held = n * 16.0 if case["bits"] == 32 else n * 4.0 + 4 * 4.0 * (n // BLOCK + 1) + n * 8.0
    return {"bytes": n * (8.0 + SIZE[case["grads"]]) + held + (2.0 * n if case["copy"] else 0), "flops": 15.0 * n}


# ------------------------------------------------------------------------------------------------ their inputs --
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _nodes(rows, zipf, n, g):
    """Node ids as a batch's endpoints and their neighbors have: Zipf over the nodes, in an order of their own."""
    w = torch.arange(1, rows + 1, dtype=torch.float64, device="cuda") ** -zipf
    cum = torch.cumsum(w, 0)
    at = torch.searchsorted(cum, torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * cum[-1]).clamp_(max=rows - 1)
    return torch.randperm(rows, generator=g, device="cuda")[at]


def _rows(n, dim, g, spread=0.5):
    x = torch.randn(n, dim, generator=g, device="cuda")
    return x * torch.exp(spread * torch.randn(n, 1, generator=g, device="cuda"))


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    k = case["kind"]
    if own:
        from paper_2608_16305_b200 import binding as B, destinations as D
        st["B"], st["D"] = B, D
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if k == "lookup":
        n, rows, dim = case["n"], case["rows"], case["dim"]
        ids = _nodes(rows, case["zipf"], n, g)
        st["ids"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.05, torch.full_like(ids, -1), ids)
        st["ids"] = st["ids"].to(torch.int32 if case["bits"] == 32 else torch.int64)
        st["table"] = _rows(rows, dim, g).to(DTYPES[case["dtype"]])
        st["dout"] = _rows(n, dim, g).to(DTYPES[case["out"]])
        st["scale"] = math.sqrt(dim)
        if own:
            st["out"], st["dtable"] = torch.empty_like(st["dout"]), torch.empty_like(st["table"])
            st["scratch"] = torch.empty(B.lookup_scratch(n, rows, dim), dtype=torch.uint8, device="cuda")
    elif k == "loss":
        n, N, d = case["n"], case["rows"], case["dim"]
        dt = DTYPES[case["dtype"]]
        table = _rows(N, d, g, 0.2)
        target = _nodes(N, 0.7, n, g)
        known = torch.rand(n, 1, generator=g, device="cuda") ** 2          # some destinations are known well, most hardly
        st["q"] = (known * table[target] + 0.6 * _rows(n, d, g, 0.2)).to(dt)
        st["table"] = table.to(dt)
        hide = torch.rand(n, generator=g, device="cuda") < case["masked"]
        st["target"] = torch.where(hide, torch.full_like(target, -1), target).to(torch.int32)
        st["bias"] = torch.randn(N, generator=g, device="cuda") if case["bias"] else None
        st["dloss"] = (0.5 + torch.rand(n, generator=g, device="cuda")) / max(1.0, n * (1.0 - case["masked"]))
        st["scale"] = 1.0 / math.sqrt(d)
        if own:
            st["loss"] = torch.empty(n, device="cuda")
            st["kept"] = torch.empty(B.destination_loss_kept(n, d), device="cuda") if case["grad"] else None
            st["scratch"] = torch.empty(B.destination_loss_scratch(n, N, d, dt), dtype=torch.uint8, device="cuda")
            st["dq"], st["dtable"] = torch.empty_like(st["q"]), torch.empty_like(st["table"])
            st["dbias"] = torch.empty_like(st["bias"]) if case["bias"] else None
    else:
        sizes = _sizes(case)
        st["p"] = [0.1 * torch.randn(s, generator=g, device="cuda") for s in sizes]
        st["g"] = []
        for s in sizes:                                    # gradients of rows of very different frequency, and zeros
            row = torch.exp(2.0 * torch.randn((s + 63) // 64, 1, generator=g, device="cuda"))
            row = torch.where(torch.rand(row.shape, generator=g, device="cuda") < 0.2, torch.zeros_like(row), row)
            x = 1e-3 * row * torch.randn((s + 63) // 64, 64, generator=g, device="cuda")
            st["g"].append(x.reshape(-1)[:s].to(DTYPES[case["grads"]]))
        st["m"] = [0.1 * x.float() for x in st["g"]]
        st["v"] = [0.5 * x.float() * x.float() + 1e-8 * torch.rand(x.numel(), generator=g, device="cuda") for x in st["g"]]
        st["decay"] = [0.0 if i % 3 == 0 and i else DECAY for i in range(len(sizes))]
        st["copy"] = [torch.empty(s, dtype=torch.bfloat16, device="cuda") if case["copy"] and i == 0 else None for i, s in enumerate(sizes)]
        st["seed"] = 1234 + seed
        if case["bits"] == 8:                              # what a program holds after some steps
            for i in range(len(sizes)):
                a = _chance(st["seed"], STEPS, i, sizes[i])
                st["m"][i], st["v"][i] = _held(st["m"][i], 127, a[0]), _held(torch.sqrt(st["v"][i]), 255, a[1])
        st["t"] = STEPS
        if own:
            st["opt"] = st["D"].AdamW(st["p"], lr=LR, betas=(B1, B2), eps=EPS, weight_decay=st["decay"], bits=case["bits"],
                                      seed=st["seed"], copies=st["copy"])
            st["opt"].steps[0] = STEPS
            for i in range(len(sizes)):
                for name in ("m", "v"):
                    mine, x = getattr(st["opt"], name)[i], st[name][i]
                    mine.copy_(x if case["bits"] == 32 else x[0])
                    if case["bits"] == 8:
                        getattr(st["opt"], name + "_scale")[i].copy_(x[1])
            del st["m"], st["v"]
        elif case["bits"] == 8:
            st["m"], u = ([_value(x) for x in st[name]] for name in ("m", "v"))
            st["v"] = [x * x for x in u]
    return st


# --------------------------------------------------------------------------------------------- the plain forms --
def _plain_lookup(st):
    ids = st["ids"].long()
    ok = ids >= 0
    at = torch.where(ok, ids, torch.zeros_like(ids))
    out = torch.where(ok[:, None], st["table"][at].float() * st["scale"], torch.zeros((), device="cuda")).to(st["dout"].dtype)
    d = torch.zeros(st["table"].shape, dtype=torch.float64, device="cuda")     # a hub's sum is long
    d.index_add_(0, at, torch.where(ok[:, None], st["dout"].double() * st["scale"], torch.zeros((), dtype=torch.float64, device="cuda")))
    return out, d.to(st["table"].dtype)


def _plain_loss(st):
    case = st["case"]
    q, table = st["q"].float(), st["table"].float()
    ok = st["target"] >= 0
    at = torch.where(ok, st["target"].long(), torch.zeros_like(st["target"].long()))
    z = torch.matmul(q, table.t()) * st["scale"]
    if st["bias"] is not None:
        z = z + st["bias"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    hit = z.gather(1, at[:, None])
    loss = torch.where(ok, (torch.log(total) + top - hit)[:, 0], torch.zeros_like(total[:, 0]))
    if not case["grad"]:
        return loss
    dz = e / total
    dz.scatter_add_(1, at[:, None], torch.full_like(hit, -1.0))
    dz *= torch.where(ok, st["dloss"], torch.zeros_like(st["dloss"]))[:, None]
    dq = (torch.matmul(dz, table) * st["scale"]).to(st["q"].dtype)
    dt = (torch.matmul(dz.t(), q) * st["scale"]).to(st["table"].dtype)
    return (loss, dq, dt) if st["bias"] is None else (loss, dq, dt, dz.sum(0))


def _mix(z):
    """SplitMix64's finaliser on int64 that wraps."""
    for shift, factor in ((30, 0xBF58476D1CE4E5B9), (27, 0x94D049BB133111EB)):
        z = (z ^ ((z >> shift) & ((1 << (64 - shift)) - 1))) * (factor - (1 << 64))
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _wrap(x):
    x &= (1 << 64) - 1
    return x - (1 << 64) if x >> 63 else x


def _chance(seed, t, tensor, n):
    """Two numbers in (0, 1) per element: for m and for u."""
    e = torch.arange(n, device="cuda")
    h = _mix(((e >> 1) + (tensor << 40)) * _wrap(0xC2B2AE3D27D4EB4F) ^ _wrap(seed ^ (t * 0x9E3779B97F4A7C15)))
    h = h >> ((e & 1) << 5)
    return [(((h >> s) & 0xFFFF).float() + 0.5) / 65536.0 for s in (0, 16)]


def _held(x, L, a):
    """Codes (signed) and scales that x becomes in 8 bits."""
    n = x.numel()
    pad = lambda v: torch.nn.functional.pad(v, (0, -n % BLOCK)).view(-1, BLOCK)
    x, a = pad(x), pad(a)
    top = x.abs().amax(1, keepdim=True)
    fine = top >= 2.0 ** -60
    s = torch.where(fine, top * float(np.float32(1.0 / (L * L))), torch.zeros_like(top))
    y = x.abs() * torch.where(fine, torch.reciprocal(s), torch.zeros_like(s))
    c = torch.floor(torch.sqrt(y))
    c = torch.where(c * c > y, c - 1.0, c)
    c = torch.where((c + 1.0) * (c + 1.0) <= y, c + 1.0, c).clamp(max=float(L))
    c = torch.where((y - c * c > a * (2.0 * c + 1.0)) & (c < L), c + 1.0, c)
    if L == 255:
        c = torch.where((c == 0.0) & (x > 0.0) & fine, torch.ones_like(c), c)
    return (torch.sign(x) * c).reshape(-1)[:n].to(torch.int16), s[:, 0].contiguous()


def _value(held):
    """The numbers that codes and scales stand for."""
    c = held[0].float()
    s = held[1].repeat_interleave(BLOCK)[:c.numel()]
    return torch.sign(c) * (c * c) * s


def _plain_adam(st):
    case = st["case"]
    st["t"] += 1
    t = st["t"]
    one = torch.ones((), device="cuda")
    c1, c2 = float(1.0 - B1 ** t), float(1.0 - B2 ** t)
    b1, b2, n1, n2 = (float(np.float32(x)) for x in (B1, B2, 1.0 - np.float32(B1), 1.0 - np.float32(B2)))
    for i, p in enumerate(st["p"]):
        g = st["g"][i].float() * GRAD_SCALE
        m = st["m"][i] * b1 + g * n1
        v = st["v"][i] * b2 + (g * n2) * g
        u = torch.sqrt(v)
        p -= LR * (st["decay"][i] * p + (m / c1) / (u / math.sqrt(c2) + EPS * one))
        if case["bits"] == 8:
            a = _chance(st["seed"], t, i, p.numel())
            m, u = _value(_held(m, 127, a[0])), _value(_held(u, 255, a[1]))
            v = u * u
        st["m"][i], st["v"][i] = m, v
        if st["copy"][i] is not None:
            st["copy"][i].copy_(p)
    return _adam_outputs(st, st["m"], st["v"])


def _adam_outputs(st, m, v):
    """Parameters, first and second moments, one after the other (the table's copy is its rounding, and comes last)."""
    return [*st["p"], *m, *v, *(c for c in st["copy"] if c is not None)]


# ------------------------------------------------------------------------------------------------- the passes --
def run(st):
    case = st["case"]
    k = case["kind"]
    if not own:
        return {"lookup": _plain_lookup, "loss": _plain_loss, "adam": _plain_adam}[k](st)
    B = st["B"]
    if k == "lookup":
        B.lookup(st["table"], st["ids"], st["out"], st["status"], scale=st["scale"])
        B.lookup_backward(st["ids"], st["dout"], st["dtable"], st["scratch"], st["status"], scale=st["scale"])
        return st["out"], st["dtable"]
    if k == "loss":
        B.destination_loss(st["q"], st["table"], st["target"], st["loss"], st["scratch"], st["status"], bias=st["bias"],
                           kept=st["kept"], scale=st["scale"])
        if not case["grad"]:
            return st["loss"]
        B.destination_loss_backward(st["q"], st["table"], st["target"], st["kept"], st["dloss"], st["dq"], st["dtable"],
                                    st["scratch"], st["status"], bias=st["bias"], dbias=st["dbias"], scale=st["scale"])
        return (st["loss"], st["dq"], st["dtable"]) if st["bias"] is None else (st["loss"], st["dq"], st["dtable"], st["dbias"])
    opt = st["opt"]
    opt.step(st["g"], grad_scale=GRAD_SCALE)
    return _adam_outputs(st, *opt.moments())


# --------------------------------------------------------------------------------- the definitions in 64 bits --
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"lookup": _exact_lookup, "loss": _exact_loss, "adam": _exact_adam}[case["kind"]](st)


def _exact_lookup(st):
    """Ids sorted, sums of runs as differences of running sums within each run's own origin."""
    rows, dim = st["table"].shape
    ids, order = torch.sort(st["ids"].long(), stable=True)
    used = order[ids >= 0]
    out = torch.zeros(st["dout"].shape, dtype=torch.float64, device="cuda")
    out[used] = st["table"].double().index_select(0, ids[ids >= 0]) * st["scale"]
    lengths = torch.bincount(ids[ids >= 0], minlength=rows)
    d = torch.segment_reduce(st["dout"].double()[used], "sum", lengths=lengths, axis=0, initial=0.0) if used.numel() else \
        torch.zeros(rows, dim, dtype=torch.float64, device="cuda")
    return out, d * st["scale"]


def _exact_loss(st):
    """Some roots at a time; gradients by the library's differentiation of the loss."""
    case = st["case"]
    n, N = case["n"], case["rows"]
    leaf = lambda x: None if x is None else x.double().requires_grad_(bool(case["grad"]))
    table, bias = leaf(st["table"]), leaf(st["bias"])
    q = leaf(st["q"])
    losses, dq = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    step = max(1, int(2e8 / N))
    for r0 in range(0, n, step):
        r = slice(r0, min(n, r0 + step))
        ok = torch.nonzero(st["target"][r] >= 0)[:, 0]
        if not ok.numel():
            continue
        rows = q[r][ok]
        z = st["scale"] * torch.einsum("id,jd->ij", rows, table)
        z = z if bias is None else z + bias[None]
        each = torch.logsumexp(z, 1) - z[torch.arange(len(ok), device="cuda"), st["target"][r][ok].long()]
        losses[r0 + ok] = each.detach()
        if case["grad"]:
            (each * st["dloss"][r][ok].double()).sum().backward()
    if not case["grad"]:
        return losses
    zero = lambda x: torch.zeros_like(x) if x.grad is None else x.grad
    out = (losses, zero(q), zero(table))
    return out if bias is None else out + (zero(bias),)


def _exact_adam(st):
    """Parameters in 64 bits; states in 8 bits by their definition, whose fp32 roundings are part of it, on the host."""
    case, t = st["case"], STEPS + 1
    P, M, V, copies = [], [], [], []
    f32 = np.float32
    for i, p in enumerate(st["p"]):
        g = st["g"][i].double() * GRAD_SCALE
        b1, b2 = float(f32(B1)), float(f32(B2))
        m = torch.lerp(g, st["m"][i].double(), b1)
        v = torch.lerp(g.square(), st["v"][i].double(), b2)
        new = p.double() * (1.0 - LR * st["decay"][i]) - LR * (m / -math.expm1(t * math.log(B1))) / (torch.sqrt(v / -math.expm1(t * math.log(B2))) + EPS)
        P.append(new)
        if st["copy"][i] is not None:
            copies.append(new)
        if case["bits"] == 8:
            n = p.numel()
            gh = st["g"][i].float().cpu().numpy() * f32(GRAD_SCALE)
            mh, vh = st["m"][i].cpu().numpy(), st["v"][i].cpu().numpy()
            m32 = mh * f32(B1) + gh * (f32(1) - f32(B1))
            u32 = np.sqrt(vh * f32(B2) + gh * (f32(1) - f32(B2)) * gh)
            e = np.arange(n, dtype=np.uint64)
            with np.errstate(over="ignore"):
                h = (np.uint64((i << 40)) + e // np.uint64(2)) * np.uint64(0xC2B2AE3D27D4EB4F)
                h ^= np.uint64((st["seed"] ^ (t * 0x9E3779B97F4A7C15)) & 0xFFFFFFFFFFFFFFFF)
                h = (h ^ (h >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
                h = (h ^ (h >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
                h ^= h >> np.uint64(31)
            words = h >> (e % np.uint64(2) * np.uint64(32))
            halves = [(words & np.uint64(0xFFFF)), (words >> np.uint64(16)) & np.uint64(0xFFFF)]
            held = []
            for x, L, bits in ((m32, 127, halves[0]), (u32, 255, halves[1])):
                a = (bits.astype(f32) + f32(0.5)) / f32(65536)
                top = np.maximum.reduceat(np.abs(x), np.arange(0, n, BLOCK))
                scale = np.where(top >= f32(2.0 ** -60), top * f32(1.0 / (L * L)), f32(0))
                with np.errstate(divide="ignore"):
                    back = np.where(scale > 0, f32(1) / scale, f32(0))
                scale, back = (np.repeat(w, BLOCK)[:n] for w in (scale, back))
                y = np.abs(x) * back
                c = np.minimum(np.floor(np.sqrt(y.astype(np.float64))), L).astype(f32)
                c += (c < L) & (y - c * c > a * (2 * c + 1))
                if L == 255:
                    c = np.where((c == 0) & (x > 0) & (scale > 0), f32(1), c)
                held.append(np.copysign(c * c * scale, x).astype(np.float64))
            m, u = (torch.from_numpy(h).cuda() for h in held)
            v = (u.float() * u.float()).double()
        M.append(m)
        V.append(v)
    return P + M + V + copies
