"""Cases of the history operators for timing: attention of roots over the histories of their nodes, and the
quantised row cache that the serving form reads.

A case names one call pattern (`kind`):

  sample   sample_window: for every root the place and length of its node's visible history in the T-CSR, and the slots
           of its window (most recent entries) and sinks (first entries)
  cache    a row cache in 4 or 8 bits: rows of a table quantised as they are written, then read back into a table
           (what a boundary refresh does at its two ends, and what appending keys and values to a history cache does)
  attend   cached_attend: one query per root and head over the window and the sinks of its node's history, keys and values
           in a cache of 4 or 8 bits, with a learned bias by buckets of the time difference (scoring, serving)
  slots    slot_attend and its backward pass: one query per root and head over its sampled slots' keys and values, with the
           learned time bias and its gradient (training)

Definitions (both forms, and the 64-bit one):

  visible history of root (node n, time t)   the entries of n's T-CSR slice with ts < t, oldest first, `len` of them
  window w, sinks s                          entries j >= len - w, and entries j < s
  bucket of a time difference                the number of bounds that are <= root time - entry time (fp64)
  logit                                      scale * q.k + bias[head, bucket]; scale = 1 / sqrt(dim)
  a root that sees nothing                   output 0
  quantised group (one row, one head)        amax = max |x|; L = 7 or 127; scale = amax / L (fp32), rounded up to bf16;
                                             r = 1 / scale (fp32); code = the integer nearest to x * r, ties to even
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
SPAN = 160_000.0          # time units that a stream covers: one event per unit, as the package's streams have


# ------------------------------------------------------------------------------------------------- the cases --
def _sample(name, nodes, places, zipf, roots, window, sinks):
    return dict(name=name, kind="sample", nodes=nodes, places=places, zipf=zipf, roots=roots, window=window, sinks=sinks)


def _cache(name, table, rows, heads, dim, bits, dtype, out):
    return dict(name=name, kind="cache", table=table, rows=rows, heads=heads, dim=dim, bits=bits, dtype=dtype, out=out)


def _attend(name, nodes, places, zipf, roots, window, sinks, heads, kv_heads, dim, bits, buckets, dtype):
    return dict(name=name, kind="attend", nodes=nodes, places=places, zipf=zipf, roots=roots, window=window, sinks=sinks,
                heads=heads, kv_heads=kv_heads, dim=dim, bits=bits, buckets=buckets, dtype=dtype)


def _slots(name, roots, slots, heads, kv_heads, dim, buckets, dtype):
    return dict(name=name, kind="slots", roots=roots, slots=slots, heads=heads, kv_heads=kv_heads, dim=dim,
                buckets=buckets, dtype=dtype)


def listed():
    return [
        # the smallest batch of the package's configurations: launches and dependent loads are what it costs
        _sample("sample_tiny", 1000, 40_000, 1.1, 600, 10, 2),
        # large batches over a few hub nodes: long slices to search, more slots than lanes
        _sample("sample_hubs", 2000, 2_600_000, 1.5, 12_000, 64, 4),
        # the keys of one batch of 600 events (both endpoints) appended to a history cache
        _cache("cache_append_q4", 320_000, 1200, 2, 50, 4, "f32", "f32"),
        # the two ends of a boundary refresh: memory rows of 20 000 nodes packed in 8 bits and written back
        _cache("cache_refresh_q8", 100_000, 20_000, 1, 100, 8, "f32", "f32"),
        # a whole history written in bulk from 16-bit rows, and read for a pass in full precision
        _cache("cache_bulk_q4", 1_000_000, 1_000_000, 4, 64, 4, "bf16", "bf16"),
        # scoring one event as it arrives: three roots, a long window, nothing to share
        _attend("attend_one_event_q4", 9000, 320_000, 1.2, 3, 4096, 4, 2, 2, 50, 4, 32, "f32"),
        # scoring a Wikipedia-shaped batch: three roots per event, two heads of 50, a cache of 8 bits
        _attend("attend_batch_q8", 9000, 320_000, 1.2, 1800, 64, 2, 2, 2, 50, 8, 32, "f32"),
        # large batches, windows of twenty: many short rows
        _attend("attend_short_q4", 17_000, 4_000_000, 1.1, 14_400, 20, 1, 2, 2, 50, 4, 16, "f32"),
        # long windows in 16-bit arithmetic, eight query heads over two cached ones
        _attend("attend_long_q4", 17_000, 4_000_000, 0.7, 12_000, 512, 8, 8, 2, 64, 4, 32, "bf16"),
        # a training batch of the smallest configuration
        _slots("slots_tiny_f32", 600, 10, 2, 2, 16, 16, "f32"),
        # a training batch of the Wikipedia shape with a few more neighbors, heads of 50
        _slots("slots_wiki_f32", 1800, 20, 2, 2, 50, 32, "f32"),
        # large batches with replay events, wide windows, 16-bit rows
        _slots("slots_large_bf16", 14_400, 64, 4, 4, 32, 32, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "cache", "attend", "slots"])
    largest = max(work(c)["bytes"] for c in listed() if c["kind"] == kind)
    if kind == "sample":
        c = _sample("", _log(rng, 200, 20_000), _log(rng, 20_000, 2_600_000), rng.choice([0.7, 1.1, 1.5]),
                    _log(rng, 1, 12_000), _log(rng, 1, 100), rng.randint(0, 9))
    elif kind == "cache":
        rows = _log(rng, 100, 1_000_000)
        c = _cache("", rows + _log(rng, 10, 100_000), rows, rng.choice([1, 2, 3, 4, 8]), rng.choice([16, 25, 32, 43, 50, 64, 86, 100, 128]),
                   rng.choice([4, 8]), rng.choice(list(DTYPES)), rng.choice(list(DTYPES)))
    elif kind == "attend":
        kv = rng.choice([1, 2, 4])
        c = _attend("", _log(rng, 500, 20_000), _log(rng, 50_000, 4_000_000), rng.choice([0.7, 1.1, 1.5]), _log(rng, 1, 12_000),
                    _log(rng, 1, 4096), rng.randint(0, 16), kv * rng.choice([1, 2, 4, 8]), kv, rng.choice([16, 25, 32, 50, 64, 100, 128]),
                    rng.choice([4, 8]), rng.choice([1, 2, 16, 32, 64]), rng.choice(list(DTYPES)))
    else:
        kv = rng.choice([1, 2, 4])
        c = _slots("", _log(rng, 20, 15_000), _log(rng, 1, 200), kv * rng.choice([1, 1, 2, 4]), kv, rng.choice([16, 25, 32, 50, 64, 100, 128]),
                   rng.choice([2, 7, 16, 32, 64]), rng.choice(list(DTYPES)))
    many = "rows" if kind == "cache" else "roots"
    while work(c)["bytes"] > largest or (kind == "attend" and c["roots"] * (c["window"] + c["sinks"]) * c["heads"] * c["dim"] > 3.2e9):
        c[many] = max(1, c[many] * 2 // 3)
    del c["name"]
    return c


def _degrees(case):
    """Entries of every node's slice: Zipf over the nodes, `places` in all, each node one at least."""
    w = 1.0 / np.arange(1, case["nodes"] + 1) ** case["zipf"]
    cum = np.floor(np.cumsum(w / w.sum()) * (case["places"] - case["nodes"])).astype(np.int64)
    cum[-1] = case["places"] - case["nodes"]
    return np.diff(cum, prepend=0) + 1


def _seen(case):
    """Expected visible entries of all roots, and expected distinct ones among them (roots of one node see nearly the same)."""
    deg = _degrees(case)
    vis = np.minimum(deg, case["window"] + case["sinks"])
    p = _root_weights(case)
    return case["roots"] * float((p * vis).sum()), float(((1.0 - (1.0 - p) ** case["roots"]) * vis).sum())


def _root_weights(case):
    """Two of three roots are endpoints of events, the third a negative drawn over all nodes."""
    deg = _degrees(case)
    return (2.0 * deg / deg.sum() + 1.0 / len(deg)) / 3.0


def work(case):
    k = case["kind"]
    if k == "sample":
        slots = case["window"] + case["sinks"]
        read = case["roots"] * (4 + 8 + 16) + _seen(case)[1] * 16
        return {"bytes": read + case["roots"] * (slots * 16 + 4 + 8 + 4), "flops": case["roots"] * 32.0}
    if k == "cache":
        n, values = case["rows"], case["rows"] * case["heads"] * case["dim"]
        held = values * case["bits"] / 8 + n * (2 * case["heads"] + 8)
        return {"bytes": values * (SIZE[case["dtype"]] + SIZE[case["out"]]) + 2 * held + n * (16 + 16), "flops": values * 4.0}
    if k == "attend":
        seen, distinct = _seen(case)
        row = 2 * case["kv_heads"] * (case["dim"] * case["bits"] / 8 + 2) + 8
        io = case["roots"] * (2 * case["heads"] * case["dim"] * SIZE[case["dtype"]] + 20)
        return {"bytes": distinct * row + io, "flops": 4.0 * seen * case["heads"] * case["dim"]}
    values = case["roots"] * case["slots"] * case["kv_heads"] * case["dim"]
    rows = case["roots"] * case["heads"] * case["dim"]
    size, full = SIZE[case["dtype"]], 0.95                 # most roots have all their slots, some a part of them
    # forward reads k and v, backward reads them again (a training step lies between) and writes their gradients
    return {"bytes": values * size * (4 * full + 2) + rows * size * 5 + case["roots"] * (case["slots"] * 16 + 24),
            "flops": 14.0 * full * case["roots"] * case["slots"] * case["heads"] * case["dim"]}


# ------------------------------------------------------------------------------------------------ their inputs --
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _histories(case, g):
    """A T-CSR: slices in time order, neighbors and event ids, and a batch of roots near the end of the stream."""
    deg = torch.from_numpy(_degrees(case)).cuda()
    P, N = case["places"], case["nodes"]
    indptr = torch.zeros(N + 1, dtype=torch.int64, device="cuda")
    indptr[1:] = torch.cumsum(deg, 0)
    node_of = torch.repeat_interleave(torch.arange(N, device="cuda"), deg)
    order = torch.argsort(torch.rand(P, generator=g, device="cuda"))          # places in order of time
    by_node = torch.argsort(node_of[order], stable=True)
    eid = (by_node // 2).to(torch.int32)                                      # an event has two places
    ts = (eid.double() + 1.0) * (SPAN / (P // 2 + 1))
    nbr = torch.randint(0, N, (P,), generator=g, device="cuda", dtype=torch.int32)
    p = torch.from_numpy(_root_weights(case)).cuda()
    cum = torch.cumsum(p, 0)
    nodes = torch.searchsorted(cum, torch.rand(case["roots"], generator=g, device="cuda", dtype=torch.float64) * cum[-1])
    nodes = nodes.clamp_(max=N - 1).to(torch.int32)
    times = SPAN * (1.0 - 0.01 * torch.rand(case["roots"], generator=g, device="cuda", dtype=torch.float64))
    return dict(indptr=indptr, nbr=nbr, eid=eid, ts=ts, nodes=nodes, times=times)


def _bounds(n):
    """Bucket bounds: logarithmic over the time differences of a stream."""
    return torch.logspace(1.0, math.log10(SPAN), n - 1, dtype=torch.float64, device="cuda") if n > 1 else torch.empty(0, dtype=torch.float64, device="cuda")


def _rows(n, heads, dim, g, dtype=torch.float32):
    """Key, value or memory rows: normal, with heads and rows of different size, as projections and GRU states have."""
    x = torch.randn(n, heads, dim, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(n, 1, 1, generator=g, device="cuda"))
    return x.to(dtype)


def _visible(st):
    """Place of the first entry and number of entries with ts < time, by halving."""
    first = st["indptr"][st["nodes"].long()]
    lo, hi = first.clone(), st["indptr"][st["nodes"].long() + 1]
    for _ in range(32):
        mid = (lo + hi) // 2
        at = st["ts"][mid.clamp(max=st["ts"].numel() - 1)]
        below = (mid < hi) & (at < st["times"])
        lo, hi = torch.where(below, mid + 1, lo), torch.where(below | (lo >= hi), hi, mid)
    return first, (lo - first).to(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    k = case["kind"]
    if own:
        from paper_2608_16305_b200 import binding as B
        st["B"] = B
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if k == "sample":
        st.update(_histories(case, g))
        R, S = case["roots"], case["window"] + case["sinks"]
        if own:
            i32 = dict(dtype=torch.int32, device="cuda")
            st["out"] = (torch.empty((R, S), **i32), torch.empty((R, S), **i32),
                         torch.empty((R, S), dtype=torch.float64, device="cuda"), torch.empty(R, **i32),
                         torch.empty(R, dtype=torch.int64, device="cuda"), torch.empty(R, **i32))
    elif k == "cache":
        n, T = case["rows"], case["table"]
        st["table"] = _rows(T, case["heads"], case["dim"], g, DTYPES[case["dtype"]])
        st["times"] = SPAN * torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        st["from"] = torch.randperm(T, generator=g, device="cuda")[:n].contiguous()      # rows of the table, 64-bit indices
        st["to"] = torch.randperm(T, generator=g, device="cuda")[:n].contiguous()        # rows of the table that is written
        st["out"] = torch.zeros(T, case["heads"], case["dim"], dtype=DTYPES[case["out"]], device="cuda")
        st["out_times"] = torch.zeros(T, dtype=torch.float64, device="cuda")
        if own:
            st["cache"] = st["B"].RowCache(n, case["heads"], case["dim"], case["bits"])
    elif k == "attend":
        st.update(_histories(case, g))
        P, H, KV, D = case["places"], case["heads"], case["kv_heads"], case["dim"]
        st["first"], st["len"] = _visible(st)
        st["q"] = _rows(case["roots"], H, D, g, DTYPES[case["dtype"]])
        st["bounds"] = _bounds(case["buckets"])
        st["bias"] = 0.5 * torch.randn(H, case["buckets"], generator=g, device="cuda")
        for name in ("k", "v"):
            if own:
                st[name] = st["B"].RowCache(P, KV, D, case["bits"], times=False)
            else:
                st[name] = (torch.empty(P, KV, D, dtype=torch.int8, device="cuda"), torch.empty(P, KV, 1, device="cuda"))
            for p0 in range(0, P, 1 << 20):
                p1 = min(P, p0 + (1 << 20))
                rows = _rows(p1 - p0, KV, D, g)
                if own:
                    at = torch.arange(p0, p1, device="cuda")
                    st["B"].cache_write(st[name], rows, st["status"], dst=at)
                else:
                    st[name][0][p0:p1], st[name][1][p0:p1] = _quantise(rows, case["bits"])
        if own:
            st["o"] = torch.empty_like(st["q"])
    else:
        R, S, H, KV, D = (case[n] for n in ("roots", "slots", "heads", "kv_heads", "dim"))
        dt = DTYPES[case["dtype"]]
        st["q"], st["do"] = _rows(R, H, D, g, dt), _rows(R, H, D, g, dt)
        st["k"] = _rows(R * S, KV, D, g, dt).view(R, S, KV, D)
        st["v"] = _rows(R * S, KV, D, g, dt).view(R, S, KV, D)
        part = torch.randint(0, S + 1, (R,), generator=g, device="cuda")
        st["cnt"] = torch.where(torch.rand(R, generator=g, device="cuda") < 0.1, part, torch.full_like(part, S)).to(torch.int32)
        st["times"] = SPAN * (0.5 + 0.5 * torch.rand(R, generator=g, device="cuda", dtype=torch.float64))
        gaps = torch.exp(8.0 * torch.rand(R, S, generator=g, device="cuda", dtype=torch.float64))
        st["ts"] = st["times"][:, None] - torch.cumsum(gaps, 1)               # most recent first
        st["bounds"] = _bounds(case["buckets"])
        st["bias"] = 0.5 * torch.randn(H, case["buckets"], generator=g, device="cuda")
        if own:
            st["o"], st["dq"] = torch.empty_like(st["q"]), torch.empty_like(st["q"])
            st["dk"], st["dv"] = torch.empty_like(st["k"]), torch.empty_like(st["v"])
            st["dbias"] = torch.empty_like(st["bias"])
            st["scratch"] = torch.empty(st["B"].slot_attend_scratch(R, H, case["buckets"]), device="cuda")
    return st


# --------------------------------------------------------------------------------------------- the plain forms --
def _quantise(x, bits):
    """Codes (int8) and scales (fp32 that bf16 holds) of groups along the last axis."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    s = amax / (7.0 if bits == 4 else 127.0)
    s = ((s.view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32)        # up to the next bf16
    s = torch.where(amax < 2.0 ** -100, torch.zeros_like(s), s)
    r = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    return torch.round(x.double() * r.double()).to(torch.int8), s              # the product is exact in 64 bits


def _window_slots(case, first, length, newest_first):
    """Places of every root's window and sinks: [R, window + sinks] and how many of them count."""
    w, s = case["window"], case["sinks"]
    length = length.long()[:, None]
    j = torch.arange(w + s, device="cuda")[None, :]
    nw = length.clamp(max=w)
    ns = (length - nw).clamp(max=s)
    if newest_first:
        at = torch.where(j < nw, length - 1 - j, j - nw)
    else:
        at = torch.where(j < ns, j, length - nw + (j - ns))
    return first[:, None] + at, j < nw + ns


def _plain_sample(st):
    case = st["case"]
    first, length = _visible(st)
    at, ok = _window_slots(case, first, length, True)
    at = torch.where(ok, at, torch.zeros_like(at))
    none = torch.full_like(at, -1, dtype=torch.int32)
    return (torch.where(ok, st["nbr"][at], none), torch.where(ok, st["eid"][at], none),
            torch.where(ok, st["ts"][at], torch.zeros_like(st["ts"][:1])), ok.sum(1).to(torch.int32), first, length)


def _plain_cache(st):
    codes, s = _quantise(st["table"][st["from"]], st["case"]["bits"])
    st["out"][st["to"]] = (codes.float() * s).to(st["out"].dtype)
    st["out_times"][st["to"]] = st["times"][st["from"]]
    return st["out"], st["out_times"]


def _bucket(bounds, dt):
    """Bounds that are <= dt, counted by comparisons."""
    n = torch.zeros(dt.shape, dtype=torch.int64, device=dt.device)
    for i in range(bounds.numel()):
        n += bounds[i] <= dt
    return n


def _softmax(z):
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isfinite(m), m, torch.zeros_like(m)))
    l = e.sum(-1, keepdim=True)
    return e / torch.where(l > 0, l, torch.ones_like(l))


def _plain_attend(st):
    case = st["case"]
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.empty_like(st["q"])
    step = max(1, int(2e8 / ((case["window"] + case["sinks"]) * H * D)))
    for r0 in range(0, case["roots"], step):
        r = slice(r0, min(case["roots"], r0 + step))
        at, ok = _window_slots(case, st["first"][r], st["len"][r], False)
        at = torch.where(ok, at, st["first"][r][:, None])                      # a visible node has one place at least
        b = _bucket(st["bounds"], st["times"][r][:, None] - st["ts"][at])
        q = st["q"][r].float().view(-1, KV, H // KV, D)
        k = st["k"][0][at].float() * st["k"][1][at]
        z = torch.einsum("rkgd,rnkd->rkgn", q, k) / math.sqrt(D)
        z = z + st["bias"][:, b].view(KV, H // KV, *b.shape).permute(2, 0, 1, 3)
        z = torch.where(ok[:, None, None, :], z, torch.full_like(z, -math.inf))
        p = _softmax(z)
        v = st["v"][0][at].float() * st["v"][1][at]
        out[r] = torch.einsum("rkgn,rnkd->rkgd", p, v).reshape(-1, H, D).to(out.dtype)
    return out


def _plain_slots(st):
    case = st["case"]
    R, S, H, KV, D = (case[n] for n in ("roots", "slots", "heads", "kv_heads", "dim"))
    scale = 1.0 / math.sqrt(D)
    ok = torch.arange(S, device="cuda")[None, :] < st["cnt"][:, None]
    b = _bucket(st["bounds"], st["times"][:, None] - st["ts"])
    q, do = (st[n].float().view(R, KV, H // KV, D) for n in ("q", "do"))
    k, v = st["k"].float(), st["v"].float()
    z = torch.einsum("rkgd,rnkd->rkgn", q, k) * scale
    z = z + st["bias"][:, b].view(KV, H // KV, R, S).permute(2, 0, 1, 3)
    p = _softmax(torch.where(ok[:, None, None, :], z, torch.full_like(z, -math.inf)))
    o = torch.einsum("rkgn,rnkd->rkgd", p, v)
    dp = torch.einsum("rkgd,rnkd->rkgn", do, v)
    dz = p * (dp - (p * dp).sum(-1, keepdim=True))
    dv = torch.einsum("rkgn,rkgd->rnkd", p, do)
    dq = torch.einsum("rkgn,rnkd->rkgd", dz, k) * scale
    dk = torch.einsum("rkgn,rkgd->rnkd", dz, q) * scale
    by_head = dz.double().permute(1, 2, 0, 3).reshape(H, R * S)                # a long sum
    db = torch.zeros(H, case["buckets"], dtype=torch.float64, device="cuda")
    for i in range(case["buckets"]):
        db[:, i] = (by_head * (b.view(1, -1) == i)).sum(1)
    t = st["q"].dtype
    return o.reshape(R, H, D).to(t), dq.reshape(R, H, D).to(t), dk.to(t), dv.to(t), db.float()


# ------------------------------------------------------------------------------------------------- the passes --
def run(st):
    case = st["case"]
    k = case["kind"]
    if not own:
        return {"sample": _plain_sample, "cache": _plain_cache, "attend": _plain_attend, "slots": _plain_slots}[k](st)
    B = st["B"]
    if k == "sample":
        B.sample_window(st["indptr"], st["nbr"], st["eid"], st["ts"], st["nodes"], st["times"], case["window"], case["sinks"],
                        *st["out"], st["status"])
        return st["out"]
    if k == "cache":
        B.cache_write(st["cache"], st["table"], st["status"], src=st["from"], times=st["times"])
        B.cache_read(st["cache"], st["out"], st["status"], dst=st["to"], times=st["out_times"])
        return st["out"], st["out_times"]
    if k == "attend":
        B.cached_attend(st["q"], st["k"], st["v"], st["first"], st["len"], case["window"], case["sinks"], st["o"], st["status"],
                        bias=st["bias"], bounds=st["bounds"], times=st["times"], ts=st["ts"])
        return st["o"]
    B.slot_attend(st["q"], st["k"], st["v"], st["cnt"], st["o"], bias=st["bias"], bounds=st["bounds"], times=st["times"], ts=st["ts"])
    B.slot_attend_backward(st["q"], st["k"], st["v"], st["cnt"], st["do"], st["dq"], st["dk"], st["dv"], bias=st["bias"],
                           bounds=st["bounds"], times=st["times"], ts=st["ts"], dbias=st["dbias"], scratch=st["scratch"])
    return st["o"], st["dq"], st["dk"], st["dv"], st["dbias"]


# --------------------------------------------------------------------------------- the definitions in 64 bits --
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"sample": _exact_sample, "cache": _exact_cache, "attend": _exact_attend, "slots": _exact_slots}[case["kind"]](st)


def _exact_sample(st):
    """One root after another on the host."""
    case = st["case"]
    ptr, nbr, eid, ts, nodes, times = (st[n].cpu().numpy() for n in ("indptr", "nbr", "eid", "ts", "nodes", "times"))
    R, w, s = case["roots"], case["window"], case["sinks"]
    o_n, o_e = np.full((R, w + s), -1, np.int32), np.full((R, w + s), -1, np.int32)
    o_t, cnt, length = np.zeros((R, w + s)), np.zeros(R, np.int32), np.zeros(R, np.int32)
    first = ptr[nodes]
    for i in range(R):
        a = ptr[nodes[i]]
        L = int(np.searchsorted(ts[a:ptr[nodes[i] + 1]], times[i], side="left"))
        recent = list(range(L - 1, max(L - w, 0) - 1, -1))
        at = a + np.array(recent + list(range(min(s, L - len(recent)))), np.int64)
        length[i], cnt[i] = L, len(at)
        o_n[i, :len(at)], o_e[i, :len(at)], o_t[i, :len(at)] = nbr[at], eid[at], ts[at]
    return tuple(torch.from_numpy(a) for a in (o_n, o_e, o_t, cnt, first, length))


def _exact_cache(st):
    """The quantiser's definition: its two fp32 quotients are part of it, the rest is exact in 64 bits."""
    case = st["case"]
    x = st["table"].index_select(0, st["from"]).double()
    top = torch.maximum(x.amax(-1), -x.amin(-1))
    s = torch.div(top.float(), 7 if case["bits"] == 4 else 127).double()
    mantissa, exponent = torch.frexp(s)
    s = torch.ldexp(torch.ceil(mantissa * 256.0), exponent - 8)                # eight bits, rounded up
    r = torch.reciprocal(s.float()).double()
    y = torch.special.round(x * r[..., None]) * s[..., None]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    times = torch.zeros_like(st["out_times"])
    out.index_copy_(0, st["to"], y)
    times.index_copy_(0, st["to"], st["times"].index_select(0, st["from"]))
    return out, times


def _exact_attend(st):
    """Root after root where they are few, in slabs of one head otherwise; sums and exponentials in 64 bits."""
    case = st["case"]
    H, KV, D, w, s = (case[n] for n in ("heads", "kv_heads", "dim", "window", "sinks"))
    if case["roots"] * (w + s) * H * D > 4e9:
        return None
    out = torch.zeros(case["roots"], H, D, dtype=torch.float64, device="cuda")
    kv_of = torch.arange(H, device="cuda") // (H // KV)
    slab = max(1, int(6e7 / ((w + s) * D)))
    j = torch.arange(w + s, device="cuda")
    for r0 in range(0, case["roots"], slab):
        r = torch.arange(r0, min(case["roots"], r0 + slab), device="cuda")
        L = st["len"][r].long()
        lo = (L - w).clamp(min=0)
        entry = torch.where(j[None] < w, lo[:, None] + j[None], (j[None] - w).expand(len(r), -1))
        seen = torch.where(j[None] < w, entry < L[:, None], entry < lo[:, None])
        at = (st["first"][r][:, None] + entry)[seen]                           # visible pairs only, one after another
        row = r[:, None].expand_as(entry)[seen]
        bucket = torch.searchsorted(st["bounds"], st["times"][row] - st["ts"][at], right=True)
        for h in range(H):
            k = st["k"][0][at, kv_of[h]].double() * st["k"][1][at, kv_of[h]].double()
            z = (st["q"][row, h].double() * k).sum(1) / math.sqrt(D) + st["bias"][h, bucket].double()
            top = torch.full((len(r),), -math.inf, dtype=torch.float64, device="cuda").scatter_reduce(0, row - r0, z, "amax")
            e = torch.exp(z - top[row - r0])
            v = st["v"][0][at, kv_of[h]].double() * st["v"][1][at, kv_of[h]].double()
            num = torch.zeros(len(r), D, dtype=torch.float64, device="cuda").index_add_(0, row - r0, e[:, None] * v)
            den = torch.zeros(len(r), dtype=torch.float64, device="cuda").index_add_(0, row - r0, e)
            out[r, h] = num / torch.where(den > 0, den, torch.ones_like(den))[:, None]
    return out


def _exact_slots(st):
    """Gradients by the library's differentiation of the forward formula in 64 bits, head by head."""
    case = st["case"]
    R, S, H, KV, D = (case[n] for n in ("roots", "slots", "heads", "kv_heads", "dim"))
    q, k, v, bias = (st[n].double().requires_grad_() for n in ("q", "k", "v", "bias"))
    bucket = torch.searchsorted(st["bounds"], st["times"][:, None] - st["ts"], right=True)
    hidden = torch.arange(S, device="cuda")[None] >= st["cnt"][:, None].long()
    outs = []
    for h in range(H):
        z = (q[:, None, h] * k[:, :, h // (H // KV)]).sum(-1) / math.sqrt(D) + bias[h][bucket]
        z = z.masked_fill(hidden, -1e300)
        e = torch.exp(z - z.amax(1, keepdim=True).detach()).masked_fill(hidden, 0.0)
        p = e / e.sum(1, keepdim=True).clamp(min=1e-300)
        outs.append((p[:, :, None] * v[:, :, h // (H // KV)]).sum(1))
    o = torch.stack(outs, 1)
    dq, dk, dv, db = torch.autograd.grad(o, (q, k, v, bias), st["do"].double())
    return o.detach(), dq, dk, dv, db
