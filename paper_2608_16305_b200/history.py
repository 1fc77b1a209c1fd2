"""Temporal attention over the histories of an event stream's nodes, for training and for scoring.

With a learned bias by buckets of the time difference in place of an encoding inside the keys, an entry's key and value depend on the
entry alone.  `EventHistory` keeps them, in 4 or 8 bits, at the entry's place in the T-CSR: they are written when the event arrives
and read by every later root, which sees the last `window` entries of its node and the first `sinks` of the rest.  For training
it hands out the same slots as arrays, over which `slot_attention` runs with gradients.

    append(places, k, v)           tgnn_cache_write: keys and values of a batch's entries (two per event)
    attend(q, nodes, times, ...)   tgnn_sample_window -> tgnn_cached_attend
    slots(nodes, times)            tgnn_sample_window: neighbors, events and times of every root's slots
    slot_attention(...)            tgnn_slot_attend, and its gradients by tgnn_slot_attend_backward

All arithmetic happens inside the library.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import torch

from . import binding as B


class TimeBias(NamedTuple):
    """A learned bias per head and bucket of the time difference: table fp32 [heads, buckets], bounds fp64 [buckets - 1] ascending
    (bucket of dt = number of bounds <= dt)."""
    table: torch.Tensor
    bounds: torch.Tensor

    @classmethod
    def logarithmic(cls, heads: int, buckets: int, nearest: float, farthest: float, device="cuda") -> "TimeBias":
        """Zeros, with bounds that grow by a constant factor from `nearest` to `farthest`."""
        n = buckets - 1
        b = [nearest] if n == 1 else [nearest * (farthest / nearest) ** (i / (n - 1)) for i in range(n)] if n else []
        return cls(torch.zeros((heads, buckets), device=device), torch.tensor(b, dtype=torch.float64, device=device))


class Slots(NamedTuple):
    """Slots of a batch of roots, [n, window + sinks] each: the window, most recent first, then the sinks; -1 / 0 behind cnt."""
    nbr: torch.Tensor
    eid: torch.Tensor
    ts: torch.Tensor
    cnt: torch.Tensor


class EventHistory:
    """Quantised keys and values of every entry of a T-CSR (indptr, nbr, eid, ts: device tensors, which stay as they are while it is used)."""

    def __init__(self, indptr, nbr, eid, ts, kv_heads: int, dim: int, window: int, sinks: int = 0, bits: int = 4):
        self.indptr, self.nbr, self.eid, self.ts = indptr, nbr, eid, ts
        self.window, self.sinks = int(window), int(sinks)
        self.k = B.RowCache(ts.numel(), kv_heads, dim, bits, times=False, device=ts.device)
        self.v = B.RowCache(ts.numel(), kv_heads, dim, bits, times=False, device=ts.device)
        self._status = torch.zeros(1, dtype=torch.int32, device=ts.device)
        self._places: Optional[torch.Tensor] = None

    def status(self) -> int:
        """4 if any call so far met an index outside its table, else 0 (reads the device)."""
        return int(self._status.item())

    def places(self, first_event: int, last_event: int) -> torch.Tensor:
        """Places of the entries of events [first_event, last_event), two per event, event by event; events outside the T-CSR have none.
        The T-CSR has to number its events one after the other, from any number on, with two entries each: ValueError otherwise
        (looked at on the first call, which reads the device)."""
        if self._places is None:                       # a stream's entries, ordered by event once
            order = torch.argsort(self.eid, stable=True)
            ids = self.eid[order]
            base = int(ids[0]) if ids.numel() else 0
            want = torch.arange(ids.numel() // 2, dtype=ids.dtype, device=ids.device) + base
            if not torch.equal(ids, want.repeat_interleave(2)):
                raise ValueError("the T-CSR's events are not numbered one after the other with two entries each")
            self._first_event, self._places = base, order
        a = max(0, first_event - self._first_event)
        return self._places[2 * a:2 * max(a, last_event - self._first_event)]

    def append(self, places: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> None:
        """Keys and values [n, kv_heads, dim] of the entries at `places` (distinct), quantised as they are written."""
        B.cache_write(self.k, k, self._status, dst=places)
        B.cache_write(self.v, v, self._status, dst=places)

    def attend(self, q: torch.Tensor, nodes: torch.Tensor, times: torch.Tensor, bias: Optional[TimeBias] = None,
               out: Optional[torch.Tensor] = None, scale: Optional[float] = None) -> torch.Tensor:
        """Attention of q [n, heads, dim] over what roots (node, time) see of their histories; zeros where that is nothing."""
        n = nodes.numel()
        first = torch.empty(n, dtype=torch.int64, device=nodes.device)
        length = torch.empty(n, dtype=torch.int32, device=nodes.device)
        B.sample_window(self.indptr, None, None, self.ts, nodes, times, self.window, self.sinks, None, None, None, None, first, length,
                        self._status)
        out = torch.empty_like(q) if out is None else out
        kw = {} if bias is None else dict(bias=bias.table, bounds=bias.bounds, times=times, ts=self.ts)
        B.cached_attend(q, self.k, self.v, first, length, self.window, self.sinks, out, self._status, scale=scale, **kw)
        return out

    def slots(self, nodes: torch.Tensor, times: torch.Tensor) -> Slots:
        """The same entries as arrays, for a training step that forms keys and values per slot."""
        n, s = nodes.numel(), self.window + self.sinks
        dev = nodes.device
        out = Slots(torch.empty((n, s), dtype=torch.int32, device=dev), torch.empty((n, s), dtype=torch.int32, device=dev),
                    torch.empty((n, s), dtype=torch.float64, device=dev), torch.empty(n, dtype=torch.int32, device=dev))
        B.sample_window(self.indptr, self.nbr, self.eid, self.ts, nodes, times, self.window, self.sinks, *out, None, None, self._status)
        return out


class _SlotAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, table, bounds, times, ts, cnt, scale):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        out = torch.empty_like(q)
        kw = {} if table is None else dict(bias=table, bounds=bounds, times=times, ts=ts)
        B.slot_attend(q, k, v, cnt, out, scale=scale, **kw)
        ctx.save_for_backward(q, k, v, table, bounds, times, ts, cnt)
        ctx.scale = scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, table, bounds, times, ts, cnt = ctx.saved_tensors
        dq, dk, dv, dbias = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), None
        kw = {}
        if table is not None:
            dbias = torch.empty_like(table)
            scratch = torch.empty(B.slot_attend_scratch(q.shape[0], q.shape[1], table.shape[1]), device=q.device)
            kw = dict(bias=table, bounds=bounds, times=times, ts=ts, dbias=dbias, scratch=scratch)
        B.slot_attend_backward(q, k, v, cnt, dout.contiguous(), dq, dk, dv, scale=ctx.scale, **kw)
        return dq, dk, dv, dbias, None, None, None, None, None


def slot_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cnt: torch.Tensor, bias: Optional[TimeBias] = None,
                   times: Optional[torch.Tensor] = None, ts: Optional[torch.Tensor] = None, scale: Optional[float] = None) -> torch.Tensor:
    """Attention of q [n, heads, dim] over the first cnt of k, v [n, slots, kv_heads, dim], differentiable in q, k, v and the bias's
    table; times [n] and ts [n, slots] are the roots' and the slots' times."""
    table, bounds = (None, None) if bias is None else (bias.table, bias.bounds)
    scale = 1.0 / math.sqrt(q.shape[-1]) if scale is None else scale
    return _SlotAttention.apply(q, k, v, table, bounds, times, ts, cnt, scale)
