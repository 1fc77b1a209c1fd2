"""A learned table of nodes: rows looked up, every root's next destination scored among all nodes, and the optimizer of both.

The link head scores an event against one sampled negative; here a root answers with a distribution over all nodes, whose rows are
learned, and the same table gives the rows of neighbor slots.  All under autograd, without a row of logits in memory.

    status()                           what calls of the two below without a status tensor have met on the device
    lookup(table, ids)                 tgnn_lookup, its gradient by tgnn_lookup_backward
    destination_loss(q, table, target) tgnn_destination_loss, its gradients by tgnn_destination_loss_backward
    AdamW(params, ...)                 tgnn_adamw_step: all tensors in one launch, moments in 32 or 8 bits
    DestinationModel(workload, ...)    all three over a workload's batches, with the attention over sampled slots between them

All arithmetic happens inside the library, but the sum of a root's own row and what it attends to, and autograd's sums of the table's three gradients (roots, slots,
answers; in the table's type, so that a bf16 table's are rounded twice more).
"""
from __future__ import annotations

import ctypes as C
from typing import Dict, List, Optional, Sequence, Tuple, Union

import torch

from . import binding as B
from .history import Slots, TimeBias, slot_attention


_flags: Dict[int, torch.Tensor] = {}


def _flag(device: torch.device) -> torch.Tensor:
    """Where calls without a status of their own record what goes wrong on the device.  (A call that is captured before any other has come is given one that
    lives in its graph, and that nobody reads.)"""
    flag = _flags.get(device.index)
    if flag is None:
        with torch.inference_mode(False):
            flag = torch.zeros(1, dtype=torch.int32, device=device)
        if device.type == "cuda" and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(device).synchronize()      # it is zero before a call on any stream gets it
            _flags[device.index] = flag
    return flag


def status(device: Union[torch.device, int, None] = None, clear: bool = False) -> int:
    """0, or what lookups and destination losses without a status of their own have met on the device (the current one by default) since it was last cleared: 4
    for an id or a target beyond its table (which counts as none), TGNN_ETIMEOUT where results are worthless.  Reads the device."""
    index = torch.cuda.current_device() if device is None else device if isinstance(device, int) else torch.device(device).index
    flag = _flags.get(torch.cuda.current_device() if index is None else index)
    code = 0 if flag is None else int(flag.item())
    if clear and code:
        flag.zero_()
    return code


class _Lookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale, dtype, status):
        table, ids = table.contiguous(), ids.contiguous()
        out = torch.empty((*ids.shape, table.shape[1]), dtype=dtype, device=table.device)
        status = _flag(table.device) if status is None else status
        B.lookup(table, ids, out, status, scale=scale)
        ctx.save_for_backward(ids)
        ctx.like, ctx.scale, ctx.status = (table.shape, table.dtype), scale, status
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        (ids,) = ctx.saved_tensors
        shape, dtype = ctx.like
        dtable = torch.empty(shape, dtype=dtype, device=dout.device)
        scratch = torch.empty(B.lookup_scratch(ids.numel(), shape[0], shape[1]), dtype=torch.uint8, device=dout.device)
        B.lookup_backward(ids, dout.contiguous(), dtable, scratch, ctx.status, scale=ctx.scale)
        return dtable, None, None, None, None


def lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
           status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[ids] as [*ids.shape, dim] of `dtype` (the table's own by default), zeros where an id is below 0; differentiable in the table.
    status: int32 [1], set to 4 where an id is beyond the table (such a row is zeros, too); without one, status() tells."""
    return _Lookup.apply(table, ids, float(scale), table.dtype if dtype is None else dtype, status)


class _DestinationLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, table, bias, target, scale, status, wanted):
        q, table, target = q.contiguous(), table.contiguous(), target.contiguous()
        bias = None if bias is None else bias.contiguous()
        (n, dim), rows, dev = q.shape, table.shape[0], q.device
        loss = torch.empty(n, device=dev)
        kept = torch.empty(B.destination_loss_kept(n, dim), device=dev) if wanted else None
        scratch = torch.empty(B.destination_loss_scratch(n, rows, dim, q.dtype), dtype=torch.uint8, device=dev)
        status = _flag(dev) if status is None else status
        B.destination_loss(q, table, target, loss, scratch, status, bias=bias, kept=kept, scale=scale)
        if wanted:
            ctx.save_for_backward(q, table, bias, target, kept)
        ctx.scale, ctx.status = scale, status
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        q, table, bias, target, kept = ctx.saved_tensors
        like = lambda x, i: torch.empty_like(x) if x is not None and ctx.needs_input_grad[i] else None
        dq, dtable, dbias = like(q, 0), like(table, 1), like(bias, 2)
        scratch = torch.empty(B.destination_loss_scratch(q.shape[0], table.shape[0], q.shape[1], q.dtype), dtype=torch.uint8, device=q.device)
        B.destination_loss_backward(q, table, target, kept, dloss.contiguous(), dq, dtable, scratch, ctx.status, bias=bias, dbias=dbias,
                                    scale=ctx.scale)
        return dq, dtable, dbias, None, None, None, None


def destination_loss(q: torch.Tensor, table: torch.Tensor, target: torch.Tensor, bias: Optional[torch.Tensor] = None,
                     scale: Optional[float] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Cross entropy [n] (fp32) of target [n] among all rows of table [rows, dim] for q [n, dim]: logits scale * q . row + bias, scale 1 / sqrt(dim) by
    default.  A target below 0 takes no part: loss 0, no gradient.  Differentiable in q, table and bias; fp32 or bf16 rows, bias fp32.  Where no gradient
    can be asked for (torch.no_grad(), no leaf that wants one) the loss alone is computed, and nothing kept.
    status: int32 [1], set to 4 where a target is beyond the table (which takes no part either); without one, status() tells."""
    # asked here: inside a Function the grad mode is off, and needs_input_grad does not go by it
    wanted = torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in (q, table, bias))
    return _DestinationLoss.apply(q, table, bias, target, scale, status, wanted)


class AdamW:
    """AdamW over all of `params` (fp32 CUDA tensors, contiguous, on one device) in one launch, moments in 32 or 8 bits.

    m, v        the moments, a list each: fp32, or int8 / uint8 codes with m_scale, v_scale (one fp32 per 256 values); saved moments are copied into them
    steps       int64 [2]; the first is the number of steps taken (set it when moments are loaded)
    copies      16-bit tensors (or None) that the new parameters are written to as well, e.g. the table that a bf16 loss reads
    weight_decay  one number, or one per tensor
    Betas are rounded to fp32; eps is 0 or a normal number of fp32; no two of parameters and copies may overlap.
    A step captured into a graph keeps lr and the addresses of parameters and gradients."""

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.0, bits: int = 32, seed: int = 0,
                 copies: Optional[Sequence[Optional[torch.Tensor]]] = None):
        self.params: List[torch.Tensor] = list(params)
        if bits not in (8, 32):
            raise B.TgnnError(B.TGNN_EINVAL, f"AdamW: moments in {bits} bits (8 or 32)")
        for p in self.params:
            if not p.is_cuda or p.dtype != torch.float32 or not p.is_contiguous() or p.device != self.params[0].device:
                raise TypeError(f"AdamW: expected contiguous fp32 tensors on one CUDA device, got {p.dtype} on {p.device}")
        decay = [float(weight_decay)] * len(self.params) if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        self.copies = [None] * len(self.params) if copies is None else list(copies)
        if len(decay) != len(self.params) or len(self.copies) != len(self.params):
            raise TypeError("AdamW: expected one weight decay and one copy (or None) per parameter")
        self.lr, self.betas, self.eps, self.bits, self.seed = float(lr), (float(betas[0]), float(betas[1])), float(eps), bits, int(seed)
        self.device = self.params[0].device if self.params else torch.device("cuda", torch.cuda.current_device())
        dev = self.device
        self.steps = torch.zeros(2, dtype=torch.int64, device=dev)
        zeros = lambda p, dt: torch.zeros(p.numel(), dtype=dt, device=dev)
        scales = lambda: [torch.zeros(B.adamw_blocks(p.numel()), device=dev) for p in self.params] if bits == 8 else None
        self.m = [zeros(p, torch.int8 if bits == 8 else torch.float32) for p in self.params]
        self.v = [zeros(p, torch.uint8 if bits == 8 else torch.float32) for p in self.params]
        self.m_scale, self.v_scale = scales(), scales()
        self._t = (B.TgnnAdamwTensor * len(self.params))()
        for i, p in enumerate(self.params):
            c = self.copies[i]
            if c is not None and (c.device != dev or c.dtype not in (torch.bfloat16, torch.float16) or c.numel() != p.numel() or not c.is_contiguous()):
                raise TypeError(f"AdamW: copy {i}: expected a contiguous 16-bit tensor of {p.numel()} elements on {dev}")
            self._t[i] = B.TgnnAdamwTensor(None, None, self.m[i].data_ptr(), self.v[i].data_ptr(),
                                           self.m_scale[i].data_ptr() if bits == 8 else None, self.v_scale[i].data_ptr() if bits == 8 else None,
                                           None if c is None else c.data_ptr(), p.numel(), decay[i], 0,
                                           B.TGNN_F16 if c is not None and c.dtype == torch.float16 else B.TGNN_BF16, 0)
        # a thread block may be at any place of any tensor when another one writes
        spans = sorted((x.data_ptr(), x.data_ptr() + x.numel() * x.element_size()) for x in self.params + self.copies if x is not None and x.numel() > 0)
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("AdamW: a tensor is given twice, or parameters or copies overlap")
        self._all = self._written(self.params)
        self._values = None

    def _written(self, grads) -> List[torch.Tensor]:
        return [x for p, c, g in zip(self.params, self.copies, grads) if g is not None for x in (p, c) if x is not None]

    def step(self, grads: Optional[Sequence[Optional[torch.Tensor]]] = None, grad_scale: float = 1.0) -> None:
        """One step on the gradients given, or on the parameters' own (.grad); a tensor without one stays as it is.  Gradients are multiplied
        by grad_scale (1 / workers for a mean, or a clipping factor)."""
        grads = [p.grad for p in self.params] if grads is None else grads if type(grads) is list else list(grads)
        B.adamw_step(self._t, self.bits, self.device.index, self.steps, self.params, grads, self.lr, self.betas[0], self.betas[1], self.eps,
                     grad_scale, self.seed)
        # written by address: autograd is told, so that a backward pass over a graph from before the step is an error and not one over the new values
        torch.autograd.graph.increment_version(self._written(grads) if type(None) in map(type, grads) else self._all)

    def moments(self) -> Tuple[List[torch.Tensor], List[torch.Tensor]]:
        """First and second moments as fp32 values: the state itself in 32 bits, else tensors that the next call overwrites."""
        if self.bits == 32:
            return self.m, self.v
        if self._values is None:
            m, v = ([torch.empty(p.numel(), device=self.device) for p in self.params] for _ in range(2))
            at = lambda x: (C.c_void_p * max(1, len(x)))(*(t.data_ptr() or None for t in x))
            self._values = (m, v, at(m), at(v))
        m, v, pm, pv = self._values
        B.adamw_moments(self._t, self.device.index, pm, pv)
        return m, v


class DestinationModel:
    """Which node a source meets next, from a learned table alone: a root's row plus attention from it over the rows of its last neighbors
    (with a learned bias by age) is scored against every node's row.

    workload    a DeviceWorkload (its events, T-CSR and batches); a batch's target events are roots at their sources and times
    dtype       of the rows that are looked up and scored: fp32, or bf16 beside fp32 weights
    heads, dim  of the attention; a row has heads * dim values, 256 at most (default: the workload's d over its heads)
    window      the last entries of its source that a root sees
    bits        of the optimizer's moments, 32 or 8"""

    def __init__(self, workload, heads: Optional[int] = None, dim: Optional[int] = None, window: Optional[int] = None, buckets: int = 16,
                 dtype: torch.dtype = torch.float32, lr: float = 1e-3, weight_decay: float = 0.0, bits: int = 32, seed: int = 0):
        cfg, dev = workload.cfg, workload.device
        self.workload = workload
        self.heads = cfg.heads if heads is None else int(heads)
        self.dim = cfg.d // self.heads if dim is None else int(dim)
        self.window = cfg.k if window is None else int(window)
        if dtype not in (torch.float32, torch.bfloat16) or not 1 <= self.heads * self.dim <= 256:
            raise B.TgnnError(B.TGNN_EINVAL, f"DestinationModel: rows of {self.heads * self.dim} values of {dtype} (fp32 or bf16, 1 to 256)")
        wide = self.heads * self.dim
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.weights = torch.randn((cfg.num_nodes, wide), generator=gen, device=dev) * wide ** -0.25
        self.table = self.weights if dtype == torch.float32 else self.weights.to(dtype)
        self.bias = torch.zeros(cfg.num_nodes, device=dev)
        self.age = TimeBias.logarithmic(self.heads, buckets, 1.0, 1e6, device=dev)
        self.leaves = [x.requires_grad_() for x in (self.table, self.bias, self.age.table)]
        self.optimizer = AdamW([self.weights.detach(), self.bias.detach(), self.age.table.detach()], lr=lr, weight_decay=[weight_decay, 0.0, 0.0],
                               bits=bits, seed=seed, copies=None if dtype == torch.float32 else [self.table.detach(), None, None])
        self._status = torch.zeros(1, dtype=torch.int32, device=dev)

    def status(self) -> int:
        """0, or the first error that a call met on the device (4: an index outside its table); reads the device."""
        return int(self._status.item())

    def slots(self, nodes: torch.Tensor, times: torch.Tensor) -> Slots:
        w, n, dev = self.workload, nodes.numel(), nodes.device
        out = Slots(*(torch.empty((n, self.window), dtype=t, device=dev) for t in (torch.int32, torch.int32, torch.float64)),
                    torch.empty(n, dtype=torch.int32, device=dev))
        B.sample_window(w.indptr, w.nbr, w.eid, w.ts, nodes, times, self.window, 0, *out, None, None, self._status)
        return out

    def loss(self, nodes: torch.Tensor, times: torch.Tensor, destinations: torch.Tensor) -> torch.Tensor:
        """Cross entropy [n] of each root's destination among all nodes (below 0: a root that takes no part); differentiable in `leaves`, and with
        nothing kept under torch.no_grad()."""
        s = self.slots(nodes, times)
        shape = (self.heads, self.dim)
        own = lookup(self.table, nodes, status=self._status)
        rows = lookup(self.table, s.nbr, status=self._status).view(*s.nbr.shape, *shape)
        seen = slot_attention(own.view(nodes.numel(), *shape), rows, rows, s.cnt, bias=self.age, times=times, ts=s.ts)
        return destination_loss(own + seen.view_as(own), self.table, destinations, bias=self.bias, status=self._status)

    def targets(self, b: int) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """Sources, times and destinations of batch b; destinations of events that only come along (a workload with embed_aux) are -1."""
        src, dst, _, t = self.workload.targets(b)
        mask = self.workload.loss_mask(b)
        return src, t, dst if mask is None else torch.where(mask != 0, dst, -1)

    def step(self, b: int) -> torch.Tensor:
        """One training step on batch b; its losses, one per event."""
        loss = self.loss(*self.targets(b))
        grads = torch.autograd.grad(loss, self.leaves, grad_outputs=torch.ones_like(loss))
        self.optimizer.step(list(grads), grad_scale=1.0 / max(1, loss.numel()))
        return loss.detach()
