"""A learned table of nodes: rows looked up, every root's next destination scored among all nodes, and the optimizer of both.

The link head scores an event against one sampled negative; here a root answers with a distribution over all nodes, whose rows are
learned, and the same table gives the rows of neighbor slots.  All under autograd, without a row of logits in memory.

    lookup(table, ids)                 tgnn_lookup, its gradient by tgnn_lookup_backward
    destination_loss(q, table, target) tgnn_destination_loss, its gradients by tgnn_destination_loss_backward
    AdamW(params, ...)                 tgnn_adamw_step: all tensors in one launch, moments in 32 or 8 bits

All arithmetic happens inside the library.
"""
from __future__ import annotations

import ctypes as C
from typing import List, Optional, Sequence, Tuple, Union

import torch

from . import binding as B


class _Lookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale, dtype, status):
        table, ids = table.contiguous(), ids.contiguous()
        out = torch.empty((*ids.shape, table.shape[1]), dtype=dtype, device=table.device)
        status = torch.zeros(1, dtype=torch.int32, device=table.device) if status is None else status
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
    status: int32 [1], set to 4 where an id is beyond the table (such a row is zeros, too)."""
    return _Lookup.apply(table, ids, float(scale), table.dtype if dtype is None else dtype, status)


class _DestinationLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, table, bias, target, scale, status):
        q, table, target = q.contiguous(), table.contiguous(), target.contiguous()
        bias = None if bias is None else bias.contiguous()
        (n, dim), rows, dev = q.shape, table.shape[0], q.device
        loss = torch.empty(n, device=dev)
        wanted = any(ctx.needs_input_grad[:3])
        kept = torch.empty(B.destination_loss_kept(n, dim), device=dev) if wanted else None
        scratch = torch.empty(B.destination_loss_scratch(n, rows, dim, q.dtype), dtype=torch.uint8, device=dev)
        status = torch.zeros(1, dtype=torch.int32, device=dev) if status is None else status
        B.destination_loss(q, table, target, loss, scratch, status, bias=bias, kept=kept, scale=scale)
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
        return dq, dtable, dbias, None, None, None


def destination_loss(q: torch.Tensor, table: torch.Tensor, target: torch.Tensor, bias: Optional[torch.Tensor] = None,
                     scale: Optional[float] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Cross entropy [n] (fp32) of target [n] among all rows of table [rows, dim] for q [n, dim]: logits scale * q . row + bias, scale 1 / sqrt(dim) by
    default.  A target below 0 takes no part: loss 0, no gradient.  Differentiable in q, table and bias; fp32 or bf16 rows, bias fp32.
    status: int32 [1], set to 4 where a target is beyond the table (which takes no part either)."""
    return _DestinationLoss.apply(q, table, bias, target, scale, status)


class AdamW:
    """AdamW over all of `params` (fp32 CUDA tensors, contiguous, on one device) in one launch, moments in 32 or 8 bits.

    m, v        the moments, a list each: fp32, or int8 / uint8 codes with m_scale, v_scale (one fp32 per 256 values)
    steps       int64 [2]; the first is the number of steps taken (set it when moments are loaded)
    copies      16-bit tensors (or None) that the new parameters are written to as well, e.g. the table that a bf16 loss reads
    weight_decay  one number, or one per tensor
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
        self._values = None

    def step(self, grads: Optional[Sequence[Optional[torch.Tensor]]] = None, grad_scale: float = 1.0) -> None:
        """One step on the gradients given, or on the parameters' own (.grad); a tensor without one stays as it is.  Gradients are multiplied
        by grad_scale (1 / workers for a mean, or a clipping factor)."""
        grads = [p.grad for p in self.params] if grads is None else grads if type(grads) is list else list(grads)
        B.adamw_step(self._t, self.bits, self.device.index, self.steps, self.params, grads, self.lr, self.betas[0], self.betas[1], self.eps,
                     grad_scale, self.seed)

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
