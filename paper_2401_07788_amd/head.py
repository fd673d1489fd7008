"""The loss of a model's last stage: softmax cross entropy of x w^T over a
large vocabulary, and its gradients.  Argument marshalling only: the arithmetic
is in the HIP kernels of libtc.so (include/tc.h), and there is no fallback.

linear_xent_step(x, w, target, weight) is the whole of it for a stage that
knows its tokens' weights beforehand (1 / count for a mean): losses and
gradients from one call, dx ready for the boundary's compressor.
linear_xent(x, w, target) gives the losses alone; where gradients are
wanted through autograd, its backward pass is that one call, both gradients
and the logits' product again (4096 tokens, 50257 entries, h 768 in bfloat16:
1.33 ms there and back, the step 1.03 ms).

Memory.  The losses alone hold no tensor of n * v elements.  A step holds
softmax numerators for `chunk` tokens: 2 bytes an entry (binary32: 8), up to
4 GiB of them unless the caller says otherwise, and more than one chunk costs
time (the sizes above: 2048 tokens at once 1.28 ms, 512 2.6 ms).  The
workspace of a stream is kept between calls until free_workspaces().

Precision.  Products and sums are binary32.  The operands of the gradients'
products have the significand of x and w: d = weight (softmax - target) is
rounded to their type (binary32: 22 bits, as x and w are, relative to the
largest of its matrix), after its numerators were held with 9 bits behind the
point in bfloat16 and 11 in binary16 where a chunk has more than 64 tokens.
include/tc.h has the ranges."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import tc


class XentStep(NamedTuple):
    """losses and log-sum-exps (float32 [n]) and the gradients of x and w"""
    loss: torch.Tensor
    lse: torch.Tensor
    dx: torch.Tensor
    dw: torch.Tensor


def _rows(t: torch.Tensor, what: str) -> int:
    """elements from one row to the next of a matrix whose rows are contiguous"""
    if t.dim() != 2:
        raise ValueError(f"{what} must be a matrix")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{what} needs contiguous rows")
    if t.shape[0] <= 1:
        return t.shape[1]
    if t.stride(0) < t.shape[1]:
        raise ValueError(f"{what}: rows overlap")
    return t.stride(0)


def _sizes(x, w, target, ignore_index, chunk):
    ldx, ldw = _rows(x, "x"), _rows(w, "w")
    if x.shape[1] != w.shape[1]:
        raise ValueError(f"x has rows of {x.shape[1]}, w of {w.shape[1]}")
    if x.dtype != w.dtype:
        raise TypeError("x and w must share a dtype")
    if target.dtype != torch.int64 or target.dim() != 1 or target.shape[0] != x.shape[0]:
        raise ValueError(f"target must be int64 [{x.shape[0]}]")
    if w.device != x.device or target.device != x.device:
        raise ValueError("x, w and target must be on one device")
    tc._need_gpu(target)
    return tc.Xent(x.shape[0], w.shape[0], x.shape[1], ldx, ldw, ignore_index, chunk, tc._dt(x), 0)


def _no_tangent(*ts):
    """forward-mode derivatives are not computed: refused, not taken for zero"""
    for t in ts:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise NotImplementedError("the loss has no forward-mode derivative")


_ws_cache = {}
_ws_bytes = {}          # by sizes: what a call of a shape needs


def _workspace(c, grad: int, device, stream, ws):
    """the given workspace, else the stream's own (kept, and grown when a call needs more)"""
    if ws is not None:
        if ws.device != device or not ws.is_contiguous():
            raise ValueError(f"ws must be contiguous and on {device}")
        return ws
    shape = (device.index, grad, c.n, c.v, c.h, c.chunk, c.dt)
    need = _ws_bytes.get(shape)
    if need is None:
        n = C.c_size_t(0)
        tc._check(tc.lib().tc_xent_workspace_bytes(C.byref(c), grad, C.byref(n)), "tc_xent_workspace_bytes")
        if len(_ws_bytes) >= tc._PLANS_MAX:
            _ws_bytes.clear()
        need = _ws_bytes[shape] = n.value
    if torch.cuda.is_current_stream_capturing():
        # a graph keeps its own: a larger call would free the stream's under it
        return torch.empty(need, dtype=torch.uint8, device=device)
    key = (device.index, stream)
    ws = _ws_cache.get(key)
    if ws is None or ws.numel() < need:
        ws = None                   # (given back before the larger one is asked for)
        _ws_cache.pop(key, None)
        ws = _ws_cache[key] = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device=device)
    return ws


def free_workspaces():
    """give the kept workspaces back (a step over many tokens holds gigabytes)"""
    _ws_cache.clear()


def _loss(x, w, target, ignore_index, chunk=0, ws=None):
    c = _sizes(x, w, target, ignore_index, chunk)
    loss = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    lse = torch.empty_like(loss)
    st = tc._stream(x.device)
    with tc._stream_lock(x.device, st):
        ws = _workspace(c, 0, x.device, st, ws)
        tc._check(tc.lib().tc_xent_loss(C.byref(c), x.data_ptr(), w.data_ptr(), target.data_ptr(), loss.data_ptr(),
                                        lse.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), st), "tc_xent_loss")
    return loss, lse


def linear_xent_step(x: torch.Tensor, w: torch.Tensor, target: torch.Tensor, weight: Optional[torch.Tensor] = None,
                     ignore_index: int = -100, chunk: int = 0, out: XentStep = None, ws: torch.Tensor = None) -> XentStep:
    """losses of the tokens x [n, h] against w [v, h], and the gradients of
    sum(weight * loss) (weight: float32 [n], None: 1).  Rows of x and w may lie
    apart.  chunk: tokens whose softmax entries are held at once (0: as many
    as 4 GiB hold).  Tokens whose target is ignore_index do not count."""
    _no_tangent(x, w, weight)
    c = _sizes(x, w, target, ignore_index, chunk)
    if weight is not None and (weight.dtype != torch.float32 or weight.shape != target.shape or weight.device != x.device):
        raise ValueError(f"weight must be float32 [{x.shape[0]}] on {x.device}")
    tc._need_gpu(weight)
    if out is None:
        loss = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        out = XentStep(loss, torch.empty_like(loss), torch.empty(x.shape, dtype=x.dtype, device=x.device),
                       torch.empty(w.shape, dtype=w.dtype, device=w.device))
    else:
        for t, s, dt, name in ((out.loss, target.shape, torch.float32, "loss"), (out.lse, target.shape, torch.float32, "lse"),
                               (out.dx, x.shape, x.dtype, "dx"), (out.dw, w.shape, w.dtype, "dw")):
            if t.shape != s or t.dtype != dt or t.device != x.device:
                raise ValueError(f"out.{name} must be {dt} {list(s)} on {x.device}")
        tc._need_gpu(*out)
    st = tc._stream(x.device)
    with tc._stream_lock(x.device, st):
        ws = _workspace(c, 1, x.device, st, ws)
        tc._check(tc.lib().tc_xent_step(C.byref(c), x.data_ptr(), w.data_ptr(), target.data_ptr(), tc._ptr(weight),
                                        out.loss.data_ptr(), out.lse.data_ptr(), out.dx.data_ptr(), out.dw.data_ptr(),
                                        ws.data_ptr(), ws.numel() * ws.element_size(), st), "tc_xent_step")
    return out


class _LinearXent(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, target, ignore_index, chunk):
        loss, lse = _loss(x, w, target, ignore_index, chunk)
        ctx.save_for_backward(x, w, target)
        ctx.more = ignore_index, chunk
        ctx.mark_non_differentiable(lse)
        return loss, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g, _):
        x, w, target = ctx.saved_tensors
        r = linear_xent_step(x, w, target, g.to(torch.float32).contiguous(), *ctx.more)
        return r.dx, r.dw, None, None, None


def linear_xent(x: torch.Tensor, w: torch.Tensor, target: torch.Tensor, ignore_index: int = -100, chunk: int = 0):
    """(loss, lse), float32 [n]: the losses of the tokens x [n, h] against
    w [v, h].  The losses are differentiable in x and w, once and backward;
    lse is not."""
    _no_tangent(x, w)
    if torch.is_grad_enabled() and (x.requires_grad or w.requires_grad):
        return _LinearXent.apply(x, w, target, ignore_index, chunk)
    return _loss(x, w, target, ignore_index, chunk)
