"""Layer operators of a language model for all workers of a level at once (hop_linear, hop_norm_*, hop_dropout of
include/hop.h) on torch tensors.

Rows (tokens) of all workers stand one behind the other, sorted by group; `offsets` (int32, device, groups + 1 entries,
see group_offsets) says where each group's rows begin.  A group is a worker with weights of its own, or an expert.  Norm
weights and gates may be views into the float32 replica ring X, gradients of weights may be written into rows of G.

  grouped_linear, grouped_linear_dx, grouped_linear_dw     products with each group's weights and their gradients
  residual_norm, residual_norm_backward                    norm, gate, dropout, residual sum and the next block's norm
  dropout, dropout_backward                                mask from a counter-based generator, never stored
  GroupedLinear, ResidualNorm, Dropout                     the same under torch.autograd (.apply), differentiable once

The plain functions record nothing for autograd: their results have no history, whatever their inputs require.  What out=
writes counts as an in-place change of that tensor; one that requires a gradient is refused unless under no_grad.

Everything runs on the current stream of the tensors' device; outputs and workspaces come from torch's allocator.  A
wrong argument raises HopError (E_ARG, E_UNSUPPORTED) before anything is launched."""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import NamedTuple, Optional

import torch

from . import hop
from .hop import HopError

if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_hop_nn.so")):
    raise ImportError("_hop_nn.so is missing: build it with `python -m paper_1902_01064_b200.build`")
from . import _hop_nn  # noqa: E402  (checks, outputs and workspaces; it calls the entries of the library that hop loaded)

_hop_nn.bind(HopError, *(C.cast(getattr(hop.lib, name), C.c_void_p).value for name in
                         ("hop_linear_workspace", "hop_linear", "hop_norm_workspace", "hop_norm_forward", "hop_norm_backward", "hop_dropout")))


def _bad(msg):
    raise HopError(hop.E_ARG, msg)


def group_offsets(counts, device="cuda") -> torch.Tensor:
    """offsets from the number of rows of each group (host integers, checked here)."""
    counts = [int(c) for c in counts]
    if not counts or min(counts) < 0 or sum(counts) >= 1 << 31 or len(counts) > hop.MAX_GROUPS:
        _bad(f"counts: 1 .. {hop.MAX_GROUPS} non-negative integers, below 2^31 in all, expected")
    ends = [0]
    for c in counts:
        ends.append(ends[-1] + c)
    return torch.tensor(ends, dtype=torch.int32).to(device)


# ---------------------------------------------------------------------------------------------- grouped products
def grouped_linear(x, w, offsets=None, *, out=None, out_dtype=None):
    """y[t] = W_g x[t] for the group g of row t.  x: rows x k; w: (groups, n, k), or (n, k) for one group."""
    return _hop_nn.linear_rows(hop.LINEAR_FORWARD, x, w, offsets, out, out_dtype)


def grouped_linear_dx(dy, w, offsets=None, *, out=None, out_dtype=None):
    """dx[t] = W_g^T dy[t]."""
    return _hop_nn.linear_rows(hop.LINEAR_DX, dy, w, offsets, out, out_dtype)


def grouped_linear_dw(dy, x, offsets=None, *, out=None, out_dtype=torch.float32, accumulate=False):
    """dW_g = sum over the group's rows of dy[t] x[t]^T, float32 by default; out: (groups, n, k) of any group and row
    stride (a view into G), added to with accumulate=True."""
    return _hop_nn.linear_dw(dy, x, offsets, out, out_dtype, accumulate)


def linear_status(device=None) -> int:
    """Error word of the product kernels on the device (0: every bounded wait was met); synchronises and clears it."""
    word, buf = C.c_int32(), C.create_string_buffer(512)
    with torch.cuda.device(device):
        rc = hop.lib.hop_linear_status(C.byref(word), buf, 512)
    if rc:
        raise HopError(rc, buf.value.decode())
    return word.value


# ---------------------------------------------------------------------------------------------- the end of a block
class NormGrads(NamedTuple):
    dx: torch.Tensor
    db: Optional[torch.Tensor]
    dw_post: Optional[torch.Tensor]
    dc_post: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dw_pre: Optional[torch.Tensor]
    dc_pre: Optional[torch.Tensor]
    dtoken_gate: Optional[torch.Tensor]


def residual_norm(x, b=None, *, w_post=None, c_post=None, gate=None, token_gate=None, w_pre=None, c_pre=None, offsets=None,
                  kind="rms", post=None, pre=None, eps=1e-5, scale=1.0, skip=1.0, p=0.0, seed=0, step=0, site=0):
    """(r, h):  r = skip * x + scale * drop(gate * norm(b)),  h = norm(r).

    norm(b) has weight w_post and shift c_post (post=True: a norm without either; without any of them b is taken as it
    is); norm(r) likewise with w_pre, c_pre, pre (h is None when nothing asks for it).  gate: a vector per group;
    token_gate: a row array.  kind "rms" (no shifts) or "layer".  drop: dropout(.., p, seed, step, site)'s mask.
    Without b, r is x itself.  r and h have x's shape."""
    return _hop_nn.norm_forward(x, b, token_gate, w_post, c_post, gate, w_pre, c_pre, offsets, kind, post, pre, eps, scale, skip, p, seed, step, site)


def residual_norm_backward(dr, dh, r, b=None, *, w_post=None, c_post=None, gate=None, token_gate=None, w_pre=None, c_pre=None,
                           offsets=None, kind="rms", post=None, pre=None, eps=1e-5, scale=1.0, skip=1.0, p=0.0, seed=0, step=0,
                           site=0, out=None) -> NormGrads:
    """Gradients of residual_norm from those of r and h (either may be None), with r as the forward pass returned it.  dx has
    r's shape, db and dtoken_gate those of b and token_gate.
    out: float32 (groups, columns) destinations by name (dw_post, dc_post, dgate, dw_pre, dc_pre), e.g. views into G."""
    return NormGrads._make(_hop_nn.norm_backward(dr, dh, r, b, token_gate, w_post, c_post, gate, w_pre, c_pre, offsets, kind, post, pre, eps, scale, skip, p,
                                                 seed, step, site, out))


# ---------------------------------------------------------------------------------------------- dropout
def dropout(x, p, seed, *, step=0, site=0, out=None):
    """x / (1 - p) where kept, 0 where dropped; the mask is a function of (seed, step, site, row, column) alone.  step
    counts iterations, site tells apart the places of a model that draw a mask.  The row is the place in x: where rows are
    sorted by group, a group's mask moves with the number of rows before it.  out may be x."""
    return _hop_nn.dropout(x, p, seed, step, site, out)


def dropout_backward(dy, p, seed, *, step=0, site=0, out=None):
    """Gradient of dropout with the same p, seed, step and site: the same mask on dy."""
    return _hop_nn.dropout(dy, p, seed, step, site, out)


# ---------------------------------------------------------------------------------------------- under torch.autograd
def _grad_rows(g):
    """A gradient as the operators take it: rows of unit stride along the columns.  autograd hands out expanded and transposed
    ones, whose leading dimensions need not join into rows; those are copied."""
    if g is None or g.numel() == 0:
        return g
    g = g.reshape(-1, g.shape[-1])
    return g if g.stride(1) == 1 or g.shape[1] == 1 else g.contiguous()


class _Final(torch.autograd.Function):
    """Gradients as they are, tied to what they were formed from by a derivative that raises."""

    @staticmethod
    def forward(ctx, count, *tensors):
        return tuple(t.detach() for t in tensors[:count])

    @staticmethod
    def backward(ctx, *grads):
        raise HopError(hop.E_UNSUPPORTED, "the layer operators' gradients can be formed once only: they have no second derivatives")


def _once(backward):
    """A backward pass whose results cannot be differentiated again: neither with respect to the incoming gradients nor to the
    saved tensors, on which they depend as well."""
    @functools.wraps(backward)
    def wrapped(ctx, *grads):
        if not torch.is_grad_enabled():         # no create_graph
            return backward(ctx, *grads)
        with torch.no_grad():
            out = list(backward(ctx, *grads))
        given = [t for t in (*grads, *ctx.saved_tensors) if t is not None and t.requires_grad]
        at = [i for i, t in enumerate(out) if t is not None]
        if given and at:
            for i, t in zip(at, _Final.apply(len(at), *(out[i] for i in at), *given)):
                out[i] = t
        return tuple(out)
    return wrapped


# Enters beside the tensors where gradients are written into destinations: backward is then recorded, and run, although
# neither rows nor weights require a gradient (the first layer on data).  It gets no gradient itself.
_DESTINATION = torch.empty(0, requires_grad=True)


class GroupedLinear(torch.autograd.Function):
    """apply(x, w, offsets, dw_into=None, accumulate=False): grouped_linear, in x's leading dimensions.  With dw_into (float32,
    e.g. a view into G) backward() writes the weight gradient there, whatever requires a gradient, and w itself gets none;
    else it comes in w's type.  (torch.autograd.grad runs only what leads to the inputs that it is given.)"""

    @classmethod
    def apply(cls, x, w, offsets=None, dw_into=None, accumulate=False):
        return super().apply(x, w, offsets, dw_into, accumulate, None if dw_into is None else _DESTINATION)

    @staticmethod
    def forward(ctx, x, w, offsets, dw_into, accumulate, destination):
        ctx.save_for_backward(x, w, offsets)
        ctx.into, ctx.accumulate = dw_into, accumulate
        return grouped_linear(x, w, offsets).view(*x.shape[:-1], w.shape[-2])

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, w, offsets = ctx.saved_tensors
        dy = _grad_rows(dy)
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = grouped_linear_dx(dy, w, offsets).view_as(x)
        if ctx.into is not None:
            grouped_linear_dw(dy, x, offsets, out=ctx.into, accumulate=ctx.accumulate)
        elif ctx.needs_input_grad[1]:
            dw = grouped_linear_dw(dy, x, offsets, out_dtype=w.dtype).view_as(w)
        return dx, dw, None, None, None, None


class ResidualNorm(torch.autograd.Function):
    """apply(x, b, w_post, c_post, gate, token_gate, w_pre, c_pre, offsets, options): residual_norm; options is a dict of its
    other arguments, and "out" of residual_norm_backward's destinations (written by backward() whatever requires a gradient;
    vectors whose gradient goes there get none)."""

    @classmethod
    def apply(cls, x, b, w_post, c_post, gate, token_gate, w_pre, c_pre, offsets=None, options=None):
        return super().apply(x, b, w_post, c_post, gate, token_gate, w_pre, c_pre, offsets, options, _DESTINATION if options and options.get("out") else None)

    @staticmethod
    def forward(ctx, x, b, w_post, c_post, gate, token_gate, w_pre, c_pre, offsets, options, destination):
        ctx.options = dict(options or {})
        ctx.into = ctx.options.pop("out", None) or {}
        r, h = residual_norm(x, b, w_post=w_post, c_post=c_post, gate=gate, token_gate=token_gate, w_pre=w_pre, c_pre=c_pre, offsets=offsets,
                             **ctx.options)
        ctx.save_for_backward(x if b is None else r, b, w_post, c_post, gate, token_gate, w_pre, c_pre, offsets)
        ctx.set_materialize_grads(False)
        if b is None:
            r = x.view_as(x)
        return r, h

    @staticmethod
    @_once
    def backward(ctx, dr, dh):
        r, b, w_post, c_post, gate, token_gate, w_pre, c_pre, offsets = ctx.saved_tensors
        if dr is None and dh is None:
            for t in ctx.into.values():
                t.zero_()
            return (None,) * 11
        g = residual_norm_backward(_grad_rows(dr), _grad_rows(dh), r, b, w_post=w_post, c_post=c_post, gate=gate, token_gate=token_gate, w_pre=w_pre, c_pre=c_pre,
                                   offsets=offsets, out=ctx.into, **ctx.options)

        def vector(name, v):
            return None if v is None or "d" + name in ctx.into else getattr(g, "d" + name).view_as(v)
        return (g.dx, g.db, vector("w_post", w_post), vector("c_post", c_post), vector("gate", gate), g.dtoken_gate, vector("w_pre", w_pre),
                vector("c_pre", c_pre), None, None, None)


class Dropout(torch.autograd.Function):
    """apply(x, p, seed, step, site): dropout."""

    @staticmethod
    def forward(ctx, x, p, seed, step=0, site=0):
        ctx.args = (p, seed, step, site)
        return dropout(x, p, seed, step=step, site=site)

    @staticmethod
    @_once
    def backward(ctx, dy):
        p, seed, step, site = ctx.args
        return dropout_backward(_grad_rows(dy), p, seed, step=step, site=site).view_as(dy), None, None, None, None
