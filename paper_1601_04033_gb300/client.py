"""Client operators on torch tensors: what a client computes between a fetch and a
push, besides its matrix products, when its model is a deep residual network.

``dropout``, ``join`` / ``join_grad`` and ``balance`` forward to the entry points
of the same names in include/fasgd.h, which say what they compute; they run on
torch's current stream and allocate their outputs and workspace from torch, on
that stream.  ``Join`` and ``dropped``, ``joined``, ``balanced`` are the same
calls inside torch's automatic differentiation.

Activations are fp32, bf16 or fp16 CUDA tensors, [..., cols], rows evenly spaced;
parameters (norm weights and biases, a learned gate) are fp32 -- views into the
client's flat copy of theta will do, and the gradients may be written straight
into views of the flat vector that is pushed.
"""

from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from . import fasgd as _f

_DTYPES = {torch.float32: _f.F32, torch.bfloat16: _f.BF16, torch.float16: _f.F16}
_NORMS = {"rms": _f.RMS_NORM, "layer": _f.LAYER_NORM}
_NOWHERE = 16      # stands for the address of a tensor without elements: never followed


class Draws(NamedTuple):
    """A dropout call's rate and whose draws it takes: the client's n-th.  n is
    to be another for every call that is to drop other elements."""
    rate: float
    seed: int = 0
    client: int = 0
    n: int = 0


def _check(rc: int):
    if rc < 0:
        raise _f.FasgdError(rc if rc in _f.STATUS_NAMES else _f.EINVAL, _f.fasgd_last_error(None))
    return rc


def _dtype(t) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"activations are fp32, bf16 or fp16, not {t.dtype}")
    return d


def _rows(t, like=None):
    """(address, rows, cols, ld) of a matrix [..., cols] whose rows are evenly spaced."""
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype):
        raise ValueError(f"{tuple(t.shape)} {t.dtype} given with {tuple(like.shape)} {like.dtype}")
    if not t.is_cuda:
        raise ValueError("CUDA tensors are expected")
    dim = t.dim()
    if dim != 2:
        if dim == 0:
            raise ValueError("a matrix [..., cols] is expected")
        try:
            t = t.view(-1, t.shape[-1])
        except RuntimeError:
            raise ValueError("the rows must be evenly spaced") from None
    rows, cols = t.shape
    step, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError("the values of a row must be contiguous")
    return t.data_ptr() or _NOWHERE, rows, cols, step


def _vector(t, cols: int, name: str):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != cols or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be {cols} contiguous fp32 values on the GPU")
    return t.data_ptr()


def dropout(x, draws: Draws, *, residual=None, out=None):
    """residual + dropout(x) (fasgd_dropout), in a new tensor or in `out`, which may
    be x or residual.  The gradient of x is dropout(gradient, draws)."""
    a = _f.DropoutArgs()
    a.x, a.rows, a.cols, a.ld_x = _rows(x)
    a.dtype = _dtype(x)
    if residual is not None:
        a.residual, _, _, a.ld_residual = _rows(residual, x)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    a.out, _, _, a.ld_out = _rows(out, x)
    a.rate, a.seed, a.client, a.n = draws
    _check(_f.fasgd_dropout(ctypes.addressof(a), _f._current_stream()))
    return out


class Joined:
    """What ``join`` gives: h (None without y), z (None without pre), and what
    ``join_grad`` needs: the tensors of the call (kept alive) and its arguments."""
    __slots__ = ("h", "z", "args", "x", "y", "parameters", "stats")


def join(x, y=None, *, post=None, post_bias=None, gate=None, pre=None, pre_bias=None, norm="rms",
         eps=1e-6, carry=1.0, branch=1.0, draws: Draws | None = None, h=None, z=None) -> Joined:
    """fasgd_join: h = carry x + branch gate dropout(N(y; post)), z = N(h; pre).
    gate: fp32 [cols], or [groups, cols] of fp32 or x's type, groups dividing the
    rows.  h, z: where to write them (new tensors if None)."""
    a = _f.JoinArgs()
    a.x, a.rows, cols, a.ld_x = _rows(x)
    a.cols = cols
    a.groups = 1
    a.dtype = _dtype(x)
    a.norm = _NORMS[norm]
    a.eps, a.carry, a.branch = eps, carry, branch
    if draws is not None:
        a.rate, a.seed, a.client, a.n = draws
    if y is not None:
        a.y, _, _, a.ld_y = _rows(y, x)
        if h is None:
            h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        a.h, _, _, a.ld_h = _rows(h, x)
    elif h is not None:
        raise ValueError("h goes with y")
    if pre is not None:
        if z is None:
            z = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        a.z, _, _, a.ld_z = _rows(z, x)
    elif z is not None:
        raise ValueError("z goes with pre")
    a.post, a.post_bias = _vector(post, cols, "post"), _vector(post_bias, cols, "post_bias")
    a.pre, a.pre_bias = _vector(pre, cols, "pre"), _vector(pre_bias, cols, "pre_bias")
    if gate is not None:
        if gate.dim() == 2:
            a.groups = gate.shape[0]
        if gate.shape[-1] != cols or gate.dim() > 2 or not gate.is_contiguous() or not gate.is_cuda:
            raise ValueError("gate must be contiguous [cols] or [groups, cols] on the GPU")
        a.gate, a.gate_dtype = gate.data_ptr(), _dtype(gate)
    stats = torch.empty(4 * a.rows, dtype=torch.float32, device=x.device)
    a.stats = stats.data_ptr() or _NOWHERE
    _check(_f.fasgd_join(ctypes.addressof(a), _f._current_stream()))
    j = Joined()
    j.h, j.z, j.args, j.x, j.y, j.stats = h, z, a, x, y, stats
    j.parameters = (post, post_bias, gate, pre, pre_bias)
    return j


class JoinGrads(NamedTuple):
    x: object = None
    y: object = None
    post: object = None
    post_bias: object = None
    gate: object = None
    pre: object = None
    pre_bias: object = None


def join_grad(j: Joined, dh, dz=None, *, into: JoinGrads = JoinGrads()) -> JoinGrads:
    """fasgd_join_grad: the gradients of ``join``'s x, y and parameters from those
    of its h (None: zero) and z.  x, y, the parameters and the stream's order are
    to be as they were.  into: where to write them (new tensors where None)."""
    a, x = _f.JoinArgs.from_buffer_copy(j.args), j.x
    post, post_bias, gate, pre, pre_bias = j.parameters
    if dh is not None:
        a.dh, _, _, a.ld_dh = _rows(dh, x)
    if dz is not None:
        a.dz, _, _, a.ld_dz = _rows(dz, x)

    dx = into.x if into.x is not None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    a.dx, _, _, a.ld_dx = _rows(dx, x)
    dy = None
    if j.y is not None:
        dy = into.y if into.y is not None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        a.dy, _, _, a.ld_dy = _rows(dy, x)
    cols = a.cols

    def vector(of, name):
        if of is None:
            return None, None
        t = getattr(into, name)
        if t is None:
            t = torch.empty_like(of)
            return t, t.data_ptr()
        return t, _vector(t, cols, name)

    dpost, a.dpost = vector(post, "post")
    dpost_bias, a.dpost_bias = vector(post_bias, "post_bias")
    dpre, a.dpre = vector(pre, "pre")
    dpre_bias, a.dpre_bias = vector(pre_bias, "pre_bias")
    dgate = None
    if gate is not None:
        dgate = into.gate if into.gate is not None else torch.empty_like(gate)
        if dgate.shape != gate.shape or dgate.dtype != gate.dtype or not dgate.is_contiguous():
            raise ValueError("the gate's gradient must be as the gate")
        a.dgate = dgate.data_ptr()
    at = ctypes.addressof(a)
    size = _check(_f.fasgd_join_workspace(at))
    space = torch.empty(size, dtype=torch.uint8, device=x.device)
    a.workspace, a.workspace_bytes = space.data_ptr(), size
    _check(_f.fasgd_join_grad(at, _f._current_stream()))
    return JoinGrads(dx, dy, dpost, dpost_bias, dgate, dpre, dpre_bias)


class Balance(NamedTuple):
    loss: object       # fp32[3]: the weighted sum, the balance loss, the z loss
    counts: object     # int32 [groups, experts]
    dlogits: object    # as logits, or None


def balance(logits, chosen, *, balance=0.01, z=0.0, groups=1, valid=None, upstream=None, grad=True) -> Balance:
    """fasgd_balance: a router's balance and z losses, its per-expert counts, and
    (grad) the gradient of the logits, times `upstream` (a device fp32 value) if
    given.  chosen: int32 [..., top]; valid: bool or uint8, one per row."""
    a = _f.BalanceArgs()
    a.logits, rows, a.cols, a.ld_logits = _rows(logits)
    a.rows, a.groups, a.top, a.dtype = rows, groups, chosen.shape[-1], _dtype(logits)
    a.balance_scale, a.z_scale = balance, z
    if chosen.dtype is not torch.int32 or not chosen.is_contiguous() or not chosen.is_cuda or \
            chosen.numel() != rows * a.top:
        raise ValueError("chosen must be contiguous int32 [..., top] on the GPU, a row for each of logits")
    a.chosen = chosen.data_ptr() or _NOWHERE
    if valid is not None:
        if valid.dtype not in (torch.uint8, torch.bool) or not valid.is_contiguous() or not valid.is_cuda or \
                valid.numel() != rows:
            raise ValueError("valid must be contiguous bool or uint8 on the GPU, one for each row")
        a.valid = valid.data_ptr()
    if upstream is not None:
        a.upstream = _vector(upstream, 1, "upstream")
    dlogits = None
    if grad:
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        a.dlogits, _, _, a.ld_dlogits = _rows(dlogits)
    counts = torch.empty((groups, a.cols), dtype=torch.int32, device=logits.device)
    loss = torch.empty(3, dtype=torch.float32, device=logits.device)
    a.counts, a.loss = counts.data_ptr(), loss.data_ptr()
    at = ctypes.addressof(a)
    size = _check(_f.fasgd_balance_workspace(at))
    space = torch.empty(size, dtype=torch.uint8, device=logits.device)
    a.workspace, a.workspace_bytes = space.data_ptr(), size
    _check(_f.fasgd_balance(at, _f._current_stream()))
    return Balance(loss, counts, dlogits)


# ---------------------------------------------------------------------------
# Inside torch's automatic differentiation
# ---------------------------------------------------------------------------
class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, draws):
        ctx.draws, ctx.both = draws, residual is not None
        return dropout(x, draws, residual=residual)

    @staticmethod
    def backward(ctx, d):
        return dropout(d.contiguous(), ctx.draws), d if ctx.both else None, None


def dropped(x, draws: Draws, residual=None):
    """``dropout``, differentiable in x and residual; no mask is kept."""
    return _Dropout.apply(x, residual, draws)


class _Join(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, post, post_bias, gate, pre, pre_bias, settings):
        j = join(x, y, post=post, post_bias=post_bias, gate=gate, pre=pre, pre_bias=pre_bias, **settings)
        ctx.save_for_backward(x, y, post, post_bias, gate, pre, pre_bias, j.stats)
        ctx.args = j.args
        ctx.set_materialize_grads(False)
        return j.h, j.z

    @staticmethod
    def backward(ctx, dh, dz):
        if dh is None and dz is None:
            return (None,) * 8
        x, y, post, post_bias, gate, pre, pre_bias, stats = ctx.saved_tensors
        j = Joined()
        j.args, j.x, j.y, j.stats = ctx.args, x, y, stats
        j.parameters = (post, post_bias, gate, pre, pre_bias)
        if dz is None and pre is not None:
            dz = torch.zeros_like(x, memory_format=torch.contiguous_format)
        g = join_grad(j, None if dh is None else dh.contiguous(), None if dz is None else dz.contiguous())
        return (*g, None)


def joined(x, y=None, *, post=None, post_bias=None, gate=None, pre=None, pre_bias=None, **settings):
    """``join``, differentiable in x, y and the parameters: (h, z), None where
    absent.  settings: norm, eps, carry, branch, draws."""
    return _Join.apply(x, y, post, post_bias, gate, pre, pre_bias, settings)


class _Balance(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, chosen, valid, settings):
        b = balance(logits, chosen, valid=valid, grad=False, **settings)
        ctx.save_for_backward(logits, chosen, valid)
        ctx.settings = settings
        ctx.mark_non_differentiable(b.counts)
        return b.loss[0], b.loss[1:], b.counts

    @staticmethod
    def backward(ctx, d, _parts, _counts):
        logits, chosen, valid = ctx.saved_tensors
        b = balance(logits, chosen, valid=valid, upstream=d.reshape(1), **ctx.settings)
        return b.dlogits, None, None, None


def balanced(logits, chosen, *, valid=None, **settings):
    """``balance``, differentiable in logits: (loss, [balance loss, z loss], counts);
    only the first has a gradient.  settings: balance, z, groups."""
    loss, parts, counts = _Balance.apply(logits, chosen, valid, settings)
    return loss, parts.detach(), counts
