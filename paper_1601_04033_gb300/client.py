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


# A small call is bound by the host, so tensors are asked as few questions as
# will do (each costs 0.06 to 0.2 us, a new tensor 1.4 us).
def _stream(t) -> int:
    """torch's current stream, which is to be on t's device."""
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError("CUDA tensors on the current device are expected")
    return _f._current_stream() if _raw_stream is None else _raw_stream(t.get_device())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _rows(t):
    """(address, rows, cols, ld) of a matrix [..., cols] whose rows are evenly spaced."""
    if t.dim() != 2:
        if t.dim() == 0:
            raise ValueError("a matrix [..., cols] is expected")
        try:
            t = t.view(-1, t.shape[-1])
        except RuntimeError:
            raise ValueError("the rows must be evenly spaced") from None
    rows, cols = t.shape
    step, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError("the values of a row must be contiguous")
    if not t.is_cuda:
        raise ValueError("CUDA tensors are expected")
    return t.data_ptr() or _NOWHERE, rows, cols, step


def _like(t, like):
    """(address, ld) of a matrix of like's shape and type."""
    if t.shape != like.shape or t.dtype is not like.dtype:
        raise ValueError(f"{tuple(t.shape)} {t.dtype} given with {tuple(like.shape)} {like.dtype}")
    p, _, _, step = _rows(t)
    return p, step


def _new(like, cols):
    """A new matrix of like's shape and type, without gaps: (tensor, address, ld)."""
    t = torch.empty(like.shape, dtype=like.dtype, device=like.device)
    return t, t.data_ptr() or _NOWHERE, cols


def _vector(t, cols: int, name: str):
    if t.dtype is not torch.float32 or t.numel() != cols or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be {cols} contiguous fp32 values on the GPU")
    return t.data_ptr()


def dropout(x, draws: Draws, *, residual=None, out=None):
    """residual + dropout(x) (fasgd_dropout), in a new tensor or in `out`, which may
    be x or residual.  The gradient of x is dropout(gradient, draws)."""
    a = _f.DropoutArgs()
    a.x, a.rows, cols, a.ld_x = _rows(x)
    a.cols = cols
    a.dtype = _dtype(x)
    if residual is not None:
        a.residual, a.ld_residual = _like(residual, x)
    if out is None:
        out, a.out, a.ld_out = _new(x, cols)
    else:
        a.out, a.ld_out = _like(out, x)
    a.rate, a.seed, a.client, a.n = draws
    _check(_f.fasgd_dropout(ctypes.addressof(a), _stream(x)))
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
    j = Joined()
    a = j.args = _f.JoinArgs()
    a.x, rows, cols, a.ld_x = _rows(x)
    a.rows = rows
    a.cols = cols
    a.groups = 1
    a.dtype = _dtype(x)
    a.norm = _NORMS[norm]
    a.eps = eps
    a.carry = carry
    a.branch = branch
    if draws is not None:
        a.rate, a.seed, a.client, a.n = draws
    if y is not None:
        a.y, a.ld_y = _like(y, x)
        if h is None:
            h, a.h, a.ld_h = _new(x, cols)
        else:
            a.h, a.ld_h = _like(h, x)
    elif h is not None:
        raise ValueError("h goes with y")
    if pre is not None:
        a.pre = _vector(pre, cols, "pre")
        if z is None:
            z, a.z, a.ld_z = _new(x, cols)
        else:
            a.z, a.ld_z = _like(z, x)
    elif z is not None:
        raise ValueError("z goes with pre")
    if post is not None:
        a.post = _vector(post, cols, "post")
    if post_bias is not None:
        a.post_bias = _vector(post_bias, cols, "post_bias")
    if pre_bias is not None:
        a.pre_bias = _vector(pre_bias, cols, "pre_bias")
    if gate is not None:
        if gate.dim() == 2:
            a.groups = gate.shape[0]
        if gate.shape[-1] != cols or gate.dim() > 2 or not gate.is_contiguous() or not gate.is_cuda:
            raise ValueError("gate must be contiguous [cols] or [groups, cols] on the GPU")
        a.gate, a.gate_dtype = gate.data_ptr(), _dtype(gate)
    j.stats = torch.empty(4 * rows, dtype=torch.float32, device=x.device)
    a.stats = j.stats.data_ptr() or _NOWHERE
    _check(_f.fasgd_join(ctypes.addressof(a), _stream(x)))
    j.h, j.z, j.x, j.y = h, z, x, y
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


def join_grad(j: Joined, dh, dz=None, *, into: JoinGrads | None = None) -> JoinGrads:
    """fasgd_join_grad: the gradients of ``join``'s x, y and parameters from those
    of its h (None: zero) and z.  x, y, the parameters and the stream's order are
    to be as they were.  into: where to write them (new tensors where None)."""
    a, x = _f.JoinArgs.from_buffer_copy(j.args), j.x
    cols = a.cols
    dx, dy, dpost, dpost_bias, dgate, dpre, dpre_bias = into if into is not None else _NO_GRADS
    post, post_bias, gate, pre, pre_bias = j.parameters
    if dh is not None:
        a.dh, a.ld_dh = _like(dh, x)
    if dz is not None:
        a.dz, a.ld_dz = _like(dz, x)
    if dx is None:
        dx, a.dx, a.ld_dx = _new(x, cols)
    else:
        a.dx, a.ld_dx = _like(dx, x)
    if j.y is None:
        dy = None
    elif dy is None:
        dy, a.dy, a.ld_dy = _new(x, cols)
    else:
        a.dy, a.ld_dy = _like(dy, x)
    if post is not None:
        dpost, a.dpost = _grad_vector(dpost, post, cols)
    if post_bias is not None:
        dpost_bias, a.dpost_bias = _grad_vector(dpost_bias, post_bias, cols)
    if pre is not None:
        dpre, a.dpre = _grad_vector(dpre, pre, cols)
    if pre_bias is not None:
        dpre_bias, a.dpre_bias = _grad_vector(dpre_bias, pre_bias, cols)
    if gate is not None:
        if dgate is None:
            dgate = torch.empty_like(gate)
        elif dgate.shape != gate.shape or dgate.dtype is not gate.dtype or not dgate.is_contiguous():
            raise ValueError("the gate's gradient must be as the gate")
        a.dgate = dgate.data_ptr()
    at = ctypes.addressof(a)
    size = _check(_f.fasgd_join_workspace(at))
    space = torch.empty(size, dtype=torch.uint8, device=x.device)
    a.workspace = space.data_ptr()
    a.workspace_bytes = size
    _check(_f.fasgd_join_grad(at, _stream(x)))
    return JoinGrads(dx, dy, dpost, dpost_bias, dgate, dpre, dpre_bias)


_NO_GRADS = JoinGrads()


def _grad_vector(t, of, cols):
    if t is None:
        t = torch.empty_like(of)
        return t, t.data_ptr()
    return t, _vector(t, cols, "a parameter's gradient")


class Balance(NamedTuple):
    loss: object       # fp32[3]: the weighted sum, the balance loss, the z loss
    counts: object     # int32 [groups, experts]
    dlogits: object    # as logits, or None


def balance(logits, chosen, *, balance=0.01, z=0.0, groups=1, valid=None, upstream=None, grad=True) -> Balance:
    """fasgd_balance: a router's balance and z losses, its per-expert counts, and
    (grad) the gradient of the logits, times `upstream` (a device fp32 value) if
    given.  chosen: int32 [..., top]; valid: bool or uint8, one per row."""
    a = _f.BalanceArgs()
    a.logits, rows, cols, a.ld_logits = _rows(logits)
    a.rows, a.cols, a.groups, top = rows, cols, groups, chosen.shape[-1]
    a.top = top
    a.dtype = _dtype(logits)
    a.balance_scale = balance
    a.z_scale = z
    if chosen.dtype is not torch.int32 or not chosen.is_contiguous() or not chosen.is_cuda or \
            chosen.numel() != rows * top:
        raise ValueError("chosen must be contiguous int32 [..., top] on the GPU, a row for each of logits")
    a.chosen = chosen.data_ptr() or _NOWHERE
    if valid is not None:
        if valid.dtype not in (torch.uint8, torch.bool) or not valid.is_contiguous() or not valid.is_cuda or \
                valid.numel() != rows:
            raise ValueError("valid must be contiguous bool or uint8 on the GPU, one for each row")
        a.valid = valid.data_ptr()
    if upstream is not None:
        a.upstream = _vector(upstream, 1, "upstream")
    at = ctypes.addressof(a)
    size = _check(_f.fasgd_balance_workspace(at))
    dlogits = None
    if grad:
        dlogits, a.dlogits, a.ld_dlogits = _new(logits, cols)
    device = logits.device
    counts = torch.empty((groups, cols), dtype=torch.int32, device=device)
    loss = torch.empty(3, dtype=torch.float32, device=device)
    space = torch.empty(size, dtype=torch.uint8, device=device)
    a.counts = counts.data_ptr()
    a.loss = loss.data_ptr()
    a.workspace = space.data_ptr()
    a.workspace_bytes = size
    _check(_f.fasgd_balance(at, _stream(logits)))
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
