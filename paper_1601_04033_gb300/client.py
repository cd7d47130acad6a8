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

A call's new tensors share one storage where they are small (1 MiB together): each
is contiguous and its own, but one that is kept keeps the others' memory, and its
storage must not be resized or freed by hand.  Tensors given as out, h, z or into
have the storages that they came with.
"""

from __future__ import annotations

import ctypes
import importlib
import warnings
from typing import NamedTuple

import torch

from . import fasgd as _f

_DTYPES = {torch.float32: _f.F32, torch.bfloat16: _f.BF16, torch.float16: _f.F16}
_NORMS = {"rms": _f.RMS_NORM, "layer": _f.LAYER_NORM}
_NOWHERE = 16      # stands for the address of a tensor without elements: never followed


def _module():
    """client_torch.cpp's module, if it was built for this torch."""
    try:
        m = importlib.import_module("._client", __package__)
    except ImportError as error:
        if not isinstance(error, ModuleNotFoundError):
            warnings.warn(f"{error}: the client operators go through ctypes", RuntimeWarning)
        return None
    if m.torch_version.split("+")[0] != torch.__version__.split("+")[0]:
        warnings.warn(f"_client was built for torch {m.torch_version}: the client operators go through ctypes",
                      RuntimeWarning)
        return None
    return m


_fast = _module()


class Draws(NamedTuple):
    """A dropout call's rate and whose draws it takes: the client's n-th.  n is
    to be another for every call that is to drop other elements.  seed counts modulo
    2^64; a client or n out of fasgd_dropout's range is refused."""
    rate: float
    seed: int = 0
    client: int = 0
    n: int = 0


def _check(rc: int):
    if rc < 0:
        raise _f.FasgdError(rc if rc in _f.STATUS_NAMES else _f.EINVAL, _f.fasgd_last_error(None))
    return rc


def _written(*given):
    """Tensors of the caller's (None: absent) that a call wrote into: their versions, which
    automatic differentiation looks at before it reads a tensor that it has saved."""
    for t in given:
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


def _done(result):
    """What a call of client_torch.cpp's gave: a negative status, or its tensors."""
    return _check(result) if type(result) is int else result


def _dtype(t) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"activations are fp32, bf16 or fp16, not {t.dtype}")
    return d


def _stream(t) -> int:
    """torch's current stream, which is to be on t's device."""
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError("CUDA tensors on the current device are expected")
    return _f._current_stream() if _raw_stream is None else _raw_stream(t.get_device())


def _one_device(first, *others):
    """The call's tensors (None: absent) are on one GPU; checked before any address is taken."""
    at = first.get_device()
    if any(t is not None and (not t.is_cuda or t.get_device() != at) for t in (first, *others)):
        raise ValueError("CUDA tensors on one device are expected")


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
    return t.data_ptr() or _NOWHERE, rows, cols, step


# The tensors of a call go into its argument struct by kind: the first matrix,
# which fixes rows, cols and dtype; matrices of its shape and type; fp32 vectors of
# cols values; and a gate, [cols] or [groups, cols] of fp32 or the first's type.
_FIRST, _LIKE, _VECTOR, _GATE = range(4)


def _intake(a, spec, *tensors):
    """Each tensor that is not None into struct a (its pointer, its ld, and what
    the first and the gate fix); ValueError where one is not what its kind says."""
    cols = None
    if hasattr(a, "gate_dtype"):
        a.groups = 1
    for (name, kind), t in zip(spec.items(), tensors):
        if t is None:
            continue
        p, rows, width, step = _rows(t)
        if kind == _FIRST:
            first, cols = t, width
            a.rows, a.cols, a.dtype = rows, width, _dtype(t)
        elif kind == _LIKE:
            if cols is not None and (t.shape != first.shape or t.dtype is not first.dtype):
                raise ValueError("matrices of one shape and type are expected")
        elif kind == _VECTOR:
            if t.dtype is not torch.float32 or t.numel() != (a.cols if cols is None else cols) or not t.is_contiguous():
                raise ValueError("parameters are contiguous fp32 vectors of cols values")
        else:
            if width != cols or t.dim() > 2 or not t.is_contiguous():
                raise ValueError("a gate is contiguous, [cols] or [groups, cols]")
            if t.dim() == 2:
                a.groups = rows
            a.gate_dtype = _dtype(t)
        setattr(a, name, p)
        if kind <= _LIKE:
            setattr(a, "ld_" + name, step)


def _draws(a, draws):
    """Draws into a struct, whose fields would cut a client or n beyond them to another's."""
    a.rate, a.seed, client, n = draws
    a.client = client if 0 <= client < 1 << 31 else -1
    a.n = n if 0 <= n < 1 << 63 else -1


def _new(like):
    """A new matrix of like's shape and type, without gaps."""
    if like.is_contiguous():
        return torch.empty_like(like)
    return torch.empty(like.shape, dtype=like.dtype, device=like.device)


_DROPOUT = dict(x=_FIRST, out=_LIKE, residual=_LIKE)


def dropout(x, draws: Draws, *, residual=None, out=None):
    """residual + dropout(x) (fasgd_dropout), in a new tensor or in `out`, which may
    be x or residual.  The gradient of x is dropout(gradient, draws)."""
    if _fast is not None:
        return _done(_fast.dropout(x, draws, residual, out))
    _one_device(x, residual, out)
    a = _f.DropoutArgs()
    at = ctypes.addressof(a)
    given = out
    if out is None:
        out = _new(x)
    _intake(a, _DROPOUT, x, out, residual)
    _draws(a, draws)
    _check(_f.fasgd_dropout(at, _stream(x)))
    _written(given)
    return out


class Joined:
    """What ``join`` gives: h (None without y), z (None without pre), and what
    ``join_grad`` needs: the tensors of the call (kept alive) and its settings (its
    argument struct; the addresses in it are not looked at again)."""
    __slots__ = ("h", "z", "args", "x", "y", "parameters", "stats")


_JOIN = dict(x=_FIRST, y=_LIKE, h=_LIKE, z=_LIKE, post=_VECTOR, post_bias=_VECTOR, gate=_GATE,
              pre=_VECTOR, pre_bias=_VECTOR)


def join(x, y=None, *, post=None, post_bias=None, gate=None, pre=None, pre_bias=None, norm="rms",
         eps=1e-6, carry=1.0, branch=1.0, draws: Draws | None = None, h=None, z=None) -> Joined:
    """fasgd_join: h = carry x + branch gate dropout(N(y; post)), z = N(h; pre).
    gate: fp32 [cols], or [groups, cols] of fp32 or x's type, groups dividing the
    rows.  h, z: where to write them (new tensors if None)."""
    j = Joined()
    j.x, j.y, j.parameters = x, y, (post, post_bias, gate, pre, pre_bias)
    if _fast is not None:
        j.h, j.z, j.stats, j.args = _done(_fast.join(x, y, post, post_bias, gate, pre, pre_bias, _NORMS[norm], eps, carry,
                                                     branch, draws, h, z))
        return j
    _one_device(x, y, *j.parameters, h, z)
    if (h is not None and y is None) or (z is not None and pre is None):
        raise ValueError("h goes with y, z with pre")
    given = h, z
    if y is not None and h is None:
        h = _new(x)
    if pre is not None and z is None:
        z = _new(x)
    a = _f.JoinArgs()
    at = ctypes.addressof(a)
    _intake(a, _JOIN, x, y, h, z, post, post_bias, gate, pre, pre_bias)
    a.norm = _NORMS[norm]
    a.eps = eps
    a.carry = carry
    a.branch = branch
    if draws is not None:
        _draws(a, draws)
    j.stats = torch.empty(4 * a.rows, dtype=torch.float32, device=x.device)
    a.stats = j.stats.data_ptr() or _NOWHERE
    _check(_f.fasgd_join(at, _stream(x)))
    _written(*given)
    j.h, j.z, j.args = h, z, bytes(a)
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
    of its h (None: zero) and z.  j's tensors (x, y, parameters, stats) may lie
    elsewhere by now; their values and the stream's order are to be as they were.
    into: where to write them (new tensors where None)."""
    x = j.x
    if _fast is not None:
        return JoinGrads(*_done(_fast.join_grad(j.args, x, j.y, dh, dz, j.parameters, into or _NO_GRADS, j.stats)))
    _one_device(x, j.y, *j.parameters, j.stats, dh, dz, *(into or _NO_GRADS))
    was = _f.JoinArgs.from_buffer_copy(j.args)
    a = _f.JoinArgs()
    at = ctypes.addressof(a)
    for name in _SETTINGS:
        setattr(a, name, getattr(was, name))
    given = into if into is not None else _NO_GRADS
    dx, dy, dpost, dpost_bias, dgate, dpre, dpre_bias = given
    post, post_bias, gate, pre, pre_bias = j.parameters
    if any(t is None and d is not None for t, d in zip((x, j.y, *j.parameters), given)):
        raise ValueError("the gradient of a tensor that is not there")
    if dx is None:
        dx = _new(x)
    if j.y is not None and dy is None:
        dy = _new(x)
    if post is not None and dpost is None:
        dpost = torch.empty_like(post)
    if post_bias is not None and dpost_bias is None:
        dpost_bias = torch.empty_like(post_bias)
    if pre is not None and dpre is None:
        dpre = torch.empty_like(pre)
    if pre_bias is not None and dpre_bias is None:
        dpre_bias = torch.empty_like(pre_bias)
    if gate is not None:
        if dgate is None:
            dgate = torch.empty_like(gate)
        elif dgate.shape != gate.shape or dgate.dtype is not gate.dtype or not dgate.is_contiguous():
            raise ValueError("the gate's gradient must be as the gate")
        a.dgate = dgate.data_ptr()
    _intake(a, _JOIN_GRAD, x, j.y, post, post_bias, gate, pre, pre_bias, dh, dz, dx, dy, dpost, dpost_bias, dpre,
            dpre_bias)
    if (a.rows, a.cols, a.dtype, a.groups) != (was.rows, was.cols, was.dtype, was.groups) or \
            any((getattr(a, n) is None) != (getattr(was, n) is None) for n in ("y", "post", "pre")):
        raise ValueError("join_grad: not the join's tensors")
    if j.stats.dtype is not torch.float32 or j.stats.numel() != 4 * a.rows or not j.stats.is_contiguous():
        raise ValueError("join_grad: not the join's statistics")
    a.stats = j.stats.data_ptr() or _NOWHERE
    size = _check(_f.fasgd_join_workspace(at))
    space = torch.empty(size, dtype=torch.uint8, device=x.device)
    a.workspace = space.data_ptr()
    a.workspace_bytes = size
    _check(_f.fasgd_join_grad(at, _stream(x)))
    _written(*given)
    return JoinGrads(dx, dy, dpost, dpost_bias, dgate, dpre, dpre_bias)


_NO_GRADS = JoinGrads()
# What join_grad takes of the forward call's struct; addresses are its own tensors'.
_SETTINGS = ("rate", "seed", "n", "client", "norm", "eps", "carry", "branch")
_JOIN_GRAD = dict(x=_FIRST, y=_LIKE, post=_VECTOR, post_bias=_VECTOR, gate=_GATE, pre=_VECTOR, pre_bias=_VECTOR,
                  dh=_LIKE, dz=_LIKE, dx=_LIKE, dy=_LIKE, dpost=_VECTOR, dpost_bias=_VECTOR, dpre=_VECTOR,
                  dpre_bias=_VECTOR)


class Balance(NamedTuple):
    loss: object       # fp32[3]: the weighted sum, the balance loss, the z loss
    counts: object     # int32 [groups, experts]
    dlogits: object    # as logits, or None


_BALANCE = dict(logits=_FIRST, dlogits=_LIKE)


def balance(logits, chosen, *, balance=0.01, z=0.0, groups=1, valid=None, upstream=None, grad=True) -> Balance:
    """fasgd_balance: a router's balance and z losses, its per-expert counts, and
    (grad) the gradient of the logits, times `upstream` (a device fp32 value) if
    given.  chosen: int32 [..., top]; valid: bool or uint8, one per row."""
    if _fast is not None:
        return Balance(*_done(_fast.balance(logits, chosen, balance, z, groups, valid, upstream, bool(grad))))
    _one_device(logits, chosen, valid, upstream)
    a = _f.BalanceArgs()
    at = ctypes.addressof(a)
    dlogits = _new(logits) if grad else None
    _intake(a, _BALANCE, logits, dlogits)
    rows = a.rows
    if not -(1 << 63) <= groups < 1 << 63:
        raise OverflowError("groups is beyond 64 bits")
    a.groups = groups
    a.top = top = chosen.shape[-1]
    a.balance_scale = balance
    a.z_scale = z
    if chosen.dtype is not torch.int32 or not chosen.is_contiguous() or chosen.numel() != rows * top:
        raise ValueError("chosen must be contiguous int32 [..., top] on the GPU, a row for each of logits")
    a.chosen = chosen.data_ptr() or _NOWHERE
    if valid is not None:
        if valid.dtype not in (torch.uint8, torch.bool) or not valid.is_contiguous() or valid.numel() != rows:
            raise ValueError("valid must be contiguous bool or uint8 on the GPU, one for each row")
        a.valid = valid.data_ptr()
    if upstream is not None:
        if upstream.dtype is not torch.float32 or upstream.numel() != 1:
            raise ValueError("upstream must be one fp32 value on the GPU")
        a.upstream = upstream.data_ptr()
    size = _check(_f.fasgd_balance_workspace(at))
    device = logits.device
    counts = torch.empty((groups, a.cols), dtype=torch.int32, device=device)
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
class _Once(torch.autograd.Function):
    """Gradients as they are, with an error in place of their derivatives."""
    @staticmethod
    def forward(ctx, count, *tensors):
        return tuple(None if t is None else t.detach() for t in tensors[:count])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the join and the balance loss have no second derivatives here")


def _once(grads, *of):
    """What a backward call returns of `grads`, which depend on the tensors `of`.  Where
    a graph is made of the call, a derivative through it raises: they are plain
    tensors, whose part would be missing without a word."""
    return _Once.apply(len(grads), *grads, *of) if torch.is_grad_enabled() else grads


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, draws):
        ctx.draws, ctx.both = draws, residual is not None
        return dropout(x, draws, residual=residual)

    @staticmethod
    def backward(ctx, d):
        again = dropped if torch.is_grad_enabled() else dropout      # linear: its gradient's gradient is its own
        return again(d.contiguous(), ctx.draws), d if ctx.both else None, None


def dropped(x, draws: Draws, residual=None):
    """``dropout``, differentiable in x and residual, any number of times; no mask is kept."""
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
        *inputs, stats = ctx.saved_tensors
        x, y, post, post_bias, gate, pre, pre_bias = inputs
        j = Joined()
        j.args, j.x, j.y, j.stats = ctx.args, x, y, stats
        j.parameters = (post, post_bias, gate, pre, pre_bias)
        with torch.no_grad():
            if dz is None and pre is not None:
                dz = torch.zeros_like(x, memory_format=torch.contiguous_format)
            g = join_grad(j, None if dh is None else dh.contiguous(), None if dz is None else dz.contiguous())
        return (*_once(g, dh, dz, *inputs), None)


def joined(x, y=None, *, post=None, post_bias=None, gate=None, pre=None, pre_bias=None, **settings):
    """``join``, differentiable in x, y and the parameters: (h, z), None where
    absent.  settings: norm, eps, carry, branch, draws.  A second derivative raises."""
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
        with torch.no_grad():
            b = balance(logits, chosen, valid=valid, upstream=d.reshape(1), **ctx.settings)
        return (*_once((b.dlogits,), d, logits), None, None, None)


def balanced(logits, chosen, *, valid=None, **settings):
    """``balance``, differentiable in logits: (loss, [balance loss, z loss], counts);
    only the first has a gradient, and a second derivative of it raises.  settings:
    balance, z, groups."""
    loss, parts, counts = _Balance.apply(logits, chosen, valid, settings)
    return loss, parts.detach(), counts
