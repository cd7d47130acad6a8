"""Client operators on torch tensors: what a client computes between a fetch and a
push when its model is a deep residual network with routed experts and a loss over
classes.

``dropout``, ``join`` / ``join_grad``, ``balance``, ``route``, ``gather``, ``combine`` /
``combine_grad``, ``multiply`` / ``multiply_grad`` and ``score`` forward to the entry
points of the same names in include/fasgd.h, which say what they compute; they run on
torch's current stream and allocate their outputs and workspace from torch, on
that stream.  ``dropped``, ``joined``, ``balanced``, ``gathered``, ``combined``,
``multiplied`` and ``scored`` are the same calls inside torch's automatic
differentiation.  ``sync`` waits for them and raises where a product gave up.

Activations are fp32, bf16 or fp16 CUDA tensors, [..., cols], rows evenly spaced;
parameters (norm weights and biases, a learned gate, experts' matrices) are fp32 --
views into the client's flat copy of theta will do, and the gradients may be written
straight into views of the flat vector that is pushed.  Experts' matrices may be of the
activations' type too; ``score``'s classes are.

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


class Route(NamedTuple):
    """What ``route`` gives: each expert's first place, each place's entry, each entry's place."""
    offsets: object    # int32 [experts + 1]
    order: object      # int32 [rows * top]
    place: object      # int32 [rows, top]


def _ints(t, what):
    if t.dtype is not torch.int32 or not t.is_contiguous():
        raise ValueError(what + " must be contiguous int32 on the GPU")
    return t.data_ptr() or _NOWHERE


def _space(a, workspace, like):
    """The workspace of a call, which its struct gets too."""
    size = _check(workspace(ctypes.addressof(a)))
    space = torch.empty(size, dtype=torch.uint8, device=like.device)
    a.workspace = space.data_ptr()
    a.workspace_bytes = size
    return space


def route(chosen, experts: int) -> Route:
    """fasgd_route: a router's choices (int32 [..., top]; outside [0, experts): none) into
    the experts' order."""
    if _fast is not None:
        return Route(*_done(_fast.route(chosen, experts)))
    _one_device(chosen)
    a = _f.RouteArgs()
    if chosen.dim() == 0:
        raise ValueError("chosen must be contiguous int32 on the GPU, [..., top]")
    a.chosen = _ints(chosen, "chosen")
    a.top = chosen.shape[-1]
    a.rows = chosen.numel() // a.top if a.top else 0
    if not -(1 << 63) <= experts < 1 << 63:
        raise OverflowError("experts is beyond 64 bits")
    a.experts = experts
    space = _space(a, _f.fasgd_route_workspace, chosen)
    n = chosen.numel()
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=chosen.device)
    order = torch.empty(n, dtype=torch.int32, device=chosen.device)
    place = torch.empty_like(chosen)
    a.offsets = offsets.data_ptr()
    a.order = order.data_ptr() or _NOWHERE
    a.place = place.data_ptr() or _NOWHERE
    _check(_f.fasgd_route(ctypes.addressof(a), _stream(chosen)))
    del space
    return Route(offsets, order, place)


def _exchange(rows_like, route, weight=None):
    """A struct of the calls between rows and places, with the route's part."""
    a = _f.ExchangeArgs()
    _, order, place = route
    if place.dim() == 0:
        raise ValueError("a route's place is [..., top]")
    a.top = place.shape[-1]
    a.rows = place.numel() // a.top if a.top else 0
    a.place = _ints(place, "a route's place")
    a.order = _ints(order, "a route's order")
    if order.numel() != place.numel():
        raise ValueError("a route's order and place have as many entries as each other")
    a.dtype = _dtype(rows_like)
    if weight is not None:
        if weight.dtype is not torch.float32 or weight.numel() != place.numel() or not weight.is_contiguous():
            raise ValueError("weight must be contiguous fp32, one for each entry")
        a.weight = weight.data_ptr() or _NOWHERE
    return a


def _at_rows(a, t):
    a.row_values, rows, cols, a.ld_rows = _rows(t)
    if rows != a.rows or (a.cols and cols != a.cols):
        raise ValueError("a matrix with a row for each of the route's is expected, as wide as its places")
    a.cols = cols


def _at_places(a, t):
    p, rows, cols, ld = _rows(t)
    if rows != a.rows * a.top or (a.cols and cols != a.cols):
        raise ValueError("a matrix with a row for each of the route's places is expected, as wide as its rows")
    a.cols = cols
    return p, ld


def _same_type(t, of):
    if t.dtype is not of.dtype:
        raise ValueError("matrices of one type are expected")


def gather(x, route: Route, *, out=None):
    """fasgd_gather: x's rows at their places, [rows * top, cols]; 0 at places that no entry has."""
    if _fast is not None:
        return _done(_fast.gather(x, tuple(route), out))
    _one_device(x, route.order, route.place, out)
    a = _exchange(x, route)
    _at_rows(a, x)
    given = out
    if out is None:
        out = torch.empty((a.rows * a.top, a.cols), dtype=x.dtype, device=x.device)
    _same_type(out, x)
    a.places, a.ld_places = _at_places(a, out)
    _check(_f.fasgd_gather(ctypes.addressof(a), _stream(x)))
    _written(given)
    return out


def combine(y, route: Route, weight=None, *, out=None):
    """fasgd_combine: each row's sum over its places in y, times weight (fp32, as the route's
    place) if given: [..., cols]."""
    if _fast is not None:
        return _done(_fast.combine(y, tuple(route), weight, out))
    _one_device(y, route.order, route.place, weight, out)
    a = _exchange(y, route, weight)
    a.places, a.ld_places = _at_places(a, y)
    given = out
    if out is None:
        out = torch.empty((*route.place.shape[:-1], a.cols), dtype=y.dtype, device=y.device)
    _same_type(out, y)
    _at_rows(a, out)
    _check(_f.fasgd_combine(ctypes.addressof(a), _stream(y)))
    _written(given)
    return out


class CombineGrads(NamedTuple):
    y: object = None
    weight: object = None


def combine_grad(y, route: Route, weight, dout, *, into: CombineGrads | None = None) -> CombineGrads:
    """fasgd_combine_grad: the gradients of ``combine``'s y and weight from that of its result.
    into: where to write them (new tensors where None)."""
    dy, dweight = into if into is not None else (None, None)
    if _fast is not None:
        return CombineGrads(*_done(_fast.combine_grad(y, tuple(route), weight, dout, dy, dweight)))
    _one_device(y, route.order, route.place, weight, dout, dy, dweight)
    if weight is None:
        raise ValueError("the gradient of a combination without weights is gather's")
    a = _exchange(y, route, weight)
    a.places, a.ld_places = _at_places(a, y)
    _same_type(dout, y)
    _at_rows(a, dout)
    given = dy, dweight
    if dy is None:
        dy = torch.empty((a.rows * a.top, a.cols), dtype=y.dtype, device=y.device)
    _same_type(dy, y)
    a.dplaces, a.ld_dplaces = _at_places(a, dy)
    if dweight is None:
        dweight = torch.empty_like(weight)
    elif dweight.dtype is not torch.float32 or dweight.numel() != weight.numel() or not dweight.is_contiguous():
        raise ValueError("the weights' gradient must be as the weights")
    a.dweight = dweight.data_ptr() or _NOWHERE
    _check(_f.fasgd_combine_grad(ctypes.addressof(a), _stream(y)))
    _written(*given)
    return CombineGrads(dy, dweight)


def _matrices(t, dims):
    """(address, shape, ld, step, flip) of a matrix, or of several one step apart, whose rows or
    (flip) columns are consecutive values."""
    if t.dim() != dims:
        raise ValueError("a matrix is expected" if dims == 2 else "[experts, inputs, outputs] is expected")
    rows, cols = t.shape[-2:]
    down, along = t.stride()[-2:]
    if along == 1 or cols == 1:
        flip, ld = 0, down
    elif down == 1 or rows == 1:
        flip, ld = 1, along
    else:
        raise ValueError("the values of a matrix' rows or columns must be contiguous")
    return t.data_ptr() or _NOWHERE, t.shape, ld, t.stride(0) if dims == 3 else 0, flip


def _products(x, w, offsets):
    """A struct of the experts' products without their matrices' addresses."""
    a = _f.MultiplyArgs()
    a.x, a.rows, a.inputs, a.ld_x = _rows(x)
    a.dtype = _dtype(x)
    a.w, (a.experts, inputs, a.outputs), a.ld_w, a.step_w, a.w_flip = _matrices(w, 3)
    if inputs != a.inputs:
        raise ValueError("w is [experts, x's columns, outputs]")
    if w.dtype is not torch.float32 and w.dtype is not x.dtype:
        raise ValueError("w is of fp32 or of x's type")
    a.w_dtype = _dtype(w)
    a.offsets = _ints(offsets, "offsets")
    if offsets.numel() != a.experts + 1:
        raise ValueError("offsets has one entry more than there are experts")
    return a


def multiply(x, w, offsets, *, out=None):
    """fasgd_multiply: rows of x, in their experts' order, times their experts' matrices
    w[e] ([experts, inputs, outputs], rows or columns contiguous; fp32 or x's type); 0
    where no expert has the row.  offsets: ``route``'s."""
    if _fast is not None:
        return _done(_fast.multiply(x, w, offsets, out))
    _one_device(x, w, offsets, out)
    a = _products(x, w, offsets)
    given = out
    if out is None:
        out = torch.empty((*x.shape[:-1], a.outputs), dtype=x.dtype, device=x.device)
    _same_type(out, x)
    a.y, rows, cols, a.ld_y = _rows(out)
    if (rows, cols) != (a.rows, a.outputs):
        raise ValueError("out is [x's rows, w's outputs]")
    space = _space(a, _f.fasgd_multiply_workspace, x)
    _check(_f.fasgd_multiply(ctypes.addressof(a), _stream(x)))
    del space
    _written(given)
    return out


class MultiplyGrads(NamedTuple):
    x: object = None
    w: object = None


def multiply_grad(x, w, offsets, dy, *, grads=(True, True), into: MultiplyGrads | None = None) -> MultiplyGrads:
    """fasgd_multiply_grad: the gradients of ``multiply``'s x (in x's type) and w (in w's type and
    layout) from that of its result.  grads: which of them; into: where to write them
    (new tensors where None)."""
    dx, dw = into if into is not None else (None, None)
    if _fast is not None:
        return MultiplyGrads(*_done(_fast.multiply_grad(x, w, offsets, dy, bool(grads[0]), bool(grads[1]), dx, dw)))
    _one_device(x, w, offsets, dy, dx, dw)
    a = _products(x, w, offsets)
    a.dy, rows, cols, a.ld_dy = _rows(dy)
    _same_type(dy, x)
    if (rows, cols) != (a.rows, a.outputs):
        raise ValueError("dy is [x's rows, w's outputs]")
    given = dx, dw
    if (dx is not None and not grads[0]) or (dw is not None and not grads[1]):
        raise ValueError("a place for a gradient that is not wanted")
    if grads[0]:
        if dx is None:
            dx = _new(x)
        _same_type(dx, x)
        a.dx, rows, cols, a.ld_dx = _rows(dx)
        if (rows, cols) != (a.rows, a.inputs):
            raise ValueError("x's gradient is as x")
    if grads[1]:
        if dw is None:
            dw = torch.empty_like(w)
        _same_type(dw, w)
        a.dw, shape, a.ld_dw, a.step_dw, a.dw_flip = _matrices(dw, 3)
        if shape != w.shape:
            raise ValueError("w's gradient is as w")
    space = _space(a, _f.fasgd_multiply_workspace, x)
    _check(_f.fasgd_multiply_grad(ctypes.addressof(a), _stream(x)))
    del space
    _written(*given)
    return MultiplyGrads(dx, dw)


class Score(NamedTuple):
    loss: object       # fp32 [1]
    rows: object       # fp32, as labels: each row's loss, 0 without a label
    dz: object         # as z, or None
    dw: object         # as w, or None
    lse: object        # fp32, as labels: each row's log-sum-exp (any value without a label)


def score(z, w, labels, *, upstream=None, grad=True, grads=(True, True), known: Score | None = None, into=None) -> Score:
    """fasgd_score: softmax cross entropy of z w ([..., cols] x [cols, classes], w of z's type, rows
    or columns contiguous) against labels (int64, one for each row of z; outside
    [0, classes): none), the mean over the rows that have one, and (grad) the gradients
    of z and w that `grads` names, times `upstream` (a device fp32 value) if given.
    known: what an earlier call with these z, w and labels gave: only gradients are
    computed.  into: (dz, dw), where to write them (new tensors where None)."""
    loss, rows, *_, lse = known if known is not None else (None,) * 5
    want = (bool(grad and grads[0]), bool(grad and grads[1]))
    dz, dw = into if into is not None else (None, None)
    if _fast is not None:
        return Score(*_done(_fast.score(z, w, labels, upstream, *want, loss, rows, lse, dz, dw)))
    _one_device(z, w, labels, upstream, loss, rows, lse, dz, dw)
    a = _f.ScoreArgs()
    a.z, a.rows, a.cols, a.ld_z = _rows(z)
    a.dtype = _dtype(z)
    a.w, (cols, a.classes), a.ld_w, _, a.w_flip = _matrices(w, 2)
    _same_type(w, z)
    if cols != a.cols:
        raise ValueError("w is [z's columns, classes]")
    if labels.dtype is not torch.int64 or not labels.is_contiguous() or labels.numel() != a.rows:
        raise ValueError("labels must be contiguous int64 on the GPU, one for each row")
    a.labels = labels.data_ptr() or _NOWHERE
    if upstream is not None:
        if upstream.dtype is not torch.float32 or upstream.numel() != 1:
            raise ValueError("upstream must be one fp32 value on the GPU")
        a.upstream = upstream.data_ptr()
    given = dz, dw
    if (dz is not None and not want[0]) or (dw is not None and not want[1]):
        raise ValueError("a place for a gradient that is not wanted")
    if want[0]:
        if dz is None:
            dz = _new(z)
        _same_type(dz, z)
        a.dz, *shape, a.ld_dz = _rows(dz)
        if shape != [a.rows, a.cols]:
            raise ValueError("z's gradient is as z")
    if want[1]:
        if dw is None:
            dw = torch.empty_like(w)
        _same_type(dw, w)
        a.dw, shape, a.ld_dw, _, a.dw_flip = _matrices(dw, 2)
        if shape != w.shape:
            raise ValueError("w's gradient is as w")
    if known is None:
        loss = torch.empty(1, dtype=torch.float32, device=z.device)
        rows, lse = (torch.empty(labels.shape, dtype=torch.float32, device=z.device) for _ in range(2))
        a.loss = loss.data_ptr()
    else:
        if any(t.dtype is not torch.float32 or t.numel() != a.rows or not t.is_contiguous() for t in (rows, lse)):
            raise ValueError("known rows and lse must be contiguous fp32, one for each row")
        a.known = 1
    a.row_loss = rows.data_ptr() or _NOWHERE
    a.lse = lse.data_ptr() or _NOWHERE
    space = _space(a, _f.fasgd_score_workspace, z)
    _check(_f.fasgd_score(ctypes.addressof(a), _stream(z)))
    del space
    _written(*given)
    return Score(loss, rows, dz, dw, lse)


def sync():
    """fasgd_client_sync: waits for torch's current stream, and raises where a wait inside a
    product has run out on this device since the last call, so that its results are NaN."""
    late = ctypes.c_int32()
    device = torch._C._cuda_getDevice()
    _check(_f.fasgd_client_sync(ctypes.byref(late), _f._current_stream() if _raw_stream is None else _raw_stream(device)))
    if late.value:
        raise _f.FasgdError(_f.EDEVICE, "a wait inside a product on the tensor cores ran out: its results are NaN")


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
        raise RuntimeError("the client operators but dropout, gather and an unweighted combine have no second derivatives here")


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


class _Gather(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, offsets, order, place):
        ctx.save_for_backward(offsets, order, place)
        ctx.shape = x.shape
        return gather(x, Route(offsets, order, place))

    @staticmethod
    def backward(ctx, d):
        again = combined if torch.is_grad_enabled() else combine
        return again(d.contiguous(), Route(*ctx.saved_tensors)).reshape(ctx.shape), None, None, None


def gathered(x, route: Route):
    """``gather``, differentiable in x, any number of times."""
    return _Gather.apply(x, *route)


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weight, offsets, order, place):
        ctx.save_for_backward(None if weight is None else y, weight, offsets, order, place)
        ctx.shape = y.shape
        return combine(y, Route(offsets, order, place), weight)

    @staticmethod
    def backward(ctx, d):
        y, weight, *route = ctx.saved_tensors
        d = d.contiguous()
        if weight is None:
            again = gathered if torch.is_grad_enabled() else gather
            return again(d, Route(*route)).reshape(ctx.shape), None, None, None, None
        with torch.no_grad():
            g = combine_grad(y, Route(*route), weight, d)
        dy, dweight = _once((g.y.reshape(ctx.shape), g.weight), d, y, weight)
        return dy, dweight, None, None, None


def combined(y, route: Route, weight=None):
    """``combine``, differentiable in y and weight; without weights any number of times, with
    them a second derivative raises."""
    return _Combine.apply(y, weight, *route)


class _Multiply(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, offsets):
        ctx.save_for_backward(x, w, offsets)
        return multiply(x, w, offsets)

    @staticmethod
    def backward(ctx, d):
        x, w, offsets = ctx.saved_tensors
        with torch.no_grad():
            g = multiply_grad(x, w, offsets, d.contiguous(), grads=ctx.needs_input_grad[:2])
        return (*_once(g, d, x, w), None)


def multiplied(x, w, offsets):
    """``multiply``, differentiable in x and w (an fp32 w has an fp32 gradient); a second
    derivative raises."""
    return _Multiply.apply(x, w, offsets)


class _Score(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, w, labels):
        s = score(z, w, labels, grad=False)
        rows = s.rows.clone()        # the caller's, who may write into it
        ctx.save_for_backward(z, w, labels, s.rows, s.lse)
        ctx.mark_non_differentiable(rows)
        return s.loss.reshape(()), rows

    @staticmethod
    def backward(ctx, d, _rows):
        z, w, labels, rows, lse = ctx.saved_tensors
        with torch.no_grad():
            s = score(z, w, labels, upstream=d.reshape(1), grads=ctx.needs_input_grad[:2],
                      known=Score(None, rows, None, None, lse))
        return (*_once((s.dz, s.dw), d, z, w), None)


def scored(z, w, labels):
    """``score``, differentiable in z and w: (loss, each row's); only the first has a gradient,
    and a second derivative of it raises."""
    return _Score.apply(z, w, labels)
