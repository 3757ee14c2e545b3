"""The matrix operators of ``include/evo.h``: calls on torch tensors that need no solver.

All of them enqueue their work on ``stream`` (the current stream of the tensors' device if it is None), allocate their
outputs and workspaces through torch on that stream, and return without waiting.  Where that is not the stream on which an argument
was made, ordering the two and keeping the argument until the work is done are the caller's.  Arguments that the library cannot
take raise ``EvoError``; there is no fallback.  None of them has a backward pass that torch records: while torch records gradients, tensors that require one are
refused (detach them, or call under ``torch.no_grad()``), and so are dual tensors of forward mode, whose tangent would be lost.  Gradients are calls of their own: a training step of a mixture of members (or experts) is

    routes = route_rows(members, groups)                    # members [rows, choices], gates [rows, choices]
    xs = take_rows(x, routes.place)
    ys = grouped_linear(xs, weight, routes.offsets, bias, activation="tanh")
    logits = combine_rows(ys, routes.place, gates)
    loss, logp, d_logits = policy_loss(logits, actions, old_logp, advantage)
    d_ys, d_gates = combine_rows_backward(d_logits, ys, routes.place, gates)
    d_xs, d_weight, d_bias = grouped_linear_backward(d_ys, xs, weight, routes.offsets, ys, activation="tanh")
    d_x = combine_rows(d_xs, routes.place)

and ``muon_step`` (which ascends: give it the gradient's negative) takes what it gives.
"""
from __future__ import annotations

import ctypes as C
import math
from functools import lru_cache
from typing import NamedTuple, Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad

from .binding import (EVO_MAX_LAYERS, Actions, EvoError, Grouped, GroupedGradient, Matrices, Matrix, Muon, NewtonSchulz, PolicyRows, RoutePairs, RowSets, _check,
                      load_library)

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INVALID_ARG = 1
_ROW_SETS, _GROUPED, _GROUPED_GRADIENT = C.sizeof(RowSets), C.sizeof(Grouped), C.sizeof(GroupedGradient)
ACTIVATIONS = {"none": 0, "tanh": 1, "relu": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
_LEAST = math.ulp(0.0)


def _require(condition: bool, where: str, what: str) -> None:
    if not condition:
        error = EvoError(INVALID_ARG, where)
        error.args = (f"{error.args[0]}: {what}",)
        raise error


def _require_no_gradient(where: str, *tensors: Optional[torch.Tensor]) -> None:
    for x in tensors:
        if x is not None and x.requires_grad and torch.is_grad_enabled():
            _require(False, where, "a tensor requires a gradient, and there is no backward pass")
    if forward_ad._current_level >= 0:
        for x in tensors:
            _require(x is None or forward_ad.unpack_dual(x).tangent is None, where, "a dual tensor, and no tangent is carried on")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # the handle without a Stream object (2 us)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class _On:
    """The tensors' device, and the stream the call goes to (one of that device), as the current ones (allocations belong to that stream).  Entering
    gives the stream's handle; nothing is switched where both are current already (6 us of a small call)."""
    __slots__ = ("device", "stream", "guard")

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream], where: str):
        self.device, self.stream, self.guard = device, stream, None
        if stream is not None:
            _require(stream.device == device, where, "a stream of another device")

    def __enter__(self) -> int:
        if self.stream is not None:
            self.guard = torch.cuda.stream(self.stream)
        elif self.device.index != _current_device():
            self.guard = torch.cuda.device(self.device)
        if self.guard is not None:
            self.guard.__enter__()
        if self.stream is not None:
            return self.stream.cuda_stream
        return _raw_stream(self.device.index) if _raw_stream else torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


@lru_cache(maxsize=256)
def _newton_schulz(steps: int, coefficients: Tuple[float, ...], eps: float, where: str) -> NewtonSchulz:
    # (the structure takes zeros, and what fp32 rounds to zero, for its defaults)
    _require(1 <= steps <= 64 and len(coefficients) == 3 and any(C.c_float(x).value for x in coefficients) and C.c_float(eps).value > 0, where,
             "steps, coefficients or eps")
    return NewtonSchulz(C.sizeof(NewtonSchulz), steps, *coefficients, eps)


@lru_cache(maxsize=1024)
def _orthogonalize_bytes(batch: int, rows: int, cols: int) -> int:
    need = C.c_size_t()
    _check(load_library().evo_orthogonalize_bytes(batch, rows, cols, C.byref(need)), "orthogonalize")
    return need.value


@lru_cache(maxsize=256)
def _matrix_list(matrices: Tuple[Tuple[int, int, int], ...], dim: int):
    """(array of evo_matrix, how many, bytes of workspace)"""
    where = "muon_step"
    _require(all(o >= 0 and 1 <= r <= 1 << 20 and 1 <= c <= 1 << 20 for o, r, c in matrices), where, "matrices are (offset, rows, cols)")
    n = len(matrices)
    items, need = (Matrix * max(n, 1))(*(Matrix(o, r, c) for o, r, c in matrices)), C.c_size_t()
    _check(load_library().evo_muon_bytes(items, n, dim, C.byref(need)), where)
    return items, n, need.value


def _matrices(x: torch.Tensor, shape, strides) -> Matrices:
    rows, cols = shape[-2:]
    # a stride that is never taken may be anything
    row_stride = strides[-2] if rows > 1 else cols
    batch = shape[0] if len(shape) == 3 else 1
    return Matrices(x.data_ptr(), TYPES[x.dtype], batch, rows, cols, strides[0] if batch > 1 else rows * row_stride, row_stride)


def orthogonalize(x: torch.Tensor, out: Optional[torch.Tensor] = None, *, steps: int = 5,
                  coefficients: Sequence[float] = COEFFICIENTS, eps: float = 1e-7,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_orthogonalize``: every matrix of ``x`` ([rows, cols] or [batch, rows, cols]; fp32, bf16 or fp16; unit
    column stride, rows and matrices one behind the other at any pitch) with its singular values moved towards 1 by Newton-Schulz steps.  ``out`` may
    be ``x``."""
    lib, where = load_library(), "orthogonalize"
    _require_no_gradient(where, x, out)
    _require(x.is_cuda and x.dtype in TYPES and x.dim() in (2, 3), where, "a fp32, bf16 or fp16 matrix or batch on a GPU")
    _require(x.shape[-1] == 1 or x.stride(-1) == 1, where, "the columns of x need unit stride")
    ns = _newton_schulz(steps, tuple(coefficients), eps, where)
    shape, device = x.shape, x.device
    with _On(device, stream, where) as st:
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=device)
        else:
            _require(out.device == device and out.dtype == x.dtype and out.shape == shape, where, "out must match x")
            _require(shape[-1] == 1 or out.stride(-1) == 1, where, "the columns of out need unit stride")
        if 0 in shape:
            return out
        a, b = _matrices(x, shape, x.stride()), _matrices(out, shape, out.stride())
        need = _orthogonalize_bytes(a.batch, a.rows, a.cols)
        work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        code = lib.evo_orthogonalize(C.byref(ns), C.byref(a), C.byref(b), None if work is None else work.data_ptr(), need, st)
    _check(code, where)
    return out


def muon_step(center: torch.Tensor, m: torch.Tensor, v: torch.Tensor, gradient: torch.Tensor,
              matrices: Sequence[Tuple[int, int, int]], step: int, *, lr: float, momentum: float = 0.95,
              nesterov: bool = True, weight_decay: float = 0.0, ns_steps: int = 5,
              coefficients: Sequence[float] = COEFFICIENTS, eps: float = 1e-7, beta1: float = 0.9, beta2: float = 0.999,
              adam_eps: float = 1e-8, out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
              stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """``evo_muon_step`` on flat fp32 vectors; ``matrices`` lists (offset, rows, cols) of the weight matrices.  Returns
    the new (center, m, v); ``out=(center, m, v)`` takes the step in place.  ``beta1``, ``beta2`` and ``adam_eps`` are taken as they
    are, 0 included."""
    lib, where = load_library(), "muon_step"
    vectors = (center, m, v, gradient) + (tuple(out) if out is not None else ())
    _require(len(vectors) in (4, 7), where, "out needs three vectors")
    _require_no_gradient(where, *vectors)
    for x in vectors:
        _require(x.is_cuda and x.device == center.device and x.dtype == torch.float32 and x.dim() == 1 and x.is_contiguous() and
                 x.numel() == center.numel(), where, "contiguous fp32 vectors of one length on one GPU")
    ns = _newton_schulz(ns_steps, tuple(coefficients), eps, where)
    # 0 selects a default in the structure; here it is the caller's: the smallest double instead, which is 0 in the kernel's fp32 (and 1 - beta is 1)
    cfg = Muon(C.sizeof(Muon), 0 if nesterov else 1, lr, momentum, weight_decay, beta1 or _LEAST, beta2 or _LEAST, adam_eps or _LEAST, ns)
    _require(1 <= step < 1 << 32, where, "the step counts from 1")
    dim = center.numel()
    items, n, need = _matrix_list(tuple(map(tuple, matrices)), dim)
    with _On(center.device, stream, where) as st:
        if out is None:
            out = (torch.empty_like(center), torch.empty_like(m), torch.empty_like(v))
        if dim == 0:
            return tuple(out)
        work = torch.empty(need, dtype=torch.uint8, device=center.device) if need else None
        code = lib.evo_muon_step(C.byref(cfg), items, n, dim, step, center.data_ptr(), m.data_ptr(), v.data_ptr(), gradient.data_ptr(),
                                 out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), None if work is None else work.data_ptr(), need, st)
    _check(code, where)
    return tuple(out)


def _rows(x: torch.Tensor, dtype: torch.dtype, device: torch.device) -> bool:
    return x.device == device and x.dtype == dtype and x.dim() == 2 and (x.stride(1) == 1 or x.shape[1] <= 1)


def _ragged(offsets: torch.Tensor, groups: int, device: torch.device, where: str) -> int:
    dtype = offsets.dtype
    _require(offsets.device == device and (dtype == torch.int32 or dtype == torch.int64) and offsets.shape == (groups + 1,) and
             offsets.is_contiguous(), where, "offsets: int32 or int64 on the same GPU, one more than groups")
    return 1 if dtype == torch.int64 else 0


def _out(out: Optional[torch.Tensor], x: torch.Tensor, rows: int, cols: int, where: str) -> torch.Tensor:
    if out is None:
        return x.new_empty((rows, cols))
    _require(_rows(out, x.dtype, x.device) and out.shape == (rows, cols), where, "out does not match")
    return out


def grouped_linear(x: torch.Tensor, weight: torch.Tensor, offsets: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                   activation: str = "none", scale: float = 1.0, out: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_grouped_linear``: ``y[r] = scale * act(weight[g] @ x[r] + bias[g])`` for the rows ``offsets[g] <= r < offsets[g + 1]``.
    x [rows, n_in], weight [groups, n_out, n_in], bias [groups, n_out]; fp32, bf16 or fp16; unit stride in the last dimension, any
    other strides that keep rows apart (a layer of theta is ``theta[:, a:b].unflatten(1, (n_out, n_in))``; an expanded weight is shared).  Rows outside all
    groups are left as they are in ``out``, and undefined without one.  ``out`` may not lie between the elements of another argument."""
    lib, where, device, dtype = load_library(), "grouped_linear", x.device, x.dtype
    _require_no_gradient(where, x, weight, bias, out)
    _require(x.is_cuda and dtype in TYPES and _rows(x, dtype, device), where, "x: fp32, bf16 or fp16 rows on a GPU")
    _require(weight.device == device and weight.dtype == dtype and weight.dim() == 3, where, "weight does not match x")
    groups, n_out, n_in = weight.shape
    rows = x.shape[0]
    stride, pitch, one = weight.stride()
    _require(groups >= 1 and n_out >= 1 and n_in >= 1 and n_in == x.shape[1] and (n_in == 1 or one == 1) and stride >= 0 and pitch >= 0, where,
             "weight does not match x")
    _require(activation in ACTIVATIONS, where, "activation")
    if bias is not None:
        _require(_rows(bias, dtype, device) and bias.shape == (groups, n_out), where, "bias does not match")
    wide = _ragged(offsets, groups, device, where)
    with _On(device, stream, where) as st:
        y = _out(out, x, rows, n_out, where)
        p = Grouped(C.sizeof(Grouped), TYPES[dtype], groups, n_in, n_out, ACTIVATIONS[activation], scale, wide, rows,
                    x.data_ptr(), x.stride(0), weight.data_ptr(), pitch if n_out > 1 else n_in, stride,
                    None if bias is None else bias.data_ptr(), 0 if bias is None else bias.stride(0), offsets.data_ptr(), y.data_ptr(),
                    y.stride(0))
        need = C.c_size_t()
        _check(lib.evo_grouped_linear_bytes(C.byref(p), C.byref(need)), where)
        work = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
        code = lib.evo_grouped_linear(C.byref(p), None if work is None else work.data_ptr(), need.value, st)
    _check(code, where)
    return y


@lru_cache(maxsize=256)
def _layers(sizes: Tuple[int, ...]):
    """(parameters, the widths as evo_actions has them)"""
    _require(2 <= len(sizes) <= EVO_MAX_LAYERS + 1 and min(sizes) >= 1 and max(sizes) <= 1 << 20, "mlp_actions", "layer_sizes")
    return sum((a + 1) * b for a, b in zip(sizes[:-1], sizes[1:])), (C.c_uint32 * (EVO_MAX_LAYERS + 1))(*sizes)


def mlp_actions(theta: torch.Tensor, layer_sizes: Sequence[int], observations: torch.Tensor, offsets: torch.Tensor, *,
                action_scale: float = 1.0, out: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_mlp_actions``: the MLP policy's actions for rows of observations, ``offsets[m] <= r < offsets[m + 1]`` being member m's.
    theta [members, >= parameters] fp32 as ``Solver.ask`` returns it (row pitch a multiple of 4, rows 16-byte aligned),
    layer_sizes the widths, input first.  Rows without a member are left as they are in ``out``, and undefined without one."""
    lib, where, device = load_library(), "mlp_actions", observations.device
    _require_no_gradient(where, theta, observations, out)
    sizes = tuple(layer_sizes)
    dim, widths = _layers(sizes)
    _require(observations.is_cuda and _rows(observations, torch.float32, device) and observations.shape[1] == sizes[0], where,
             "observations: fp32 rows of the first layer's width on a GPU")
    members, rows = theta.shape[0], observations.shape[0]
    _require(_rows(theta, torch.float32, device) and members >= 1 and theta.shape[1] >= dim, where, "theta does not match")
    wide = _ragged(offsets, members, device, where)
    with _On(device, stream, where) as st:
        y = _out(out, observations, rows, sizes[-1], where)
        pitch = theta.stride(0) if members > 1 else -(-max(dim, theta.stride(0)) // 4) * 4
        p = Actions(C.sizeof(Actions), members, len(sizes) - 1, widths, action_scale, wide, rows, theta.data_ptr(), pitch,
                    observations.data_ptr(), observations.stride(0), offsets.data_ptr(), y.data_ptr(), y.stride(0))
        need = C.c_size_t()
        _check(lib.evo_mlp_actions_bytes(C.byref(p), C.byref(need)), where)
        work = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
        code = lib.evo_mlp_actions(C.byref(p), None if work is None else work.data_ptr(), need.value, st)
    _check(code, where)
    return y


class Routes(NamedTuple):
    """Pairs of a row and a choice sorted by member: ``offsets`` [groups + 1], ``source`` [pairs] (the pair at each place, -1 behind the last), ``place``
    (of ``members``' shape, -1 without a member); int32."""
    offsets: torch.Tensor
    source: torch.Tensor
    place: torch.Tensor


def _pairs(x: torch.Tensor, dtype: torch.dtype, device: torch.device, shape=None) -> bool:
    return x.device == device and x.dtype == dtype and x.dim() in (1, 2) and (x.dim() == 1 or x.stride(1) == 1 or x.shape[1] <= 1) and \
        (shape is None or x.shape == shape)


@lru_cache(maxsize=1024)
def _route_bytes(groups: int, choices: int, rows: int) -> int:
    need, p = C.c_size_t(), RoutePairs(C.sizeof(RoutePairs), groups, choices, 0, rows, None, choices)
    _check(load_library().evo_route_rows_bytes(C.byref(p), C.byref(need)), "route_rows")
    return need.value


def route_rows(members: torch.Tensor, groups: int, *, stream: Optional[torch.cuda.Stream] = None) -> Routes:
    """``evo_route_rows``: the stable order by member of the pairs of ``members`` ([rows] or [rows, choices], int32 or int64).  Numbers outside
    [0, groups) are no member: padded rows, choices that were dropped."""
    lib, where, device = load_library(), "route_rows", members.device
    _require(members.is_cuda and members.dtype in (torch.int32, torch.int64) and _pairs(members, members.dtype, device), where,
             "members: int32 or int64, [rows] or [rows, choices], on a GPU")
    choices = members.shape[1] if members.dim() == 2 else 1
    _require(1 <= groups <= 1 << 20 and choices >= 1 and members.numel() < 1 << 31, where, "groups or members")
    with _On(device, stream, where) as st:
        n = members.numel()
        like = members if members.dtype == torch.int32 else torch.empty(0, dtype=torch.int32, device=device)
        routes = Routes(like.new_empty(groups + 1), like.new_empty(n), like.new_empty(members.shape))
        p = RoutePairs(C.sizeof(RoutePairs), groups, choices, 1 if members.dtype == torch.int64 else 0, members.shape[0], members.data_ptr(),
                       members.stride(0), *(x.data_ptr() for x in routes))
        need = _route_bytes(groups, choices, members.shape[0])
        work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        code = lib.evo_route_rows(C.byref(p), None if work is None else work.data_ptr(), need, st)
    _check(code, where)
    return routes


def _row_sets(rows: torch.Tensor, sorted_rows: torch.Tensor, place: torch.Tensor, weights: Optional[torch.Tensor]) -> RowSets:
    count, cols = rows.shape
    at, pitch = (None, 0) if weights is None else (weights.data_ptr(), weights.stride(0))
    return RowSets(_ROW_SETS, TYPES[rows.dtype], place.shape[1] if place.dim() == 2 else 1, cols, count, sorted_rows.shape[0], place.data_ptr(), place.stride(0), at, pitch,
                   rows.data_ptr(), rows.stride(0), sorted_rows.data_ptr(), sorted_rows.stride(0))


def _check_rows(where: str, x: torch.Tensor, place: torch.Tensor, weights: Optional[torch.Tensor], rows: Optional[int]) -> None:
    device = x.device
    _require(x.is_cuda and x.dtype in TYPES and x.dim() == 2 and x.shape[1] >= 1 and (x.stride(1) == 1 or x.shape[1] == 1), where, "fp32, bf16 or fp16 rows on a GPU")
    shape = place.shape
    _require(place.device == device and place.dtype == torch.int32 and
             (len(shape) == 1 or (len(shape) == 2 and shape[1] >= 1 and (place.stride(1) == 1 or shape[1] == 1))) and (rows is None or shape[0] == rows), where,
             "place: int32, [rows] or [rows, choices], as route_rows gives it")
    _require(weights is None or (weights.device == device and weights.dtype == torch.float32 and weights.shape == shape and
                                 (len(shape) == 1 or weights.stride(1) == 1 or shape[1] == 1)), where, "weights: fp32, of place's shape")


def take_rows(x: torch.Tensor, place: torch.Tensor, weights: Optional[torch.Tensor] = None, *, out: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_take_rows``: ``out[place[r, j]] = weights[r, j] * x[r]`` (weights None: 1), the rows in sorted order.  Rows that no place names are left as
    they are in ``out``, and undefined without one (which has a row for every pair).  The gradient of x is ``combine_rows(d_out, place, weights)``."""
    lib, where, device = load_library(), "take_rows", x.device
    _require_no_gradient(where, x, weights, out)
    _check_rows(where, x, place, weights, x.shape[0] if x.dim() else 0)
    _require(out is None or out.dim() == 2, where, "out does not match")
    with _On(device, stream, where) as st:
        y = _out(out, x, place.numel() if out is None else out.shape[0], x.shape[1], where)
        code = lib.evo_take_rows(C.byref(_row_sets(x, y, place, weights)), st)
    _check(code, where)
    return y


def combine_rows(y: torch.Tensor, place: torch.Tensor, weights: Optional[torch.Tensor] = None, *, out: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_combine_rows``: ``out[r] = sum over j of weights[r, j] * y[place[r, j]]`` (weights None: 1), rows back from sorted order; zeros where
    a row has no place."""
    lib, where, device = load_library(), "combine_rows", y.device
    _require_no_gradient(where, y, weights, out)
    _check_rows(where, y, place, weights, None)
    with _On(device, stream, where) as st:
        x = _out(out, y, place.shape[0], y.shape[1], where)
        code = lib.evo_combine_rows(C.byref(_row_sets(x, y, place, weights)), st)
    _check(code, where)
    return x


def combine_rows_backward(d_out: torch.Tensor, y: torch.Tensor, place: torch.Tensor, weights: torch.Tensor, *, out: Optional[torch.Tensor] = None,
                          stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``evo_combine_rows_backward``: the gradients (of y, of weights) of ``combine_rows(y, place, weights)`` for the gradient ``d_out`` of its result.
    Rows of y that no place names are left as they are in ``out`` (the gradient of y), and undefined without one; a row that two places name, which route_rows never gives, has
    numbers of either's gradient and not their sum.  Without weights the gradient of y
    is ``take_rows(d_out, place)``."""
    lib, where, device = load_library(), "combine_rows_backward", y.device
    _require_no_gradient(where, d_out, y, weights, out)
    _check_rows(where, y, place, weights, None)
    _require(weights is not None, where, "weights")
    _require(_rows(d_out, y.dtype, device) and d_out.shape == (place.shape[0], y.shape[1]), where, "the gradient does not match")
    with _On(device, stream, where) as st:
        dy = _out(out, y, y.shape[0], y.shape[1], where)
        dw = weights.new_empty(place.shape)
        p = _row_sets(d_out, y, place, weights)
        p.d_sorted_gradient, p.ld_sorted_gradient, p.d_weights_gradient, p.ld_weights_gradient = dy.data_ptr(), dy.stride(0), dw.data_ptr(), dw.stride(0)
        code = lib.evo_combine_rows_backward(C.byref(p), st)
    _check(code, where)
    return dy, dw


def grouped_linear_backward(dy: torch.Tensor, x: Optional[torch.Tensor], weight: torch.Tensor, offsets: torch.Tensor, y: Optional[torch.Tensor] = None, *,
                            activation: str = "none", scale: float = 1.0, wanted: Tuple[bool, bool, bool] = (True, True, True),
                            shared_bias: bool = False, out: Sequence[Optional[torch.Tensor]] = (None, None, None),
                            stream: Optional[torch.cuda.Stream] = None) -> Tuple[Optional[torch.Tensor], ...]:
    """``evo_grouped_linear_backward``: the gradients (of x, of weight, of the bias) of ``y = grouped_linear(x, weight, offsets, bias, activation=...,
    scale=...)`` for the gradient ``dy`` of y; None where ``wanted`` says so.  y is needed with an activation, x for the gradient of weight.  Groups that share their weights (an
    expanded weight, stride 0) or, with ``shared_bias``, their bias have one gradient, [1, ...], the sum over all groups.  ``out`` may give any of the
    three a place, of any strides that keep rows apart: a layer's gradients inside rows like theta's.  Rows of x outside all groups are left as
    they are in ``out``, and undefined without one."""
    lib, where, device, dtype = load_library(), "grouped_linear_backward", dy.device, dy.dtype
    _require(len(wanted) == 3 and len(out) == 3, where, "wanted and out are for x, weight and bias")
    _require_no_gradient(where, dy, x, weight, y, *out)
    _require(dy.is_cuda and dtype in TYPES and _rows(dy, dtype, device), where, "dy: fp32, bf16 or fp16 rows on a GPU")
    _require(weight.device == device and weight.dtype == dtype and weight.dim() == 3, where, "weight does not match dy")
    groups, n_out, n_in = weight.shape
    rows = dy.shape[0]
    stride, pitch, one = weight.stride()
    _require(groups >= 1 and n_out >= 1 and n_in >= 1 and n_out == dy.shape[1] and (n_in == 1 or one == 1) and stride >= 0 and pitch >= 0, where,
             "weight does not match dy")
    _require(activation in ACTIVATIONS, where, "activation")
    _require((y is not None or activation == "none") and (y is None or (_rows(y, dtype, device) and y.shape == dy.shape)), where, "y does not match")
    _require((x is not None or not wanted[1]) and (x is None or (_rows(x, dtype, device) and x.shape == (rows, n_in))), where, "x does not match")
    wide = _ragged(offsets, groups, device, where)
    sets = [1 if groups > 1 and stride == 0 else groups, 1 if shared_bias else groups]
    with _On(device, stream, where) as st:
        dx = _out(out[0], dy, rows, n_in, where) if wanted[0] else None
        dweight, dbias = out[1] if wanted[1] else None, out[2] if wanted[2] else None
        if dweight is not None:
            _require(dweight.device == device and dweight.dtype == dtype and dweight.shape == (sets[0], n_out, n_in) and (n_in == 1 or dweight.stride(2) == 1), where,
                     "the gradient of weight does not match")
        elif wanted[1]:
            dweight = dy.new_empty((sets[0], n_out, n_in))
        if dbias is not None:
            _require(_rows(dbias, dtype, device) and dbias.shape == (sets[1], n_out), where, "the gradient of the bias does not match")
        elif wanted[2]:
            dbias = dy.new_empty((sets[1], n_out))
        no = (None, 0)
        f = Grouped(_GROUPED, TYPES[dtype], groups, n_in, n_out, ACTIVATIONS[activation], scale, wide, rows, *(no if x is None else (x.data_ptr(), x.stride(0))),
                    weight.data_ptr(), pitch if n_out > 1 else n_in, stride, None, 0, offsets.data_ptr(), *(no if y is None else (y.data_ptr(), y.stride(0))))
        apart, down = (0, 0) if dweight is None else dweight.stride()[:2]
        p = GroupedGradient(_GROUPED_GRADIENT, 1 if sets[0] < groups else 0, 1 if sets[1] < groups else 0, dy.data_ptr(), dy.stride(0),
                            *(no if dx is None else (dx.data_ptr(), dx.stride(0))), None if dweight is None else dweight.data_ptr(), down if n_out > 1 else n_in, apart,
                            *(no if dbias is None else (dbias.data_ptr(), dbias.stride(0))))
        need = C.c_size_t()
        _check(lib.evo_grouped_linear_backward_bytes(C.byref(f), C.byref(p), C.byref(need)), where)
        work = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
        code = lib.evo_grouped_linear_backward(C.byref(f), C.byref(p), None if work is None else work.data_ptr(), need.value, st)
    _check(code, where)
    return dx, dweight, dbias


class PolicyLoss(NamedTuple):
    loss: torch.Tensor
    logp: torch.Tensor
    gradient: Optional[torch.Tensor]


@lru_cache(maxsize=1024)
def _policy_bytes(rows: int) -> int:
    need, p = C.c_size_t(), PolicyRows(C.sizeof(PolicyRows), 0, 1, 0, rows)
    p.d_loss = 4
    _check(load_library().evo_policy_loss_bytes(C.byref(p), C.byref(need)), "policy_loss")
    return need.value


def policy_loss(logits: torch.Tensor, actions: torch.Tensor, old_logp: torch.Tensor, advantage: torch.Tensor, *, ref_logp: Optional[torch.Tensor] = None,
                weights: Optional[torch.Tensor] = None, clip: Tuple[float, float] = (0.2, 0.2), kl: float = 0.0, gradient: bool = True,
                out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> PolicyLoss:
    """``evo_policy_loss``: the clipped policy loss (to be minimised) of rows of ``logits`` [rows, n] (fp32, bf16 or fp16) with ``kl`` times the estimate
    ``exp(ref - logp) - (ref - logp) - 1`` of the divergence from a reference policy; its sum over the rows times ``weights`` (None: the mean), the log probability of every
    row's action, and the gradient of the logits (``gradient`` False: None; ``out`` may be ``logits``; for rows of logits inside wider ones, an ``out`` of the same pitch takes half
    the time or less).  ``clip``: how far a ratio may fall below and rise above 1.
    actions int32 or int64; old_logp, advantage, ref_logp and weights fp32, [rows].  A row whose action is outside [0, n) or whose weight is 0
    is padding.  Logits of minus infinity are forbidden actions."""
    lib, where, device = load_library(), "policy_loss", logits.device
    _require_no_gradient(where, logits, old_logp, advantage, ref_logp, weights, out)
    _require(logits.is_cuda and logits.dtype in TYPES and _rows(logits, logits.dtype, device) and logits.shape[1] >= 1, where,
             "logits: fp32, bf16 or fp16 rows on a GPU")
    rows, n = logits.shape
    _require(actions.device == device and actions.dtype in (torch.int32, torch.int64) and actions.shape == (rows,) and actions.is_contiguous(), where,
             "actions: int32 or int64, one a row")
    for x in (old_logp, advantage, ref_logp, weights):
        _require(x is None or (x.device == device and x.dtype == torch.float32 and x.shape == actions.shape and x.is_contiguous()), where,
                 "old_logp, advantage, ref_logp and weights: contiguous fp32, one a row")
    _require(old_logp is not None and advantage is not None and (ref_logp is not None or kl == 0.0), where, "old_logp, advantage or ref_logp is missing")
    _require(len(clip) == 2 and (out is None or gradient), where, "clip or out")
    with _On(device, stream, where) as st:
        d_logits = _out(out, logits, rows, n, where) if gradient else None
        loss, logp = old_logp.new_empty(()), old_logp.new_empty(rows)
        p = PolicyRows(C.sizeof(PolicyRows), TYPES[logits.dtype], n, 1 if actions.dtype == torch.int64 else 0, rows, clip[0], clip[1], kl,
                       logits.data_ptr(), logits.stride(0), actions.data_ptr(), old_logp.data_ptr(), advantage.data_ptr(),
                       None if ref_logp is None else ref_logp.data_ptr(), None if weights is None else weights.data_ptr(), loss.data_ptr(), logp.data_ptr())
        if d_logits is not None:
            p.d_gradient, p.ld_gradient = d_logits.data_ptr(), d_logits.stride(0)
        need = _policy_bytes(rows)
        work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        code = lib.evo_policy_loss(C.byref(p), None if work is None else work.data_ptr(), need, st)
    _check(code, where)
    return PolicyLoss(loss, logp, d_logits)
