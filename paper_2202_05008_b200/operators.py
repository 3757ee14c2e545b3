"""The matrix operators of ``include/evo.h``: calls on torch tensors that need no solver.

All of them enqueue their work on ``stream`` (the current stream of the tensors' device if it is None), allocate their
outputs and workspaces through torch on that stream, and return without waiting.  Where that is not the stream on which an argument
was made, ordering the two and keeping the argument until the work is done are the caller's.  Arguments that the library cannot
take raise ``EvoError``; there is no fallback.  None of them has a backward pass: while torch records gradients, tensors that require one are
refused (detach them, or call under ``torch.no_grad()``).
"""
from __future__ import annotations

import ctypes as C
import math
from functools import lru_cache
from typing import Optional, Sequence, Tuple

import torch

from .binding import EVO_MAX_LAYERS, Actions, EvoError, Grouped, Matrices, Matrix, Muon, NewtonSchulz, _check, load_library

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INVALID_ARG = 1
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


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # the handle without a Stream object (2 us)


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
        elif self.device.index != torch.cuda.current_device():
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
        return torch.empty((rows, cols), dtype=x.dtype, device=x.device)
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
