"""The matrix operators of ``include/evo.h``: calls on torch tensors that need no solver.

All of them enqueue their work on ``stream`` (the current stream of the tensors' device if it is None), allocate their
outputs and workspaces through torch on that stream, and return without waiting.  Arguments that the library cannot
take raise ``EvoError``; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

import torch

from .binding import EVO_MAX_LAYERS, Actions, EvoError, Grouped, Matrices, Matrix, Muon, NewtonSchulz, _check, load_library

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INVALID_ARG = 1
ACTIVATIONS = {"none": 0, "tanh": 1, "relu": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _require(condition: bool, where: str, what: str) -> None:
    if not condition:
        error = EvoError(INVALID_ARG, where)
        error.args = (f"{error.args[0]}: {what}",)
        raise error


class _On:
    """The tensors' device, and the stream the call goes to, as the current ones (allocations belong to that stream)."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream]):
        self.guard = torch.cuda.device(device) if stream is None else torch.cuda.stream(stream)
        self.device = device
        self.stream = stream

    def __enter__(self) -> int:
        self.guard.__enter__()
        return (self.stream if self.stream is not None else torch.cuda.current_stream(self.device)).cuda_stream

    def __exit__(self, *exc):
        return self.guard.__exit__(*exc)


def _newton_schulz(steps: int, coefficients: Sequence[float], eps: float, where: str) -> NewtonSchulz:
    _require(1 <= steps <= 64 and len(coefficients) == 3 and any(coefficients) and eps > 0, where, "steps, coefficients or eps")
    return NewtonSchulz(C.sizeof(NewtonSchulz), steps, *coefficients, eps)


def _matrices(x: torch.Tensor) -> Matrices:
    batched = x.dim() == 3
    rows, cols = x.shape[-2:]
    # a stride that is never taken may be anything
    row_stride = x.stride(-2) if rows > 1 else cols
    batch = x.shape[0] if batched else 1
    return Matrices(x.data_ptr(), TYPES[x.dtype], batch, rows, cols, x.stride(0) if batch > 1 else rows * row_stride, row_stride)


def orthogonalize(x: torch.Tensor, out: Optional[torch.Tensor] = None, *, steps: int = 5,
                  coefficients: Sequence[float] = COEFFICIENTS, eps: float = 1e-7,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_orthogonalize``: every matrix of ``x`` ([rows, cols] or [batch, rows, cols]; fp32, bf16 or fp16; unit
    column stride) with its singular values moved towards 1 by Newton-Schulz steps.  ``out`` may be ``x``."""
    lib, where = load_library(), "orthogonalize"
    _require(x.is_cuda and x.dtype in TYPES and x.dim() in (2, 3), where, "a fp32, bf16 or fp16 matrix or batch on a GPU")
    _require(x.shape[-1] == 1 or x.stride(-1) == 1, where, "the columns of x need unit stride")
    with _On(x.device, stream) as st:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _require(out.device == x.device and out.dtype == x.dtype and out.shape == x.shape, where, "out must match x")
        _require(out.shape[-1] == 1 or out.stride(-1) == 1, where, "the columns of out need unit stride")
        if x.numel() == 0:
            return out
        ns = _newton_schulz(steps, coefficients, eps, where)
        a, b, need = _matrices(x), _matrices(out), C.c_size_t()
        _check(lib.evo_orthogonalize_bytes(a.batch, a.rows, a.cols, C.byref(need)), where)
        work = torch.empty(need.value, dtype=torch.uint8, device=x.device) if need.value else None
        _check(lib.evo_orthogonalize(C.byref(ns), C.byref(a), C.byref(b), None if work is None else work.data_ptr(), need.value, st),
               where)
    return out


def muon_step(center: torch.Tensor, m: torch.Tensor, v: torch.Tensor, gradient: torch.Tensor,
              matrices: Sequence[Tuple[int, int, int]], step: int, *, lr: float, momentum: float = 0.95,
              nesterov: bool = True, weight_decay: float = 0.0, ns_steps: int = 5,
              coefficients: Sequence[float] = COEFFICIENTS, eps: float = 1e-7, beta1: float = 0.9, beta2: float = 0.999,
              adam_eps: float = 1e-8, out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
              stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """``evo_muon_step`` on flat fp32 vectors; ``matrices`` lists (offset, rows, cols) of the weight matrices.  Returns
    the new (center, m, v); ``out=(center, m, v)`` takes the step in place."""
    lib, where = load_library(), "muon_step"
    vectors = (center, m, v, gradient) + (tuple(out) if out is not None else ())
    _require(len(vectors) in (4, 7), where, "out needs three vectors")
    for x in vectors:
        _require(x.is_cuda and x.device == center.device and x.dtype == torch.float32 and x.dim() == 1 and x.is_contiguous() and
                 x.numel() == center.numel(), where, "contiguous fp32 vectors of one length on one GPU")
    ns = _newton_schulz(ns_steps, coefficients, eps, where)
    cfg = Muon(C.sizeof(Muon), 0 if nesterov else 1, lr, momentum, weight_decay, beta1, beta2, adam_eps, ns)
    _require(all(o >= 0 and 1 <= r <= 1 << 20 and 1 <= c <= 1 << 20 for o, r, c in matrices) and step >= 1, where,
             "matrices are (offset, rows, cols), the step counts from 1")
    n, dim = len(matrices), center.numel()
    items = (Matrix * max(n, 1))(*(Matrix(o, r, c) for o, r, c in matrices))
    with _On(center.device, stream) as st:
        if out is None:
            out = (torch.empty_like(center), torch.empty_like(m), torch.empty_like(v))
        if dim == 0:
            return tuple(out)
        need = C.c_size_t()
        _check(lib.evo_muon_bytes(items, n, dim, C.byref(need)), where)
        work = torch.empty(need.value, dtype=torch.uint8, device=center.device) if need.value else None
        _check(lib.evo_muon_step(C.byref(cfg), items, n, dim, step, center.data_ptr(), m.data_ptr(), v.data_ptr(),
                                 gradient.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(),
                                 None if work is None else work.data_ptr(), need.value, st), where)
    return tuple(out)


def _rows(x: torch.Tensor, dtype: torch.dtype, like: torch.Tensor) -> bool:
    return x.is_cuda and x.device == like.device and x.dtype == dtype and x.dim() == 2 and (x.shape[1] <= 1 or x.stride(1) == 1)


def _ragged(offsets: torch.Tensor, groups: int, like: torch.Tensor, where: str) -> int:
    _require(offsets.device == like.device and offsets.dtype in (torch.int32, torch.int64) and offsets.dim() == 1 and
             offsets.numel() == groups + 1 and offsets.is_contiguous(), where, "offsets: int32 or int64 on the same GPU, one more than groups")
    return 1 if offsets.dtype == torch.int64 else 0


def _out(out: Optional[torch.Tensor], x: torch.Tensor, cols: int, where: str) -> torch.Tensor:
    if out is None:
        return torch.empty(x.shape[0], cols, dtype=x.dtype, device=x.device)
    _require(_rows(out, x.dtype, x) and out.shape == (x.shape[0], cols), where, "out does not match")
    return out


def grouped_linear(x: torch.Tensor, weight: torch.Tensor, offsets: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                   activation: str = "none", scale: float = 1.0, out: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_grouped_linear``: ``y[r] = scale * act(weight[g] @ x[r] + bias[g])`` for the rows ``offsets[g] <= r < offsets[g + 1]``.
    x [rows, n_in], weight [groups, n_out, n_in], bias [groups, n_out]; fp32, bf16 or fp16; unit stride in the last dimension, any
    other strides (a layer of theta is ``theta[:, a:b].unflatten(1, (n_out, n_in))``; an expanded weight is shared).  Rows outside all
    groups are left as they are in ``out``, and undefined without one."""
    lib, where = load_library(), "grouped_linear"
    _require(x.is_cuda and x.dtype in TYPES and _rows(x, x.dtype, x), where, "x: fp32, bf16 or fp16 rows on a GPU")
    _require(weight.device == x.device and weight.dtype == x.dtype and weight.dim() == 3 and weight.shape[0] >= 1 and
             weight.shape[2] == x.shape[1] and (weight.shape[2] <= 1 or weight.stride(2) == 1), where, "weight does not match x")
    groups, n_out, n_in = weight.shape
    _require(n_out >= 1 and n_in >= 1 and activation in ACTIVATIONS, where, "sizes or activation")
    _require(weight.stride(0) >= 0 and weight.stride(1) >= 0, where, "weight strides")
    if bias is not None:
        _require(_rows(bias, x.dtype, x) and bias.shape == (groups, n_out) and (n_out == 1 or bias.stride(1) == 1), where, "bias does not match")
    wide = _ragged(offsets, groups, x, where)
    with _On(x.device, stream) as st:
        y = _out(out, x, n_out, where)
        p = Grouped(C.sizeof(Grouped), TYPES[x.dtype], groups, n_in, n_out, ACTIVATIONS[activation], scale, wide, x.shape[0],
                    x.data_ptr(), x.stride(0), weight.data_ptr(), weight.stride(1) if n_out > 1 else n_in, weight.stride(0),
                    None if bias is None else bias.data_ptr(), 0 if bias is None else bias.stride(0), offsets.data_ptr(), y.data_ptr(),
                    y.stride(0))
        _check(lib.evo_grouped_linear(C.byref(p), st), where)
    return y


def mlp_actions(theta: torch.Tensor, layer_sizes: Sequence[int], observations: torch.Tensor, offsets: torch.Tensor, *,
                action_scale: float = 1.0, out: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``evo_mlp_actions``: the MLP policy's actions for rows of observations, ``offsets[m] <= r < offsets[m + 1]`` being member m's.
    theta [members, >= parameters] fp32 as ``Solver.ask`` returns it (row pitch a multiple of 4, rows 16-byte aligned),
    layer_sizes the widths, input first.  Rows without a member are left as they are in ``out``, and undefined without one."""
    lib, where = load_library(), "mlp_actions"
    sizes = tuple(layer_sizes)
    _require(2 <= len(sizes) <= EVO_MAX_LAYERS + 1 and min(sizes) >= 1, where, "layer_sizes")
    _require(observations.is_cuda and _rows(observations, torch.float32, observations) and observations.shape[1] == sizes[0], where,
             "observations: fp32 rows of the first layer's width on a GPU")
    dim = sum((a + 1) * b for a, b in zip(sizes[:-1], sizes[1:]))
    _require(_rows(theta, torch.float32, observations) and theta.shape[0] >= 1 and theta.shape[1] >= dim, where, "theta does not match")
    members = theta.shape[0]
    wide = _ragged(offsets, members, observations, where)
    with _On(observations.device, stream) as st:
        y = _out(out, observations, sizes[-1], where)
        pitch = theta.stride(0) if members > 1 else -(-max(dim, theta.stride(0)) // 4) * 4
        p = Actions(C.sizeof(Actions), members, len(sizes) - 1, (C.c_uint32 * (EVO_MAX_LAYERS + 1))(*sizes), action_scale, wide,
                    observations.shape[0], theta.data_ptr(), pitch, observations.data_ptr(), observations.stride(0), offsets.data_ptr(),
                    y.data_ptr(), y.stride(0))
        need = C.c_size_t()
        _check(lib.evo_mlp_actions_bytes(C.byref(p), C.byref(need)), where)
        work = torch.empty(need.value, dtype=torch.uint8, device=observations.device) if need.value else None
        _check(lib.evo_mlp_actions(C.byref(p), None if work is None else work.data_ptr(), need.value, st), where)
    return y
