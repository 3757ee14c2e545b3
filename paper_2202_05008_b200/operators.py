"""The matrix operators of ``include/evo.h``: calls on torch tensors that need no solver.

All of them enqueue their work on ``stream`` (the current stream of the tensors' device if it is None), allocate their
outputs and workspaces through torch on that stream, and return without waiting.  Arguments that the library cannot
take raise ``EvoError``; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

import torch

from .binding import EvoError, Matrices, Matrix, Muon, NewtonSchulz, _check, load_library

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INVALID_ARG = 1
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
