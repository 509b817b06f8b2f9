"""Operators of a model's block around the sequences: residual addition with
dropout and norm, dropout, linear attention, log probabilities of given tokens.

As the rest of the binding this only marshals arguments (and checks the
shapes, which the C ABI cannot see); every step runs in the library's kernels.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import _check, _ptr, _stream, lib
from .sequence import CMat, Checkpoint, _device, _floats, _mat, _want


class CNorm(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("eps", ctypes.c_float), ("drop", ctypes.c_float),
                ("seed", ctypes.c_uint64), ("first_row", ctypes.c_int64)]


def _declare(L) -> None:
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    f32, u64 = ctypes.c_float, ctypes.c_uint64
    M, Nm = ctypes.POINTER(CMat), ctypes.POINTER(CNorm)
    for name, res, args in (
            ("emb_norm_fwd", i32, [i64, i32, Nm, M, M, M, M, M, vp]),
            ("emb_norm_workspace_size", sz, [i64, i32]),
            ("emb_norm_bwd", i32, [i64, i32, Nm, M, M, M, M, M, vp, i32, vp, sz, vp]),
            ("emb_dropout", i32, [i64, i32, f32, u64, i64, M, M, vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args


_SEED = (1 << 64) - 1


# ---------------------------------------------------------------- norm

class Norm:
    """Residual addition, dropout and root-mean-square norm (emb_norm_fwd), and
    its backward:

        total = residual + dropout(x)
        y = weight * total / sqrt(mean(total^2) + eps)

    ``weight`` is a contiguous fp32 vector on the GPU, the caller's.  ``drop``
    is the share dropped; its mask follows from the ``seed`` that a call gives,
    so the backward is given the forward's.  ``max_rows`` sizes the weight
    gradient's workspace (0: no weight gradient).  Calls with a weight gradient
    on one object must be ordered."""

    def __init__(self, weight, eps: float = 1e-6, drop: float = 0.0, max_rows: int = 0):
        import torch
        if weight.dim() != 1 or weight.numel() < 1:
            raise ValueError("weight is a vector")
        self.dim = int(weight.numel())
        self.weight = weight
        if not 0.0 <= drop < 1.0:
            raise ValueError("drop is a share below 1")
        if not 0.0 <= eps < float("inf"):
            raise ValueError("eps is a number of at least 0")
        self._at = _floats(weight, (self.dim,), "weight")
        self.max_rows = max_rows
        self._c = CNorm(self._at, eps, drop, 0, 0)
        self._ref = ctypes.byref(self._c)
        self.ws, self._ws, self._wsb = None, None, 0
        if max_rows > 0:
            self._wsb = int(lib().emb_norm_workspace_size(max_rows, self.dim))
            if self._wsb == 0:
                raise ValueError("rows too wide or too many for one call")
            self.ws = torch.empty(self._wsb, dtype=torch.uint8, device=weight.device)
            self._ws = self.ws.data_ptr()

    def _take(self, seed: int, first_row: int) -> None:
        c = self._c
        at = self.weight.data_ptr()
        if at != self._at:      # the tensor has got other memory
            self._at = c.weight = _floats(self.weight, (self.dim,), "weight")
        c.seed, c.first_row = seed & _SEED, first_row

    def forward(self, x, y=None, residual=None, total=None, saved: Optional[Checkpoint] = None, seed: int = 0,
                first_row: int = 0, stream=None) -> None:
        """y, and ``total`` (which the backward reads), and y in 8 bits in
        ``saved``; each may be left out, but not both forms of y."""
        x = _mat(x)
        n, D = x.rows, self.dim
        _want(x, n, D, "x")
        refs = []
        for m, name in ((residual, "residual"), (total, "total"), (y, "y")):
            if m is not None:
                m = _mat(m)
                _want(m, n, D, name)
            refs.append(m)
        if saved is not None:
            saved = _mat(saved.mat)
            _want(saved, n, D, "saved")
        refs.append(saved)
        self._take(seed, first_row)
        _check("emb_norm_fwd", lib().emb_norm_fwd(n, D, self._ref, x.ref,
                                                  *(m.ref if m is not None else None for m in refs), _stream(stream)))

    def backward(self, total, dy, dtotal=None, branch=None, arriving=None, dweight=None, add: bool = False,
                 seed: int = 0, first_row: int = 0, stream=None) -> None:
        """From dy and the gradient ``arriving`` at the total by its other uses
        (None: zero): ``dtotal``, which is the residual's gradient, ``branch``,
        that of x, and ``dweight`` (fp32), with ``add`` added to what is there."""
        total, dy = _mat(total), _mat(dy)
        n, D = total.rows, self.dim
        _want(total, n, D, "total")
        _want(dy, n, D, "dy")
        refs = []
        for m, name in ((arriving, "arriving"), (dtotal, "dtotal"), (branch, "branch")):
            if m is not None:
                m = _mat(m)
                _want(m, n, D, name)
            refs.append(m.ref if m is not None else None)
        if dweight is not None and n > self.max_rows:
            raise ValueError("batch larger than the norm's workspace")
        self._take(seed, first_row)
        _check("emb_norm_bwd", lib().emb_norm_bwd(
            n, D, self._ref, total.ref, dy.ref, *refs, _floats(dweight, (D,), "dweight"), int(add), self._ws,
            self._wsb, _stream(stream)))


def dropout(x, y, drop: float, seed: int, first_row: int = 0, stream=None) -> None:
    """y = x with a share ``drop`` of its values zeroed and the others scaled by
    1 / (1 - drop) (emb_dropout).  The mask is a function of the seed, the row's
    number (counted from ``first_row``) and the column, so the gradient is the
    same call on dy.  y may be x."""
    x, y = _mat(x), _mat(y)
    _want(y, x.rows, x.cols, "y")
    _check("emb_dropout", lib().emb_dropout(x.rows, x.cols, drop, seed & _SEED, first_row, x.ref, y.ref,
                                            _stream(stream)))
