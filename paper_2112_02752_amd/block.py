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


class CHeads(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int64), ("num_seqs", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("dk", ctypes.c_int32), ("dv", ctypes.c_int32),
                ("offsets", ctypes.c_void_p), ("q", CMat), ("k", CMat), ("v", CMat), ("decay", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("first", ctypes.c_void_p)]


def _declare(L) -> None:
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    f32, u64 = ctypes.c_float, ctypes.c_uint64
    M, Nm, H = ctypes.POINTER(CMat), ctypes.POINTER(CNorm), ctypes.POINTER(CHeads)
    for name, res, args in (
            ("emb_norm_fwd", i32, [i64, i32, Nm, M, M, M, M, M, vp]),
            ("emb_norm_workspace_size", sz, [i64, i32]),
            ("emb_norm_bwd", i32, [i64, i32, Nm, M, M, M, M, M, vp, i32, vp, sz, vp]),
            ("emb_dropout", i32, [i64, i32, f32, u64, i64, M, M, vp]),
            ("emb_linear_states_size", sz, [i64, i32, i32, i32]),
            ("emb_linear_fwd", i32, [H, M, vp, vp, sz, vp]),
            ("emb_linear_bwd", i32, [H, vp, sz, M, M, M, M, vp, vp, vp, sz, vp]),
            ("emb_linear_step", i32, [i64, i32, i32, i32, i32, M, M, M, vp, f32, vp, i64, vp, M, vp]),
            ("emb_logp_fwd", i32, [i64, i32, M, vp, i32, f32, vp, vp, i32, vp, vp, vp, vp]),
            ("emb_logp_bwd", i32, [i64, i32, M, vp, i32, f32, vp, vp, vp, M, vp]),
            ("emb_logp_train", i32, [i64, i32, M, vp, i32, f32, vp, vp, vp, M, vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args


_SEED = (1 << 64) - 1


_ask_device = None


def _device_now() -> int:
    """The current device (where PyTorch offers it, without what its Python call adds)."""
    global _ask_device
    if _ask_device is None:
        import torch
        torch.cuda.current_device()     # initialises
        _ask_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _ask_device()


def _here(mats, tensors) -> None:
    """A call runs on the current device: its matrices and vectors (None: left
    out) have to lie there."""
    now = _device_now()
    for m in mats:
        if m is not None and m.device != now:
            raise ValueError("matrices lie on the current device (torch.cuda.device chooses it)")
    for t in tensors:
        if t is not None and t.get_device() != now:
            raise ValueError("tensors lie on the current device (torch.cuda.device chooses it)")


# ---------------------------------------------------------------- norm

class Norm:
    """Residual addition, dropout and root-mean-square norm (emb_norm_fwd), and
    its backward:

        total = residual + dropout(x)
        y = weight * total / sqrt(mean(total^2) + eps)

    ``weight`` is a contiguous fp32 vector on the GPU, the caller's.  ``drop``
    is the share dropped; its mask follows from the ``seed`` that a call gives,
    so the backward is given the forward's (and a captured call keeps the one it
    was captured with).  ``max_rows`` sizes the weight
    gradient's workspace (0: no weight gradient).  Calls with a weight gradient
    on one object must be ordered; others need not be, nor come from one thread."""

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
        self.eps, self.drop, self.max_rows = eps, drop, max_rows
        self.ws, self._ws, self._wsb = None, None, 0
        if max_rows > 0:
            self._wsb = int(lib().emb_norm_workspace_size(max_rows, self.dim))
            if self._wsb == 0:
                raise ValueError("rows too wide or too many for one call")
            self.ws = torch.empty(self._wsb, dtype=torch.uint8, device=weight.device)
            self._ws = self.ws.data_ptr()

    def _call(self, seed: int, first_row: int):
        """A call's descriptor: its own, for another thread's call may come before this one has read it."""
        at = self.weight.data_ptr()
        if at != self._at:      # the tensor has got other memory
            at = self._at = _floats(self.weight, (self.dim,), "weight")
        return ctypes.byref(CNorm(at, self.eps, self.drop, seed & _SEED, first_row))

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
        _here((x, *refs), (self.weight,))
        _check("emb_norm_fwd", lib().emb_norm_fwd(n, D, self._call(seed, first_row), x.ref,
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
        mats = []
        for m, name in ((arriving, "arriving"), (dtotal, "dtotal"), (branch, "branch")):
            if m is not None:
                m = _mat(m)
                _want(m, n, D, name)
            mats.append(m)
        _here((total, dy, *mats), (self.weight, dweight, self.ws))
        if dweight is not None and n > self.max_rows:
            raise ValueError("batch larger than the norm's workspace")
        _check("emb_norm_bwd", lib().emb_norm_bwd(
            n, D, self._call(seed, first_row), total.ref, dy.ref, *(m.ref if m is not None else None for m in mats),
            _floats(dweight, (D,), "dweight"), int(add), self._ws, self._wsb, _stream(stream)))


def dropout(x, y, drop: float, seed: int, first_row: int = 0, stream=None) -> None:
    """y = x with a share ``drop`` of its values zeroed and the others scaled by
    1 / (1 - drop) (emb_dropout).  The mask is a function of the seed, the row's
    number (counted from ``first_row``) and the column, so the gradient is the
    same call on dy.  y may be x."""
    x, y = _mat(x), _mat(y)
    _want(y, x.rows, x.cols, "y")
    _here((x, y), ())
    _check("emb_dropout", lib().emb_dropout(x.rows, x.cols, drop, seed & _SEED, first_row, x.ref, y.ref,
                                            _stream(stream)))


# ---------------------------------------------------------------- linear attention

def _head_widths(q, k, v, heads: int, groups: int):
    """Widths of the heads, from the matrices' columns."""
    if groups < 1 or heads < 1 or heads % groups != 0:
        raise ValueError("heads are a multiple of groups")
    if k.cols % groups != 0 or v.cols % groups != 0 or k.cols == 0 or v.cols == 0:
        raise ValueError("keys and values have whole heads")
    dk, dv = k.cols // groups, v.cols // groups
    _want(q, k.rows, heads * dk, "q")
    _want(v, k.rows, groups * dv, "v")
    return dk, dv


class Heads:
    """The inputs of linear attention over ragged sequences (see emb_heads):
    int32 offsets [M + 1] on the GPU, queries of ``heads`` heads, keys and values
    of ``groups``, of one type, an fp32 decay for every key head and first
    states [M][groups][dk][dv] or None."""

    def __init__(self, offsets, q, k, v, decay, heads: int, groups: Optional[int] = None, scale: float = 1.0,
                 first=None):
        import torch
        if offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous():
            raise ValueError("offsets are a contiguous int32 vector")
        _device(offsets, "offsets")
        self.heads, self.groups = heads, heads if groups is None else groups
        self.q, self.k, self.v = _mat(q), _mat(k), _mat(v)
        self.offsets, self.decay, self.scale, self.first = offsets, decay, scale, first
        self._c = CHeads()
        self.ref = ctypes.byref(self._c)
        self._key = None
        self.c()

    def c(self) -> CHeads:
        """The C descriptor; made again if a tensor has got other memory."""
        q, k, v, first = self.q, self.k, self.v, self.first
        key = (self.offsets.data_ptr(), self.offsets.numel(), q.tensor.data_ptr(), k.tensor.data_ptr(),
               v.tensor.data_ptr(), self.decay.data_ptr(), first.data_ptr() if first is not None else 0)
        if key != self._key:
            for m in (q, k, v):
                m.c()
            self.tokens, self.seqs = k.rows, key[1] - 1
            self.dk, self.dv = _head_widths(q, k, v, self.heads, self.groups)
            self.states = (self.seqs, self.groups, self.dk, self.dv)
            c = self._c
            c.num_tokens, c.num_seqs, c.heads, c.groups = self.tokens, self.seqs, self.heads, self.groups
            c.dk, c.dv, c.offsets, c.scale = self.dk, self.dv, key[0], self.scale
            c.q, c.k, c.v = q._c, k._c, v._c
            c.decay = _floats(self.decay, (self.groups,), "decay")
            c.first = _floats(first, self.states, "first")
            self._key = key
        return self._c


class LinearAttention:
    """Linear attention with a decay for each key head, with its workspace, for
    batches of up to ``max_tokens`` tokens (no buffer depends on the number of
    sequences: ``max_seqs`` is not looked at); with ``train`` there is room for
    the backward of the last forward's batch, which reads the states that the
    forward left here.  Calls on one object must be ordered."""

    def __init__(self, max_tokens: int, max_seqs: int, heads: int, groups: int, dk: int, dv: int, device="cuda",
                 train: bool = True):
        import torch
        if heads < 1 or groups < 1 or heads % groups != 0 or dk < 1 or dv < 1:
            raise ValueError("heads are a multiple of groups, and of at least one column")
        self.max_tokens, self.max_seqs = max_tokens, max_seqs
        self.heads, self.groups, self.dk, self.dv = heads, groups, dk, dv
        size = int(lib().emb_linear_states_size(max_tokens, groups, dk, dv))
        new = lambda: _device(torch.empty(max(size, 256), dtype=torch.uint8, device=device),  # noqa: E731
                              "a linear attention's workspace")
        self.states = new()
        self.ws = new() if train else None
        self._states, self._ws, self._size = self.states.data_ptr(), _ptr(self.ws), max(size, 256)
        self._tokens = None

    def _take(self, heads: Heads):
        heads.c()
        if heads.tokens > self.max_tokens or (heads.heads, heads.groups, heads.dk, heads.dv) != (
                self.heads, self.groups, self.dk, self.dv):
            raise ValueError("batch larger than the linear attention's buffers, or of other heads")
        return heads.ref

    def forward(self, heads: Heads, y, last=None, stream=None) -> None:
        """y (N x heads * dv), and the state after each sequence into ``last``
        (fp32 [M][groups][dk][dv])."""
        ref = self._take(heads)
        y = _mat(y)
        _want(y, heads.tokens, self.heads * self.dv, "y")
        _here((heads.q, heads.k, heads.v, y), (heads.offsets, heads.decay, heads.first, last, self.states))
        self._tokens = None
        _check("emb_linear_fwd", lib().emb_linear_fwd(ref, y.ref, _floats(last, heads.states, "last"), self._states,
                                                      self._size, _stream(stream)))
        self._tokens = heads.tokens, heads.seqs

    def backward(self, heads: Heads, dy, dq, dk, dv, dlast=None, dfirst=None, stream=None) -> None:
        """Gradients of the last forward, whose inputs these are: of the
        queries, keys, values and first states, from those of y and of the last
        states."""
        ref = self._take(heads)
        if self.ws is None or self._tokens != (heads.tokens, heads.seqs):
            raise ValueError("backward follows the forward of the same batch on an object made with train")
        mats = [_mat(m) for m in (dy, dq, dk, dv)]
        for m, cols, name in zip(mats, (self.heads * self.dv, self.heads * self.dk, self.groups * self.dk,
                                        self.groups * self.dv), ("dy", "dq", "dk", "dv")):
            _want(m, heads.tokens, cols, name)
        _here((heads.q, heads.k, heads.v, *mats),
              (heads.offsets, heads.decay, heads.first, dlast, dfirst, self.states, self.ws))
        _check("emb_linear_bwd", lib().emb_linear_bwd(
            ref, self._states, self._size, *(m.ref for m in mats), _floats(dlast, heads.states, "dlast"),
            _floats(dfirst, heads.states, "dfirst"), self._ws, self._size, _stream(stream)))


def linear_attention_step(q, k, v, decay, state, y, heads: int, groups: Optional[int] = None, scale: float = 1.0,
                          slots=None, stream=None) -> None:
    """One token of each running sequence (emb_linear_step): row i of q, k, v
    and y belongs to ``state[slots[i]]`` (fp32 [slots][groups][dk][dv], updated in
    place; ``slots`` int32, None: row i); tokens whose slot is no row of
    ``state`` get zeros."""
    q, k, v, y = _mat(q), _mat(k), _mat(v), _mat(y)
    groups = heads if groups is None else groups
    dk, dv = _head_widths(q, k, v, heads, groups)
    n = k.rows
    _want(y, n, heads * dv, "y")
    _here((q, k, v, y), (decay, state, slots))
    rows = int(state.shape[0])
    sp = None
    if slots is not None:
        if slots.numel() != n or slots.element_size() != 4 or slots.is_floating_point() or not slots.is_contiguous():
            raise ValueError("slots are a contiguous int32 vector, one a token")
        sp = _device(slots, "slots").data_ptr()
    elif n > rows:
        raise ValueError("more tokens than states")
    _check("emb_linear_step", lib().emb_linear_step(
        n, heads, groups, dk, dv, q.ref, k.ref, v.ref, _floats(decay, (groups,), "decay"), scale,
        _floats(state, (rows, groups, dk, dv), "state"), rows, sp, y.ref, _stream(stream)))


# ---------------------------------------------------------------- answers

MAX_TOP = 32        # EMB_MAX_TOP


def _ids(ids, n: int):
    """Address and bytes of a value of a contiguous int32 or int64 vector of n ids."""
    if ids.dim() != 1 or ids.numel() != n or ids.is_floating_point() or ids.element_size() not in (4, 8) \
            or not ids.is_contiguous():
        raise ValueError(f"ids are a contiguous int32 or int64 vector of {n} values")
    if not ids.is_cuda:
        _device(ids, "ids")
    return ids.data_ptr(), ids.element_size()


class LogProbs:
    """Log probabilities of given tokens under softmax(scale * logits), with the
    entropy, the ``top`` likeliest tokens and the logits' gradient
    (emb_logp_fwd), for up to ``max_rows`` rows of ``cols`` logits.  An id outside
    the columns (usually -1) stands for no token.  ``forward`` leaves what
    ``backward`` needs of each row here; ``train`` does both in one pass where
    the gradient of the log probabilities is known before.  Calls of ``forward``
    and ``backward`` on one object must be ordered."""

    def __init__(self, max_rows: int, cols: int, top: int = 0, scale: float = 1.0, device="cuda"):
        import torch
        if cols < 1 or not 0 <= top <= min(cols, MAX_TOP):
            raise ValueError(f"top is at most {MAX_TOP} and the number of columns")
        if not 0.0 < scale < float("inf"):
            raise ValueError("scale is above zero")
        self.max_rows, self.cols, self.top, self.scale = max_rows, cols, top, scale
        self.stats = _device(torch.empty((max(1, max_rows), 4), device=device), "a row's statistics")
        self._stats = self.stats.data_ptr()
        self._rows = None

    def _take(self, logits, ids, *tensors):
        logits = _mat(logits)
        n = logits.rows
        _want(logits, n, self.cols, "logits")
        if n > self.max_rows:
            raise ValueError("more rows than there is room for")
        _here((logits,), (ids, self.stats) + tensors)
        return (logits, n) + (_ids(ids, n) if ids is not None else (None, 4))

    def forward(self, logits, ids, logp, entropy=None, top_ids=None, top_logp=None, stream=None) -> None:
        """``logp`` and ``entropy`` (fp32 [rows], each may be None, ``ids`` with
        ``logp``), ``top_ids`` (int32) and ``top_logp`` (fp32) [rows][top]."""
        import torch
        logits, n, at, size = self._take(logits, ids, logp, entropy, top_ids, top_logp)
        tops = (n, self.top)
        if self.top > 0:
            if top_ids is None or top_logp is None:
                raise ValueError("top alternatives want top_ids and top_logp")
            if top_ids.shape != tops or top_ids.dtype != torch.int32 or not top_ids.is_contiguous():
                raise ValueError(f"top_ids is a contiguous int32 tensor of shape {tops}")
            _device(top_ids, "top_ids")
        lp, tl = _floats(logp, (n,), "logp"), _floats(top_logp, tops, "top_logp") if self.top > 0 else None
        self._rows = None
        _check("emb_logp_fwd", lib().emb_logp_fwd(
            n, self.cols, logits.ref, at, size, self.scale, lp, _floats(entropy, (n,), "entropy"), self.top,
            _ptr(top_ids) if self.top > 0 else None, tl, self._stats, _stream(stream)))
        self._rows = n

    def backward(self, logits, ids, dlogp, dlogits, dentropy=None, stream=None) -> None:
        """``dlogits`` from the gradients of the last forward's ``logp`` and
        ``entropy`` (each may be None, ``ids`` with ``dlogp``); ``dlogits`` may be
        ``logits``."""
        logits, n, at, size = self._take(logits, ids, dlogp, dentropy)
        if self._rows != n:
            raise ValueError("backward follows the forward of the same rows")
        dlogits = _mat(dlogits)
        _want(dlogits, n, self.cols, "dlogits")
        _here((dlogits,), ())
        _check("emb_logp_bwd", lib().emb_logp_bwd(
            n, self.cols, logits.ref, at, size, self.scale, self._stats, _floats(dlogp, (n,), "dlogp"),
            _floats(dentropy, (n,), "dentropy"), dlogits.ref, _stream(stream)))

    def train(self, logits, ids, logp, dlogp, dlogits, entropy=None, stream=None) -> None:
        """``logp`` (and ``entropy``; each may be None) and the gradient of
        sum(dlogp * logp) in ``dlogits``, which may be ``logits``."""
        logits, n, at, size = self._take(logits, ids, logp, dlogp, entropy)
        dlogits = _mat(dlogits)
        _want(dlogits, n, self.cols, "dlogits")
        _here((dlogits,), ())
        _check("emb_logp_train", lib().emb_logp_train(
            n, self.cols, logits.ref, at, size, self.scale, _floats(dlogp, (n,), "dlogp"), _floats(logp, (n,), "logp"),
            _floats(entropy, (n,), "entropy"), dlogits.ref, _stream(stream)))
