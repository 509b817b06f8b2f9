"""Sequences of tokens over the layer's tables: lookup of single tokens with
the gradient by sorted tokens, a gated linear recurrence, activations kept in
8 bits, and the layer that runs them together.

As the rest of the binding this only marshals arguments (and checks the
shapes, which the C ABI cannot see); every step runs in the library's kernels.
The projections of ``SequenceLayer`` are plain matrix products of PyTorch's.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import (BF16, FP32, Batch, CUpdate, DedupBuffers, StepFailed, Tables, _check, _ptr, _stream, _update, lib,
               read_status, workspace_init)

SAVED8 = 2
SPAN = 64           # EMB_SCAN_SPAN: positions between kept states
GROUP = 32          # EMB_SAVED_GROUP: columns that share an exponent
LAYOUT = {"rows": 0, "table": 1, "table_add": 2}


class CMat(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("exps", ctypes.c_void_p), ("ld_exps", ctypes.c_int64)]


class CToken(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("pad_row", ctypes.c_int64)]


class CScan(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int64), ("num_seqs", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("offsets", ctypes.c_void_p), ("x", CMat), ("f", CMat), ("o", CMat), ("bias", ctypes.c_void_p),
                ("h0", ctypes.c_void_p)]


def _declare(L) -> None:
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    from . import CBatch, CTables
    T, B, Up = ctypes.POINTER(CTables), ctypes.POINTER(CBatch), ctypes.POINTER(CUpdate)
    M, Tok, S = ctypes.POINTER(CMat), ctypes.POINTER(CToken), ctypes.POINTER(CScan)
    for name, res, args in (
            ("emb_token_fwd", i32, [T, B, Tok, M, vp]),
            ("emb_token_grad", i32, [T, B, Tok, M, vp, vp, vp, vp, vp, i32, Up, vp, sz, vp]),
            ("emb_scan_workspace_size", sz, [i64, i32]),
            ("emb_scan_fwd", i32, [S, M, vp, vp, vp, sz, vp]),
            ("emb_scan_bwd", i32, [S, vp, M, vp, M, M, M, vp, vp, vp, sz, vp]),
            ("emb_scan_step", i32, [i64, i32, M, M, M, vp, vp, i64, vp, M, vp]),
            ("emb_save", i32, [i64, i32, M, M, vp]),
            ("emb_restore", i32, [i64, i32, M, M, vp]),
            ("emb_weight_grad_workspace_size", sz, [i64, i32, i32]),
            ("emb_weight_grad", i32, [i64, i32, i32, M, M, vp, i32, vp, sz, vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args


def _device(t, what: str):
    if not t.is_cuda:
        raise ValueError(f"{what} must lie on the GPU")
    return t


class Mat:
    """A matrix of activations as the C ABI takes it: a 2-d fp32 or bf16
    tensor whose columns are contiguous, rows at any stride (a slice of a wider
    tensor's columns, or ``cols`` of them from column ``first`` on); an 8-bit one
    comes from ``Checkpoint.columns``.  Kept by a program between calls, it
    costs a call one address check."""

    __slots__ = ("tensor", "exps", "rows", "cols", "_c", "_at", "_at_exps", "_fixed", "_first", "ref")

    def __init__(self, tensor, exps=None, cols: Optional[int] = None, first: int = 0):
        self.tensor, self.exps, self._fixed, self._first = tensor, exps, cols, first
        self._c = CMat()
        self.ref = ctypes.byref(self._c)
        self._take()

    def _take(self) -> None:
        import torch
        tensor, exps = self.tensor, self.exps
        if tensor.dim() != 2 or (tensor.shape[1] > 1 and tensor.stride(1) != 1):
            raise ValueError("a matrix has two dimensions and contiguous columns")
        _device(tensor, "a matrix")
        rows, wide = int(tensor.shape[0]), int(tensor.shape[1])
        ld = int(tensor.stride(0)) if rows > 1 else max(int(tensor.stride(0)), wide)
        if exps is not None:
            if tensor.dtype != torch.int8 or exps.dtype != torch.uint8:
                raise ValueError("a checkpoint holds int8 codes and uint8 exponents")
            dtype, le = SAVED8, int(exps.stride(0)) if rows > 1 else int(exps.shape[1])
        else:
            if tensor.dtype not in (torch.float32, torch.bfloat16):
                raise ValueError("a matrix is fp32 or bf16")
            dtype, le = BF16 if tensor.dtype == torch.bfloat16 else FP32, 0
        if ld < wide:
            raise ValueError("rows overlap")
        first, cols = self._first, self._fixed
        if first < 0 or (cols is not None and (cols < 0 or first + cols > wide)) or first > wide:
            raise ValueError(f"columns {first} on of {wide}")
        self.rows, self.cols = rows, wide - first if cols is None else cols
        at = self._at = tensor.data_ptr()
        self._at_exps = exps.data_ptr() if exps is not None else None
        c = self._c
        c.ld, c.dtype, c.ld_exps = ld, dtype, le
        c.data = at + first * (1 if exps is not None else 4 if dtype == FP32 else 2) if at else None
        c.exps = self._at_exps + first // GROUP if self._at_exps else None

    @property
    def dtype(self) -> int:
        return self._c.dtype

    def c(self) -> CMat:
        """The C descriptor; made again if a tensor has got other memory."""
        if self.tensor.data_ptr() != self._at or (self.exps is not None and self.exps.data_ptr() != self._at_exps):
            self._take()
        return self._c


def _mat(m) -> Mat:
    if not isinstance(m, Mat):
        return Mat(m)
    m.c()
    return m


def _want(m: Mat, rows: int, cols: int, what: str) -> None:
    if m.rows != rows or m.cols != cols:
        raise ValueError(f"{what} has {m.rows} x {m.cols} values, {rows} x {cols} are wanted")


def _floats(t, shape, what: str) -> Optional[int]:
    """Address of a contiguous fp32 tensor of this shape, or None."""
    if t is None:
        return None
    if t.shape != shape or t.element_size() != 4 or not t.is_floating_point() or not t.is_contiguous():
        raise ValueError(f"{what} is a contiguous fp32 tensor of shape {shape}")
    if not t.is_cuda:
        _device(t, what)
    return t.data_ptr()


# ---------------------------------------------------------------- tokens

def _check_state(opt: Optional[str], state, rows: int, dim: int) -> None:
    """Refuse accumulators that the kernels would read or write past, or whose
    values are no fp32: one a row ("adagrad") or one a value ("adagrad_ew")."""
    if state is None or opt not in ("adagrad", "adagrad_ew"):
        return
    per = dim if opt == "adagrad_ew" else 1
    flat = state.dim() == 1 or (state.dim() > 1 and state.numel() == state.shape[0] * per)
    if not flat or state.numel() < rows * per or state.element_size() != 4 or not state.is_floating_point() \
            or not state.is_contiguous() or (per == 1 and state.numel() != state.shape[0]):
        raise ValueError(f"state is a contiguous fp32 tensor of {rows}{f' x {dim}' if per > 1 else ''} accumulators")
    _device(state, "state")


def token_fwd(tables: Tables, batch: Batch, out, scale: float = 1.0, pad_row: int = -1, stream=None) -> None:
    """out[j] = scale * W[key(j)] for every token of the batch's sequences
    (emb_token_fwd); zeros for tokens of the global row ``pad_row``."""
    out = _mat(out)
    _want(out, int(batch.indices.numel()), int(tables.weights.shape[1]), "out")
    tok = CToken(scale, pad_row)
    _check("emb_token_fwd", lib().emb_token_fwd(ctypes.byref(tables.c()), ctypes.byref(batch.c()), ctypes.byref(tok),
                                                out.ref, _stream(stream)))


def token_grad(tables: Tables, batch: Batch, grad_out, dedup: DedupBuffers, grad=None, layout: str = "rows",
               scale: float = 1.0, pad_row: int = -1, opt: Optional[str] = None, lr: float = 0.0, eps: float = 0.0,
               state=None, rounding: str = "nearest", seed: int = 0, stream=None) -> None:
    """Gradient of ``token_fwd`` by sorted tokens (emb_token_grad), after
    ``unique_ids`` of the same batch into ``dedup``: gradient rows in ``grad``
    as ``layout`` says, or with ``opt`` the optimizer step."""
    grad_out = _mat(grad_out)
    n, D = int(batch.indices.numel()), int(tables.weights.shape[1])
    _want(grad_out, n, D, "grad_out")
    if grad is not None:
        rows = n if layout == "rows" else int(tables.row_offset[-1])
        if int(grad.shape[0]) < rows:
            raise ValueError("grad has too few rows")
        _floats(grad, (int(grad.shape[0]), D), "grad")
    _check_state(opt, state, int(tables.row_offset[-1]), D)
    tok = CToken(scale, pad_row)
    upd = ctypes.byref(_update(opt, lr, eps, state, rounding, seed)) if opt is not None else None
    d = dedup
    _check("emb_token_grad", lib().emb_token_grad(
        ctypes.byref(tables.c()), ctypes.byref(batch.c()), ctypes.byref(tok), grad_out.ref, _ptr(d.sort_perm),
        _ptr(d.seg_offsets), _ptr(d.unique_keys), _ptr(d.num_unique), _ptr(grad), LAYOUT[layout], upd, _ptr(d.ws),
        d.ws.numel(), _stream(stream)))


def _check_status(ws, stream) -> None:
    st = read_status(ws, stream)
    if st[0]:
        raise StepFailed(*st)


class TokenLayer:
    """Lookup of single tokens from the tables, scaled, with its backward:
    the table's gradient or the optimizer step on the rows that were looked up.
    ``pad_row`` (a global row, or -1) stands for padding: it gives zeros and is
    never trained.  ``max_tokens`` sizes the dedup of the backward (0: a layer
    that only looks up).  Calls on one layer must be ordered."""

    def __init__(self, tables: Tables, scale: float = 1.0, pad_row: int = -1, opt: Optional[str] = None,
                 lr: float = 0.0, eps: float = 1e-8, state=None, max_tokens: int = 0, max_seqs: int = 0,
                 rounding: str = "nearest", seed: int = 0):
        self.tables, self.opt = tables, opt
        self.dim = int(tables.weights.shape[1])
        self._rows = int(tables.row_offset[-1])
        self._tok = CToken(scale, pad_row)
        self._tokp = ctypes.byref(self._tok)
        self.max_tokens = max_tokens
        self.seed, self.steps_done = seed, 0
        self.dedup = None
        if max_tokens > 0:
            d = self.dedup = DedupBuffers(tables.weights.device, max_tokens, max_seqs, self.dim)
            self._dd = tuple(_ptr(t) for t in (d.unique_keys, d.counts, d.seg_offsets, d.sort_perm, d.num_unique,
                                               d.ws)) + (d.ws.numel(),)
        self._upd = None
        if opt is not None:
            _check_state(opt, state, self._rows, self.dim)
            self._updc = _update(opt, lr, eps, state, rounding, seed)
            self._upd = ctypes.byref(self._updc)
            self._state, self._state_at = state, _ptr(state)

    def forward(self, batch: Batch, out, stream=None) -> None:
        out = _mat(out)
        _want(out, batch.indices.numel(), self.dim, "out")
        _check("emb_token_fwd", lib().emb_token_fwd(ctypes.byref(self.tables.c()), ctypes.byref(batch.c()),
                                                    self._tokp, out.ref, _stream(stream)))

    def _backward(self, batch: Batch, grad_out, grad, layout: int, upd, stream) -> None:
        n = batch.indices.numel()
        if n > self.max_tokens:
            raise ValueError("batch larger than the layer's buffers")
        if self.dedup is None:
            raise ValueError("a layer without max_tokens only looks up")
        g = _mat(grad_out)
        _want(g, n, self.dim, "grad_out")
        L, s = lib(), _stream(stream)
        uk, cnt, seg, perm, nu, ws, wsb = self._dd
        ct, cb = ctypes.byref(self.tables.c()), ctypes.byref(batch.c())
        _check("emb_unique_ids", L.emb_unique_ids(ct, cb, uk, cnt, seg, perm, nu, ws, wsb, s))
        _check("emb_token_grad", L.emb_token_grad(ct, cb, self._tokp, g.ref, perm, seg, uk, nu, grad, layout, upd, ws,
                                                  wsb, s))

    def table_grad(self, batch: Batch, grad_out, grad, add: bool = False, stream=None) -> None:
        """The gradient of every row of the tables into ``grad`` (fp32, rows x
        dim): written, or with ``add`` added to what is there."""
        self._backward(batch, grad_out, _floats(grad, (self._rows, self.dim), "grad"),
                       LAYOUT["table_add" if add else "table"], None, stream)

    def row_grads(self, batch: Batch, grad_out, grad_rows, stream=None) -> None:
        """Gradient rows of the batch's distinct tokens (``dedup.unique_keys``,
        ``dedup.num_unique``) into ``grad_rows`` (fp32, at least a row a token)."""
        if int(grad_rows.shape[0]) < batch.indices.numel():
            raise ValueError("grad_rows has too few rows")
        self._backward(batch, grad_out, _floats(grad_rows, (int(grad_rows.shape[0]), self.dim), "grad_rows"),
                       LAYOUT["rows"], None, stream)

    def _can_update(self) -> None:
        if self._upd is None:
            raise ValueError("a layer without an optimizer cannot update")
        if self.opt != "sgd" and self._state is None:
            raise ValueError(f"{self.opt} needs its accumulators as state")
        if _ptr(self._state) != self._state_at:     # the tensor has got other memory
            _check_state(self.opt, self._state, self._rows, self.dim)
            self._updc.state = self._state_at = _ptr(self._state)

    def update(self, batch: Batch, grad_out, stream=None) -> None:
        """The optimizer step on the rows that were looked up."""
        self._can_update()
        self._updc.seed = self.seed + self.steps_done
        self._backward(batch, grad_out, None, LAYOUT["rows"], self._upd, stream)
        self.steps_done += 1

    def check(self, stream=None) -> None:
        """Raise StepFailed if the last backward failed on the device (it then
        wrote no table row)."""
        if self.dedup is None:
            raise ValueError("a layer without max_tokens only looks up")
        _check_status(self.dedup.ws, stream)


# ---------------------------------------------------------------- recurrence

class Scan:
    """The inputs of a gated linear recurrence over ragged sequences (see
    emb_scan): int32 offsets [M + 1] on the GPU, values, forget gates and output
    gates (None: no output gate) as N x D matrices of one type, fp32 bias [D]
    and first states [M][D] or None."""

    def __init__(self, offsets, x, f, o=None, bias=None, h0=None):
        import torch
        if offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous():
            raise ValueError("offsets are a contiguous int32 vector")
        _device(offsets, "offsets")
        self.x, self.f, self.o = _mat(x), _mat(f), _mat(o) if o is not None else None
        self.offsets, self.bias, self.h0 = offsets, bias, h0
        self._c = CScan()
        self.ref = ctypes.byref(self._c)
        self._key = None
        self.c()

    def c(self) -> CScan:
        """The C descriptor; made again if a tensor has got other memory."""
        x, f, o, bias, h0 = self.x, self.f, self.o, self.bias, self.h0
        key = (self.offsets.data_ptr(), self.offsets.numel(), x.tensor.data_ptr(), f.tensor.data_ptr(),
               o.tensor.data_ptr() if o is not None else 0, bias.data_ptr() if bias is not None else 0,
               h0.data_ptr() if h0 is not None else 0)
        if x.exps is not None:
            key += tuple(m.exps.data_ptr() for m in (x, f, o) if m is not None and m.exps is not None)
        if key != self._key:
            x.c()
            f.c()
            if o is not None:
                o.c()
            self.tokens, self.dim, self.seqs = x.rows, x.cols, key[1] - 1
            _want(f, self.tokens, self.dim, "f")
            if o is not None:
                _want(o, self.tokens, self.dim, "o")
            c = self._c
            c.num_tokens, c.num_seqs, c.dim, c.offsets = self.tokens, self.seqs, self.dim, key[0]
            c.x, c.f, c.o = x._c, f._c, o._c if o is not None else CMat()
            c.bias = _floats(bias, (self.dim,), "bias")
            c.h0 = _floats(h0, (self.seqs, self.dim), "h0")
            self._key = key
        return self._c


def scan_workspace_size(num_tokens: int, dim: int) -> int:
    return int(lib().emb_scan_workspace_size(num_tokens, dim))


class Recurrence:
    """The gated linear recurrence with its workspace, for batches of up to
    ``max_tokens`` tokens (no buffer depends on the number of sequences:
    ``max_seqs`` is not looked at); with ``train`` the forward keeps a state every
    64 positions for the backward of the same batch.  Calls on one object must
    be ordered."""

    def __init__(self, max_tokens: int, max_seqs: int, dim: int, device="cuda", train: bool = True):
        import torch
        n = max(1, max_tokens)
        size = scan_workspace_size(n, dim)
        if size == 0:
            raise ValueError("batch too large for one call")
        self.max_tokens, self.max_seqs, self.dim = n, max_seqs, dim
        self.ws = _device(torch.empty(size, dtype=torch.uint8, device=device), "a recurrence's workspace")
        self._ws, self._wsb = self.ws.data_ptr(), size
        workspace_init(self.ws[:256])
        self.states = torch.empty(((n + SPAN - 1) // SPAN, dim), device=device) if train else None
        self._states = _ptr(self.states)
        self._tokens = None

    def _scan(self, scan: Scan):
        scan.c()
        if scan.tokens > self.max_tokens or scan.dim != self.dim:
            raise ValueError("batch larger than the recurrence's buffers, or of another width")
        return scan.ref

    def forward(self, scan: Scan, y, h_last=None, stream=None) -> None:
        """y (and the state after each sequence into ``h_last``, fp32 [M][D])."""
        ref = self._scan(scan)
        y = _mat(y)
        _want(y, scan.tokens, self.dim, "y")
        _check("emb_scan_fwd", lib().emb_scan_fwd(ref, y.ref,
                                                  _floats(h_last, (scan.seqs, self.dim), "h_last"), self._states,
                                                  self._ws, self._wsb, _stream(stream)))
        self._tokens = scan.tokens

    def backward(self, scan: Scan, dy, dx, df, do=None, dbias=None, dh_last=None, dh0=None, stream=None) -> None:
        """Gradients of the last forward: of the inputs, the bias and the first
        states, from those of y and of the last states.  ``scan`` is the
        forward's, or one whose matrices are restored from its checkpoints."""
        ref = self._scan(scan)
        if self.states is None or self._tokens != scan.tokens:
            raise ValueError("backward follows the forward of the same batch on a recurrence made with train")
        mats = [_mat(m) for m in (dy, dx, df)] + ([_mat(do)] if scan.o is not None else [])
        for m, name in zip(mats, ("dy", "dx", "df", "do")):
            _want(m, scan.tokens, self.dim, name)
        each = (scan.seqs, self.dim)
        _check("emb_scan_bwd", lib().emb_scan_bwd(
            ref, self._states, mats[0].ref, _floats(dh_last, each, "dh_last"), mats[1].ref, mats[2].ref,
            mats[3].ref if scan.o is not None else None, _floats(dbias, (self.dim,), "dbias"),
            _floats(dh0, each, "dh0"), self._ws, self._wsb, _stream(stream)))


    def check(self, stream=None) -> None:
        """Raise StepFailed if a wait inside a call since this object was made
        ran out (values are NaN from there on)."""
        _check_status(self.ws, stream)


def scan_step(x, f, o, state, y, bias=None, slots=None, stream=None) -> None:
    """One token of each running sequence (emb_scan_step): row i of x, f, o (or
    None) and y belongs to state row ``slots[i]`` (int32; None: row i), which is
    updated in place; tokens whose slot is no row of ``state`` get zeros."""
    x, f, y = _mat(x), _mat(f), _mat(y)
    n, D = x.rows, x.cols
    _want(f, n, D, "f")
    _want(y, n, D, "y")
    if o is not None:
        o = _mat(o)
        _want(o, n, D, "o")
    rows = state.shape[0]
    sp = None
    if slots is not None:
        if slots.numel() != n or slots.element_size() != 4 or slots.is_floating_point() or not slots.is_contiguous():
            raise ValueError("slots are a contiguous int32 vector, one a token")
        sp = _device(slots, "slots").data_ptr()
    _check("emb_scan_step", lib().emb_scan_step(n, D, x.ref, f.ref, o.ref if o is not None else None,
                                                _floats(bias, (D,), "bias"), _floats(state, (rows, D), "state"), rows,
                                                sp, y.ref, _stream(stream)))


# ---------------------------------------------------------------- checkpoints

def _scratch(size: int, device, stream):
    """Workspace of one call on ``stream``, taken from the caching allocator in
    that stream's order and given back in it: neither a call on another stream
    nor what is allocated after this call gets it while the call may run."""
    import torch
    if stream is None:
        return torch.empty(size, dtype=torch.uint8, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return torch.empty(size, dtype=torch.uint8, device=device)


class Checkpoint:
    """Activations kept in 8 bits: codes (int8) and an exponent a group of 32
    columns, for ``rows`` rows of ``dim`` columns."""

    def __init__(self, rows: int, dim: int, device="cuda"):
        import torch
        groups = (dim + GROUP - 1) // GROUP
        self._take(torch.empty((rows, groups * GROUP), dtype=torch.int8, device=device),
                   torch.empty((rows, groups), dtype=torch.uint8, device=device), dim)

    @classmethod
    def of(cls, codes, exps, dim: int) -> "Checkpoint":
        """A checkpoint that exists already: codes [rows][dim rounded up to
        32] and exponents [rows][groups]."""
        groups = (dim + GROUP - 1) // GROUP
        if tuple(codes.shape) != (codes.shape[0], groups * GROUP) or tuple(exps.shape) != (codes.shape[0], groups):
            raise ValueError("codes and exponents of whole groups are wanted")
        if not (codes.is_contiguous() and exps.is_contiguous()):
            raise ValueError("codes and exponents are contiguous")
        self = cls.__new__(cls)
        self._take(codes, exps, dim)
        return self

    def _take(self, codes, exps, dim: int) -> None:
        self.codes, self.exps, self.dim, self.rows = codes, exps, dim, int(codes.shape[0])
        self.mat = Mat(codes, exps, dim)

    def columns(self, first: int, count: int) -> Mat:
        """Columns first .. first + count - 1 as a matrix (for ``Scan``)."""
        if first % GROUP != 0 or first < 0 or count < 1 or first + count > self.dim:
            raise ValueError("columns of a checkpoint start at a group's first")
        return Mat(self.codes, self.exps, count, first)

    def pack(self, src, stream=None) -> None:
        src = _mat(src)
        _want(src, self.rows, self.dim, "src")
        _check("emb_save", lib().emb_save(self.rows, self.dim, src.ref, self.mat.ref, _stream(stream)))

    def unpack(self, dst, stream=None) -> None:
        dst = _mat(dst)
        _want(dst, self.rows, self.dim, "dst")
        _check("emb_restore", lib().emb_restore(self.rows, self.dim, self.mat.ref, dst.ref, _stream(stream)))

    def weight_grad(self, dy, dw, add: bool = False, stream=None) -> None:
        """dw[k][c] = sum over rows of the restored value times dy[row][c]: the
        gradient of the weights [dim][cols] (fp32) of a projection of what was
        packed (emb_weight_grad)."""
        dy = _mat(dy)
        _want(dy, self.rows, dy.cols, "dy")
        size = lib().emb_weight_grad_workspace_size(self.rows, self.dim, dy.cols)
        ws = _scratch(size, self.codes.device, stream) if size else None
        _check("emb_weight_grad", lib().emb_weight_grad(
            self.rows, self.dim, dy.cols, self.mat.ref, dy.ref, _floats(dw, (self.dim, dy.cols), "dw"), int(add),
            _ptr(ws), size, _stream(stream)))


# ---------------------------------------------------------------- together

class SequenceLayer:
    """A sequence layer over the tables: token rows, a projection to values,
    forget gates and output gates, the gated recurrence.

        rows = scale * W[token]                    (N x D, bf16)
        x | f | o = rows @ weight                  (N x 3H, bf16)
        y = sigmoid(o) * scan(x, f + bias)         (N x H, bf16)

    A training step is ``forward``, the caller's loss, ``backward``.  Between
    the two only checkpoints are kept, in 8 bits: of the rows (for the
    projection's weight gradient) and of the projection (for the recurrence's
    backward), 1.03 bytes a value instead of 2.  The layer holds room for those
    of ``max_tokens`` tokens from its first training forward on; rows and
    projection in full width are the caching allocator's for the length of a
    call, so a model's layers share them.  ``step`` is one token of each running
    sequence (serving), with states in a pool of slots.

    The backward reads the 8-bit checkpoints always; who wants its activations
    in 16 bits calls TokenLayer and Recurrence.

    ``weight`` is a bf16 D x 3H tensor and ``bias`` an fp32 one of H values, both
    the caller's: ``backward`` leaves their gradients in fp32 and trains the
    tables' rows itself (TokenLayer.update).  H is a multiple of 32."""

    def __init__(self, tables: Tables, weight, bias, max_tokens: int, max_seqs: int, scale: float = 1.0,
                 pad_row: int = -1, opt: str = "adagrad", lr: float = 0.01, eps: float = 1e-8, state=None,
                 rounding: str = "nearest", seed: int = 0):
        import torch
        dim, cols = (int(x) for x in weight.shape)
        if weight.dtype != torch.bfloat16 or cols % (3 * GROUP) != 0 or dim != int(tables.weights.shape[1]):
            raise ValueError("weight is a bf16 D x 3H tensor, H a multiple of 32")
        self.dim, self.hidden = dim, cols // 3
        self.weight, self.bias = weight, bias
        dev = tables.weights.device
        self.tokens = TokenLayer(tables, scale=scale, pad_row=pad_row, opt=opt, lr=lr, eps=eps, state=state,
                                 max_tokens=max_tokens, max_seqs=max_seqs, rounding=rounding, seed=seed)
        self.recurrence = Recurrence(max_tokens, max_seqs, self.hidden, dev)
        self._max, self._dev = max_tokens, dev
        self._room = self._saved = None
        self._n, self._offsets = -1, 0

    def _full(self, n: int):
        """Rows and projection of n tokens in full width, for one call."""
        import torch
        b16 = dict(dtype=torch.bfloat16, device=self._dev)
        return torch.empty((n, self.dim), **b16), torch.empty((n, 3 * self.hidden), **b16)

    def _project(self, batch: Batch, n: int):
        import torch
        rows, proj = self._full(n)
        self.tokens.forward(batch, rows)
        torch.mm(rows, self.weight, out=proj)
        return rows, proj, [Mat(proj, cols=self.hidden, first=i * self.hidden) for i in range(3)]

    def forward(self, batch: Batch, y, h_last=None, h0=None, train: bool = True) -> None:
        """y (N x H, bf16) and the state after each sequence (fp32 M x H) of
        the batch's sequences, from first states ``h0`` or zero; with ``train``
        what the backward needs is kept (``h0`` too: the caller may write to it
        before the backward, or give it as ``h_last``).  Runs on the current
        stream."""
        n = int(batch.indices.numel())
        if n > self.recurrence.max_tokens:
            raise ValueError("batch larger than the layer's buffers")
        rows, proj, parts = self._project(batch, n)
        first = h0.clone() if train and h0 is not None else None
        self.recurrence.forward(Scan(batch.offsets, *parts, bias=self.bias, h0=h0), y, h_last)
        self._n = -1
        if train:
            if self._room is None:
                self._room = tuple(Checkpoint(self._max, d, self._dev) for d in (self.dim, 3 * self.hidden))
            if self._saved is None or self._saved[0].rows != n:
                self._saved = tuple(Checkpoint.of(c.codes[:n], c.exps[:n], c.dim) for c in self._room)
            self._saved[0].pack(rows)
            self._saved[1].pack(proj)
            self._n, self._offsets, self._h0 = n, int(batch.offsets.numel()), first

    def backward(self, batch: Batch, dy, dweight, dbias, dh_last=None, dh0=None, add: bool = False) -> None:
        """Backward of the last ``forward``, whose batch this is: the gradients of
        the weights (fp32 D x 3H) and the bias (fp32 H, or None), with ``add``
        added to what is there, and the optimizer's step on the table rows."""
        import torch
        n, H = int(batch.indices.numel()), self.hidden
        if n != self._n or int(batch.offsets.numel()) != self._offsets:
            raise ValueError("backward follows a training forward of the same batch")
        # (all that can be refused is, before the first kernel: the step can then be repeated)
        self.tokens._can_update()
        dy = _mat(dy)
        _want(dy, n, H, "dy")
        if dy.dtype != BF16:
            raise ValueError("dy is bf16")
        if _floats(dweight, (self.dim, 3 * H), "dweight") is None:
            raise ValueError("dweight is wanted")
        _floats(dbias, (H,), "dbias")
        for t, name in ((dh_last, "dh_last"), (dh0, "dh0")):
            _floats(t, (self._offsets - 1, H), name)
        self._n = -1
        saved_rows, saved_proj = self._saved
        scan = Scan(batch.offsets, *(saved_proj.columns(i * H, H) for i in range(3)), bias=self.bias, h0=self._h0)
        drows, dproj = self._full(n)
        db = torch.empty_like(dbias) if add and dbias is not None else dbias
        self.recurrence.backward(scan, dy, *(Mat(dproj, cols=H, first=i * H) for i in range(3)), dbias=db,
                                 dh_last=dh_last, dh0=dh0)
        if db is not dbias:
            dbias += db
        saved_rows.weight_grad(dproj, dweight, add=add)
        torch.mm(dproj, self.weight.t(), out=drows)
        self.tokens.update(batch, drows)

    def check(self) -> None:
        """Raise StepFailed if the last backward's dedup or a recurrence failed on
        the device."""
        if self.tokens.dedup is not None:
            self.tokens.check()
        self.recurrence.check()

    def step(self, batch: Batch, state, y, slots=None) -> None:
        """The next token of each running sequence (one a sequence in
        ``batch``): y (N x H, bf16), the states updated in their slots."""
        n = int(batch.indices.numel())
        if n > self.recurrence.max_tokens:
            raise ValueError("batch larger than the layer's buffers")
        _, _, (x, f, o) = self._project(batch, n)
        scan_step(x, f, o, state, y, bias=self.bias, slots=slots)
