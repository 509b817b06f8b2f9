"""Host checks of the operators over sequences, without a GPU: every refusal
returns before anything is enqueued (the pointers here are none), and the
binding's own checks of shapes."""
import ctypes

import pytest

import paper_2112_02752_amd as emb
from paper_2112_02752_amd.sequence import CMat, CScan, CToken, SAVED8

class L:
    """The library's functions, loaded by their first call: not while the tests
    of a run are collected, before PyTorch's own HIP runtime is loaded."""


def _load(name):
    return lambda *a: getattr(emb.lib(), name)(*a)


for _name in emb.EXPORTED:
    setattr(L, _name, staticmethod(_load(_name)))
OK, EINVAL, EWORKSPACE, EUNSUPPORTED = emb.EMB_OK, emb.EMB_EINVAL, emb.EMB_EWORKSPACE, emb.EMB_EUNSUPPORTED


def _tables(row_offset=(0, 100), dim=16, dtype=0, weights=0x1000):
    ro = (ctypes.c_int64 * len(row_offset))(*row_offset)
    t = emb.CTables(len(row_offset) - 1, ro, dim, dtype, weights)
    t._keep = ro
    return t


def _batch(B=4, offsets=0x2000, indices=0x3000, n=10):
    return emb.CBatch(B, offsets, indices, n, 4)


def _m(data=0x4000, ld=16, dtype=0, exps=None, ld_exps=0):
    return CMat(data, ld, dtype, exps, ld_exps)


def test_lookup_refusals():
    def call(t=None, b=None, tok=CToken(1.0, -1), out=_m()):
        return L.emb_token_fwd(ctypes.byref(t or _tables()), ctypes.byref(b or _batch()),
                               ctypes.byref(tok) if tok else None, ctypes.byref(out) if out else None, None)

    assert call(tok=None) == EINVAL
    assert call(tok=CToken(1.0, 100)) == EINVAL            # a padding row outside the tables
    assert call(out=None) == EINVAL
    assert call(out=_m(data=None)) == EINVAL
    assert call(out=_m(ld=15)) == EINVAL                   # rows overlap
    assert call(out=_m(dtype=SAVED8)) == EINVAL
    assert call(out=_m(dtype=7)) == EINVAL
    assert call(out=_m(data=0x4002)) == EINVAL             # not aligned to a value
    assert call(t=_tables(dim=3)) == EUNSUPPORTED
    assert call(t=_tables(weights=None)) == EINVAL
    assert call(b=_batch(n=1 << 30)) == EUNSUPPORTED
    assert call(b=_batch(indices=None)) == EINVAL
    assert call(b=_batch(n=0, indices=None), out=None) == OK


def test_token_gradient_refusals():
    need = emb.workspace_size(1000, 4, 16)
    sgd, bad, stateless = emb.CUpdate(0, 0.1), emb.CUpdate(5, 0.1), emb.CUpdate(1, 0.1)

    def call(t=None, b=None, tok=CToken(1.0, -1), dy=_m(), perm=0x100, grad=0x10000, layout=0, fuse=None, ws=0x100000,
             nbytes=need):
        return L.emb_token_grad(ctypes.byref(t or _tables()), ctypes.byref(b or _batch(n=1000)), ctypes.byref(tok),
                                ctypes.byref(dy), perm, 0x200, 0x300, 0x400, grad, layout,
                                ctypes.byref(fuse) if fuse else None, ws, nbytes, None)

    assert call(grad=None) == EINVAL                       # neither a gradient nor an update
    assert call(fuse=sgd) == EINVAL                        # both
    assert call(grad=None, fuse=bad) == EINVAL
    assert call(grad=None, fuse=stateless) == EINVAL
    assert call(layout=3) == EINVAL
    assert call(grad=0x10004) == EINVAL                    # not 16-byte aligned
    assert call(tok=CToken(1.0, 100)) == EINVAL
    assert call(dy=_m(ld=8)) == EINVAL
    assert call(dy=_m(dtype=SAVED8)) == EINVAL
    assert call(perm=None) == EINVAL
    assert call(ws=None) == EINVAL
    assert call(ws=0x100010) == EWORKSPACE
    assert call(nbytes=need - 256) == EWORKSPACE
    assert call(t=_tables(dim=8196), dy=_m(ld=9000)) == EUNSUPPORTED
    assert call(t=_tables(dim=4100), dy=_m(ld=9000)) == EUNSUPPORTED   # wide rows go eight columns a lane
    # element-wise accumulators are read as vectors
    assert call(grad=None, fuse=emb.CUpdate(2, 0.1, 0.0, 0x504)) == EINVAL


def _scan(n=100, m=3, d=16, offsets=0x2000, x=None, f=None, o=None):
    return CScan(n, m, d, offsets, x or _m(), f or _m(0x5000), o or _m(0x6000), None, None)


def test_scan_refusals():
    need = emb.scan_workspace_size(100, 16)
    assert need > 0 and need % 256 == 0
    assert emb.scan_workspace_size(-1, 16) == 0 and emb.scan_workspace_size(10, 0) == 0
    assert emb.scan_workspace_size(1 << 31, 16) == 0
    assert emb.scan_workspace_size(0, 16) > 0

    def fwd(s=None, y=_m(0x7000), ws=0x100000, nbytes=need):
        return L.emb_scan_fwd(ctypes.byref(s or _scan()), ctypes.byref(y) if y else None, None, None, ws, nbytes, None)

    assert fwd(s=_scan(n=-1)) == EINVAL
    assert fwd(s=_scan(m=-1)) == EINVAL
    assert fwd(s=_scan(m=0)) == EINVAL                     # tokens of no sequence
    assert fwd(s=_scan(d=0)) == EINVAL
    assert fwd(s=_scan(offsets=None)) == EINVAL
    assert fwd(s=_scan(n=1 << 31)) == EUNSUPPORTED
    assert fwd(s=_scan(n=(1 << 31) - 100, d=8192)) == EUNSUPPORTED     # more blocks than 32 bits count
    assert fwd(s=_scan(x=_m(data=None))) == EINVAL
    assert fwd(s=_scan(f=_m(dtype=1))) == EINVAL           # two types
    assert fwd(s=_scan(o=_m(ld=4))) == EINVAL
    assert fwd(y=None) == EINVAL
    assert fwd(y=_m(dtype=1)) == EINVAL
    assert fwd(ws=None) == EINVAL
    assert fwd(ws=0x100008) == EWORKSPACE
    assert fwd(nbytes=need - 256) == EWORKSPACE
    q = lambda at: _m(at, 32, SAVED8, 0x9000, 1)  # noqa: E731
    saved = _scan(x=q(0x4000), f=q(0x5000), o=q(0x6000))
    assert fwd(s=saved) == EUNSUPPORTED                    # the forward reads no checkpoints

    def bwd(s=None, states=0x8000, dy=_m(0x7000), dx=_m(0x7100), df=_m(0x7200), do=_m(0x7300), nbytes=need):
        r = lambda m: ctypes.byref(m) if m else None  # noqa: E731
        return L.emb_scan_bwd(ctypes.byref(s or _scan()), states, r(dy), None, r(dx), r(df), r(do), None, None,
                              0x100000, nbytes, None)

    assert bwd(states=None) == EINVAL
    for name in ("dy", "dx", "df", "do"):
        assert bwd(**{name: None}) == EINVAL, name
        assert bwd(**{name: _m(0x7000, 8)}) == EINVAL, name
    assert bwd(dx=_m(0x7100, dtype=1)) == EINVAL
    b16 = dict(dy=_m(0x7000, dtype=1), dx=_m(0x7100, dtype=1), df=_m(0x7200, dtype=1), do=_m(0x7300, dtype=1))
    assert bwd(**b16) == EINVAL                            # gradients of another type than the inputs
    assert bwd(nbytes=need - 256) == EWORKSPACE
    assert bwd(s=_scan(x=q(0x4010), f=q(0x5000), o=q(0x6000))) == EINVAL    # codes not aligned
    assert bwd(s=_scan(x=_m(0x4000, 24, SAVED8, 0x9000, 1), f=q(0x5000), o=q(0x6000))) == EINVAL
    assert bwd(s=_scan(x=_m(0x4000, 32, SAVED8, None, 1), f=q(0x5000), o=q(0x6000))) == EINVAL
    assert bwd(s=_scan(f=q(0x5000))) == EINVAL


def test_scan_step_refusals():
    def call(n=5, d=16, x=_m(), f=_m(), o=_m(), state=0x8000, slots=5, y=_m()):
        r = lambda m: ctypes.byref(m) if m else None  # noqa: E731
        return L.emb_scan_step(n, d, r(x), r(f), r(o), None, state, slots, None, r(y), None)

    assert call(n=-1) == EINVAL and call(d=0) == EINVAL and call(slots=-1) == EINVAL
    assert call(n=1 << 31) == EUNSUPPORTED
    assert call(state=None) == EINVAL
    for name in ("x", "f", "y"):
        assert call(**{name: None}) == EINVAL, name
    assert call(o=_m(dtype=1)) == EINVAL
    assert call(x=_m(dtype=SAVED8)) == EINVAL
    assert call(f=_m(ld=3)) == EINVAL
    assert call(n=0, x=None, f=None, y=None) == OK


def test_checkpoint_refusals():
    saved = _m(0x8000, 32, SAVED8, 0x9000, 1)
    for fn, order in ((L.emb_save, lambda full, q: (full, q)), (L.emb_restore, lambda full, q: (q, full))):
        def call(n=5, d=16, full=_m(), q=saved):
            a, b = order(full, q)
            return fn(n, d, ctypes.byref(a) if a else None, ctypes.byref(b) if b else None, None)

        assert call(n=-1) == EINVAL and call(d=0) == EINVAL
        assert call(n=1 << 31) == EUNSUPPORTED
        assert call(full=None) == EINVAL and call(q=None) == EINVAL
        assert call(full=saved) == EINVAL and call(q=_m()) == EINVAL
        assert call(full=_m(ld=8)) == EINVAL
        assert call(d=33, full=_m(ld=40)) == EINVAL        # codes of 33 columns take 64
        assert call(q=_m(0x8004, 32, SAVED8, 0x9000, 1)) == EINVAL
        assert call(q=_m(0x8000, 40, SAVED8, 0x9000, 1)) == EINVAL
        assert call(q=_m(0x8000, 32, SAVED8, 0x9000, 0)) == EINVAL
        assert call(n=0, full=None, q=None) == OK


def test_weight_gradient_refusals():
    q = _m(0x8000, 64, SAVED8, 0x9000, 2)
    need = L.emb_weight_grad_workspace_size(5000, 64, 16)
    assert need > 0 and need % 256 == 0                    # one tile of dw: the rows are cut
    assert L.emb_weight_grad_workspace_size(-1, 64, 16) == 0
    assert L.emb_weight_grad_workspace_size(1 << 31, 64, 16) == 0

    def call(n=5000, k=64, c=16, x=q, dy=_m(), dw=0x7000, ws=0x100000, nbytes=need):
        r = lambda m: ctypes.byref(m) if m else None  # noqa: E731
        return L.emb_weight_grad(n, k, c, r(x), r(dy), dw, 0, ws, nbytes, None)

    assert call(n=-1) == EINVAL and call(k=0) == EINVAL and call(c=0) == EINVAL and call(dw=None) == EINVAL
    assert call(n=1 << 31) == EUNSUPPORTED
    assert call(x=None) == EINVAL and call(x=_m(ld=64)) == EINVAL
    assert call(k=65) == EINVAL
    assert call(dy=None) == EINVAL and call(dy=_m(ld=15)) == EINVAL and call(dy=q) == EINVAL
    assert call(ws=None) == EINVAL
    assert call(ws=0x100010) == EWORKSPACE and call(nbytes=need - 256) == EWORKSPACE


def test_binding_checks_need_no_gpu():
    import torch
    with pytest.raises(ValueError, match="GPU"):
        emb.Mat(torch.zeros(3, 4))
    with pytest.raises(ValueError, match="two dimensions"):
        emb.Mat(torch.zeros(3))
    with pytest.raises(ValueError, match="contiguous columns"):
        emb.Mat(torch.zeros(3, 4).t())
    with pytest.raises(ValueError, match="offsets"):
        emb.Scan(torch.zeros(3), None, None)
    with pytest.raises(ValueError, match="whole groups"):
        emb.Checkpoint.of(torch.zeros(3, 40, dtype=torch.int8), torch.zeros(3, 2, dtype=torch.uint8), 40)
