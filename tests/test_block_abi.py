"""Host checks of the operators of a model's block, without a GPU: every refusal
returns before anything is enqueued (the pointers here are none), and the
binding's own checks."""
import ctypes

import pytest

import paper_2112_02752_amd as emb
from paper_2112_02752_amd.block import CNorm
from paper_2112_02752_amd.sequence import CMat, SAVED8

OK, EINVAL, EWORKSPACE, EUNSUPPORTED = emb.EMB_OK, emb.EMB_EINVAL, emb.EMB_EWORKSPACE, emb.EMB_EUNSUPPORTED
NAN, INF = float("nan"), float("inf")


def _m(data=0x4000, ld=64, dtype=0, exps=None, ld_exps=0):
    return CMat(data, ld, dtype, exps, ld_exps)


def _ref(m):
    return ctypes.byref(m) if m is not None else None


def _norm(weight=0x1000, eps=1e-6, drop=0.0, seed=1, first_row=0):
    return CNorm(weight, eps, drop, seed, first_row)


def test_norm_refusals():
    def call(n=10, d=64, norm=_norm(), x=_m(), residual=_m(), total=_m(), y=_m(), saved=None):
        return emb.lib().emb_norm_fwd(n, d, _ref(norm), _ref(x), _ref(residual), _ref(total), _ref(y), _ref(saved), None)

    assert call(n=0, x=None, y=None) == OK
    assert call(n=-1) == EINVAL
    assert call(d=0) == EINVAL
    assert call(norm=None) == EINVAL
    assert call(d=16385, x=_m(ld=1 << 15)) == EUNSUPPORTED
    assert call(n=1 << 31) == EUNSUPPORTED
    for bad in (_norm(eps=-1.0), _norm(eps=NAN), _norm(eps=INF), _norm(drop=1.0), _norm(drop=-0.1), _norm(drop=NAN),
                _norm(drop=1 - 2.0 ** -20), _norm(first_row=-1), _norm(weight=0x1002)):
        assert call(norm=bad) == EINVAL
    assert call(x=None) == EINVAL
    assert call(x=_m(data=None)) == EINVAL
    assert call(x=_m(ld=63)) == EINVAL                     # rows overlap
    assert call(x=_m(dtype=SAVED8)) == EINVAL
    assert call(x=_m(dtype=5)) == EINVAL
    assert call(x=_m(data=0x4002)) == EINVAL               # not aligned to a value
    assert call(y=_m(dtype=1)) == EINVAL                   # another type than x's
    assert call(residual=_m(dtype=1)) == EINVAL            # a narrower stream
    assert call(x=_m(dtype=1), y=_m(dtype=1), residual=_m(dtype=1), total=_m()) == EINVAL  # two types of stream
    assert call(y=None) == EINVAL                          # nothing asked for
    assert call(saved=_m()) == EINVAL
    assert call(saved=_m(0x4000, 64, SAVED8, None, 2)) == EINVAL
    assert call(saved=_m(0x4000, 32, SAVED8, 0x100, 2)) == EINVAL
    assert call(saved=_m(0x4010, 64, SAVED8, 0x100, 2)) == EINVAL


def test_norm_backward_refusals():
    need = emb.lib().emb_norm_workspace_size(10, 64)
    assert need > 0 and need % 256 == 0
    for n, d in ((-1, 64), (10, 0), (10, 16385), (1 << 31, 64)):
        assert emb.lib().emb_norm_workspace_size(n, d) == 0

    def call(n=10, d=64, norm=_norm(), total=_m(), dy=_m(), arriving=None, dtotal=_m(), branch=_m(), dw=0x8000,
             ws=0x100000, size=need):
        return emb.lib().emb_norm_bwd(n, d, _ref(norm), _ref(total), _ref(dy), _ref(arriving), _ref(dtotal),
                                      _ref(branch), dw, 0, ws, size, None)

    assert call(total=None) == EINVAL
    assert call(dy=None) == EINVAL
    assert call(arriving=_m(dtype=1)) == EINVAL
    assert call(branch=_m(dtype=1)) == EINVAL
    assert call(dtotal=_m(ld=3)) == EINVAL
    assert call(dw=0x8002) == EINVAL
    assert call(ws=None) == EINVAL
    assert call(ws=0x100010) == EWORKSPACE
    assert call(size=need - 256) == EWORKSPACE
    assert call(norm=_norm(drop=1.5)) == EINVAL
    assert call(n=0, total=None, dy=None, dw=None, ws=None, size=0) == OK


def test_dropout_refusals():
    def call(n=10, d=64, p=0.1, first=0, x=_m(), y=_m()):
        return emb.lib().emb_dropout(n, d, p, 1, first, _ref(x), _ref(y), None)

    assert call(n=0, x=None) == OK
    assert call(n=-1) == EINVAL
    assert call(d=0) == EINVAL
    for p in (1.0, -0.1, NAN, 1 - 2.0 ** -20):
        assert call(p=p) == EINVAL
    assert call(first=-1) == EINVAL
    assert call(x=None) == EINVAL
    assert call(y=_m(dtype=1)) == EINVAL
    assert call(y=_m(ld=10)) == EINVAL
    assert call(n=1 << 31) == EUNSUPPORTED
    assert call(n=1 << 30, d=1 << 12, x=_m(ld=1 << 12), y=_m(ld=1 << 12)) == EUNSUPPORTED


def test_norm_of_the_binding():
    import torch
    with pytest.raises(ValueError, match="GPU"):
        emb.Norm(torch.ones(8))
    with pytest.raises(ValueError, match="vector"):
        emb.Norm(torch.ones(8, 2))
    with pytest.raises(ValueError, match="share"):
        emb.Norm(torch.ones(8), drop=1.0)
    with pytest.raises(ValueError, match="eps"):
        emb.Norm(torch.ones(8), eps=-1.0)
    with pytest.raises(ValueError, match="eps"):
        emb.Norm(torch.ones(8), eps=NAN)
    with pytest.raises(ValueError, match="fp32"):
        emb.Norm(torch.ones(8, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="fp32"):
        emb.Norm(torch.ones(16)[::2])
