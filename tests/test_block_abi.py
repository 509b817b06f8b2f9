"""Host checks of the operators of a model's block, without a GPU: every refusal
returns before anything is enqueued (the pointers here are none), and the
binding's own checks."""
import ctypes

import pytest

import paper_2112_02752_amd as emb
from paper_2112_02752_amd.block import CHeads, CNorm
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


def _heads(n=60, m=3, heads=4, groups=2, dk=16, dv=8, offsets=0x2000, q=None, k=None, v=None, decay=0x3000, scale=1.0,
           first=None):
    return CHeads(n, m, heads, groups, dk, dv, offsets, q or _m(), k or _m(), v or _m(), decay, scale, first)


BAD_HEADS = [(dict(n=-1), EINVAL), (dict(m=-1), EINVAL), (dict(m=0), EINVAL), (dict(heads=0), EINVAL),
             (dict(groups=0), EINVAL), (dict(heads=3), EINVAL), (dict(dk=0), EINVAL), (dict(dv=0), EINVAL),
             (dict(dk=257), EUNSUPPORTED), (dict(dv=257), EUNSUPPORTED), (dict(n=1 << 31), EUNSUPPORTED),
             (dict(offsets=None), EINVAL), (dict(offsets=0x2002), EINVAL), (dict(decay=None), EINVAL),
             (dict(decay=0x3001), EINVAL), (dict(first=0x3002), EINVAL), (dict(scale=NAN), EINVAL),
             (dict(scale=INF), EINVAL), (dict(q=_m(ld=63)), EINVAL), (dict(k=_m(data=None)), EINVAL),
             (dict(v=_m(dtype=1)), EINVAL), (dict(q=_m(dtype=SAVED8)), EINVAL), (dict(k=_m(data=0x4001)), EINVAL),
             # more blocks than a grid holds
             (dict(m=(1 << 31) - 1), EUNSUPPORTED)]


def test_linear_attention_refusals():
    size = emb.lib().emb_linear_states_size
    assert size(64, 2, 16, 8) == 0 and size(65, 2, 16, 8) == 1024
    assert size(1 << 30, 2, 16, 8) == 256 * 1024            # segments grow instead
    for bad in ((-1, 2, 16, 8), (1 << 31, 2, 16, 8), (10, 0, 16, 8), (10, 2, 0, 8), (10, 2, 16, 257)):
        assert size(*bad) == 0

    def fwd(h=None, y=_m(0x7000), last=0x5000, states=0x100000, bytes_=0):
        return emb.lib().emb_linear_fwd(_ref(h or _heads()), _ref(y), last, states, bytes_, None)

    def bwd(h=None, dy=_m(0x7000), dq=_m(0x8000), dk=_m(0x9000), dv=_m(0xa000), states=0x100000, bytes_=0, dlast=0x5000, dfirst=0x6000,
            ws=0x200000, wsb=0):
        return emb.lib().emb_linear_bwd(_ref(h or _heads()), states, bytes_, _ref(dy), _ref(dq), _ref(dk), _ref(dv),
                                        dlast, dfirst, ws, wsb, None)

    for kw, status in BAD_HEADS:
        assert fwd(_heads(**kw)) == status, kw
        assert bwd(_heads(**kw)) == status, kw
    assert emb.lib().emb_linear_fwd(None, None, None, None, 0, None) == EINVAL
    empty = _heads(n=0, m=0, q=_m(data=None), decay=None)
    assert fwd(empty, y=None) == OK and bwd(empty, dy=None) == OK
    assert fwd(y=None) == EINVAL
    assert fwd(y=_m(ld=31)) == EINVAL
    assert fwd(y=_m(dtype=1)) == EINVAL
    assert fwd(last=0x5001) == EINVAL
    assert fwd(y=_m(0x4000)) == EINVAL                     # over an input
    far = _m(0x7000, (1 << 22) + 4)
    assert fwd(y=far) == EUNSUPPORTED                      # rows of more than 16 MB
    assert fwd(_heads(k=far)) == EUNSUPPORTED
    assert bwd(dk=far) == EUNSUPPORTED
    for name in ("dq", "dk", "dv"):
        for over in (0x4000, 0x7000):
            assert bwd(**{name: _m(over)}) == EINVAL
    assert bwd(_heads(first=0x6000)) == EINVAL             # first states' gradient over them
    assert fwd(_heads(first=0x5000), last=0x5000) == EINVAL
    long = _heads(n=65)
    assert fwd(long, bytes_=1023) == EWORKSPACE
    assert fwd(long, states=0x100010, bytes_=1024) == EWORKSPACE
    assert fwd(long, states=None, bytes_=1024) == EINVAL
    for name in ("dy", "dq", "dk", "dv"):
        for bad in (None, _m(data=None), _m(ld=15), _m(dtype=1)):
            assert bwd(**{name: bad}) == EINVAL
    assert bwd(dlast=0x6000) == EINVAL
    assert bwd(dfirst=0x6002) == EINVAL
    assert bwd(long, bytes_=1024) == EWORKSPACE
    assert bwd(long, wsb=1024) == EWORKSPACE
    assert bwd(long, bytes_=1024, wsb=1024, ws=0x100000) == EINVAL


def test_linear_step_refusals():
    def call(n=10, heads=4, groups=2, dk=16, dv=8, q=_m(), k=_m(), v=_m(), decay=0x3000, scale=1.0, state=0x5000,
             num=20, slots=0x6000, y=_m(0x7000)):
        return emb.lib().emb_linear_step(n, heads, groups, dk, dv, _ref(q), _ref(k), _ref(v), decay, scale, state, num,
                                         slots, _ref(y), None)

    assert call(n=0, q=None, state=None) == OK
    for kw in (dict(n=-1), dict(num=-1), dict(heads=3), dict(groups=0), dict(dk=0), dict(decay=None), dict(state=None),
               dict(state=0x5001), dict(slots=0x6001), dict(scale=NAN), dict(q=None), dict(k=_m(ld=31)),
               dict(v=_m(dtype=1)), dict(y=_m(data=None)), dict(y=_m(dtype=SAVED8))):
        assert call(**kw) == EINVAL, kw
    assert call(dk=257) == EUNSUPPORTED
    assert call(n=1 << 31) == EUNSUPPORTED
    assert call(n=1 << 28) == EUNSUPPORTED                 # more blocks than a grid holds


def test_log_probability_refusals():
    L = emb.lib()

    def fwd(n=10, d=64, x=_m(), ids=0x1000, size=8, scale=1.0, logp=0x2000, entropy=0x3000, top=2, ti=0x4000, tl=0x5000,
            stats=0x6000):
        return L.emb_logp_fwd(n, d, _ref(x), ids, size, scale, logp, entropy, top, ti, tl, stats, None)

    def bwd(n=10, d=64, x=_m(), ids=0x1000, size=8, scale=1.0, stats=0x6000, dlogp=0x2000, dentropy=0x3000,
            dx=_m(0x8000)):
        return L.emb_logp_bwd(n, d, _ref(x), ids, size, scale, stats, dlogp, dentropy, _ref(dx), None)

    def train(n=10, d=64, x=_m(), ids=0x1000, size=8, scale=1.0, dlogp=0x2000, logp=None, entropy=None, dx=_m(0x8000)):
        return L.emb_logp_train(n, d, _ref(x), ids, size, scale, dlogp, logp, entropy, _ref(dx), None)

    for call in (fwd, bwd, train):
        for kw in (dict(n=-1), dict(d=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF),
                   dict(size=2), dict(ids=0x1004), dict(ids=0x1002, size=4), dict(x=None), dict(x=_m(ld=63)),
                   dict(x=_m(dtype=SAVED8)), dict(x=_m(data=0x4002)), dict(ids=None)):
            assert call(**kw) == EINVAL, (call, kw)
        assert call(n=1 << 31) == EUNSUPPORTED
        assert call(d=(1 << 30) + 1, x=_m(ld=1 << 31)) == EUNSUPPORTED
        assert call(n=0, x=None, ids=None) == OK
    assert fwd(n=(1 << 31) - 100, d=1 << 20, x=_m(ld=1 << 20)) == EUNSUPPORTED   # more blocks than a grid holds
    assert bwd(n=(1 << 31) - 100, d=1 << 20, x=_m(ld=1 << 20), dx=_m(0x8000, 1 << 20)) == EUNSUPPORTED
    for kw in (dict(logp=None), dict(logp=0x2002), dict(entropy=0x3001), dict(top=-1), dict(top=65), dict(ti=None),
               dict(tl=None), dict(ti=0x4002), dict(stats=0x6004)):
        assert fwd(**kw) == EINVAL, kw
    assert fwd(top=33) == EUNSUPPORTED
    for call in (bwd, train):
        for kw in (dict(dlogp=None), dict(dlogp=0x2002), dict(dx=None), dict(dx=_m(0x8000, 63)),
                   dict(dx=_m(0x8000, 64, 1)), dict(dx=_m(0x4000, 65))):
            assert call(**kw) == EINVAL, (call, kw)
    assert bwd(stats=None) == EINVAL
    assert bwd(stats=0x6004) == EINVAL


def test_log_probabilities_of_the_binding():
    for kw in (dict(cols=0), dict(cols=10, top=11), dict(cols=100, top=33), dict(cols=10, top=-1)):
        with pytest.raises(ValueError, match="top"):
            emb.LogProbs(4, **kw)
    for scale in (0.0, -1.0, NAN, INF):
        with pytest.raises(ValueError, match="scale"):
            emb.LogProbs(4, 10, scale=scale)
    with pytest.raises(ValueError, match="GPU"):
        emb.LogProbs(4, 10, device="cpu")


def test_linear_attention_of_the_binding():
    import torch
    with pytest.raises(ValueError, match="multiple"):
        emb.LinearAttention(10, 1, 3, 2, 8, 8)
    with pytest.raises(ValueError, match="column"):
        emb.LinearAttention(10, 1, 2, 2, 0, 8)
    with pytest.raises(ValueError, match="GPU"):
        emb.LinearAttention(10, 1, 2, 2, 8, 8, device="cpu")
    for bad in (torch.zeros(3), torch.zeros(3, dtype=torch.int64), torch.zeros((2, 2), dtype=torch.int32),
                torch.zeros(6, dtype=torch.int32)[::2], torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(ValueError, match="offsets"):
            emb.Heads(bad, None, None, None, None, heads=2)
    with pytest.raises(ValueError, match="GPU"):
        emb.Heads(torch.zeros(3, dtype=torch.int32), None, None, None, None, heads=2)


def test_matrices_of_another_device(monkeypatch):
    """Refused before the library is called."""
    import torch
    from paper_2112_02752_amd import block

    class Stub(emb.Mat):
        """A matrix without a GPU."""

        def __init__(self, rows, cols, device):
            self.tensor, self.exps, self.rows, self.cols = self, None, rows, cols
            self._at, self.device, self._c = 0, device, CMat()
            self.ref = ctypes.byref(self._c)

        def data_ptr(self):
            return 0

        def get_device(self):
            return self.device

    monkeypatch.setattr(block, "_device_now", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        emb.dropout(Stub(4, 8, 0), Stub(4, 8, 1), 0.1, 1)
    with pytest.raises(ValueError, match="current device"):
        emb.dropout(Stub(4, 8, 1), Stub(4, 8, 0), 0.1, 1)
    with pytest.raises(ValueError, match="current device"):
        emb.linear_attention_step(Stub(4, 8, 1), Stub(4, 8, 1), Stub(4, 8, 0), None, torch.zeros(4), Stub(4, 8, 1), 2)
    class Vector:
        def __init__(self, device):
            self.device = device

        def get_device(self):
            return self.device

    mats = [Stub(4, 8, 1) for _ in range(4)]
    for bad in range(3):
        decay, state, slots = (Vector(0 if i == bad else 1) for i in range(3))
        with pytest.raises(ValueError, match="tensors lie on the current device"):
            emb.linear_attention_step(*mats[:3], decay, state, mats[3], 2, slots=slots)


def test_outputs_across_inputs():
    """An output in place has its input's strides; what other blocks still read is not written."""
    L, a, b = emb.lib(), _m(0x4000, 64), _m(0x4000, 80)
    other, out = _m(0x8000, 64), _m(0xc000, 64)
    n, d, norm = 10, 32, _norm()

    def fwd(x=other, residual=None, total=None, y=out, rows=n):
        return L.emb_norm_fwd(rows, d, _ref(norm), _ref(x), _ref(residual), _ref(total), _ref(y), None, None)

    for kw in (dict(x=a, y=b), dict(residual=a, total=b), dict(x=a, total=b), dict(residual=b, y=a)):
        assert fwd(**kw) == EINVAL, kw

    def bwd(total=other, dy=_m(0x9000), arriving=None, dtotal=None, dbranch=None):
        return L.emb_norm_bwd(n, d, _ref(norm), _ref(total), _ref(dy), _ref(arriving), _ref(dtotal), _ref(dbranch),
                              None, 0, None, 0, None)

    for out_name in ("dtotal", "dbranch"):
        for in_name in ("total", "dy", "arriving"):
            assert bwd(**{out_name: a, in_name: b}) == EINVAL, (out_name, in_name)
    assert L.emb_dropout(n, d, 0.5, 1, 0, _ref(a), _ref(b), None) == EINVAL
    assert L.emb_logp_bwd(n, d, _ref(a), 0x1000, 4, 1.0, 0x2000, 0x3000, None, _ref(b), None) == EINVAL
    assert L.emb_logp_train(n, d, _ref(a), 0x1000, 4, 1.0, 0x2000, 0x3000, None, _ref(b), None) == EINVAL
    for logp, entropy in ((0x2000, None), (None, 0x2000)):
        assert L.emb_logp_train(n, d, _ref(a), 0x1000, 4, 1.0, 0x2000, logp, entropy, _ref(out), None) == EINVAL
    for at in (0x4000, 0x5000, 0x6000):
        assert L.emb_linear_step(n, 2, 2, 16, 16, _ref(_m(0x4000)), _ref(_m(0x5000)), _ref(_m(0x6000)), 0x1000, 1.0,
                                 0x2000, n, None, _ref(_m(at)), None) == EINVAL
