"""Operators of a model's block where offsets pass 32 bits: rows far apart, of
which only the used columns are touched, against the same rows side by side
(bit for bit: the variants are chosen by widths and alignment alone)."""
import pytest

from .block_plain import DEV, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _far(x, ld):
    """The rows of x, `ld` values apart."""
    import torch
    n, d = x.shape
    view = torch.empty((n - 1) * ld + d, dtype=x.dtype, device=DEV).as_strided((n, d), (ld, 1))
    view.copy_(x)
    return view


def test_norm_and_dropout_of_rows_far_apart():
    import torch
    import paper_2112_02752_amd as emb
    say("far rows: norm, dropout")
    torch.manual_seed(1)
    near = [torch.randn((3, 520), device=DEV).bfloat16() for _ in range(4)]
    far = [_far(x, (1 << 30) + 64) for x in near]          # the last at 4 GB
    assert far[0].stride(0) * 2 * 2 > 1 << 32
    w = torch.ones(520, device=DEV)
    norm = emb.Norm(w, drop=0.2, max_rows=3)
    out = []
    for x, res, dy, arr in (near, far):
        total, y, dt, dx, dw = torch.empty_like(near[0]), torch.empty_like(near[0]), torch.empty_like(near[0]), \
            torch.empty_like(near[0]), torch.empty_like(w)
        norm.forward(x, y, residual=res, total=total, seed=3)
        norm.backward(total, dy, dt, branch=dx, arriving=arr, dweight=dw, seed=3)
        z = torch.empty_like(near[0])
        emb.dropout(x, z, 0.3, 5)
        out.append((total, y, dt, dx, dw, z))
    norm.forward(near[0], far[0], residual=near[1], total=far[1], seed=3)
    norm.backward(far[1], near[2], far[2], branch=far[3], arriving=near[3], seed=3)
    for a, b in zip(*out):
        assert torch.equal(a, b)
    for a, b in zip(out[0][:4], (far[1], far[0], far[2], far[3])):
        assert torch.equal(a, b)


def test_linear_attention_of_rows_far_apart():
    import torch
    import paper_2112_02752_amd as emb
    say("far rows: linear attention")
    torch.manual_seed(2)
    n, h, g, dk, dv, ld = 280, 2, 1, 16, 32, (1 << 23) - 64   # 16 MB a row, 4.7 GB in all
    near = [torch.randn((n, c), device=DEV).bfloat16() for c in (h * dk, g * dk, g * dv, h * dv)]
    far = [_far(x, ld) for x in near]
    offs = torch.tensor([0, 30, 280], dtype=torch.int32, device=DEV)
    decay = torch.tensor([0.95], device=DEV)
    out = []
    for q, k, v, dy in (near, far):
        heads = emb.Heads(offs, q, k, v, decay, heads=h, groups=g)
        att = emb.LinearAttention(n, 2, h, g, dk, dv)
        far_y = q is far[0]
        y = _far(torch.empty_like(near[3]), ld) if far_y else torch.empty_like(near[3])
        last = torch.empty((2, g, dk, dv), device=DEV)
        att.forward(heads, y, last)
        dq = _far(torch.empty_like(near[0]), ld) if far_y else torch.empty_like(near[0])
        dkey, dval = torch.empty_like(near[1]), torch.empty_like(near[2])
        att.backward(heads, dy, dq, dkey, dval)
        state = torch.zeros((n, g, dk, dv), device=DEV)
        z = torch.empty_like(near[3])
        emb.linear_attention_step(q, k, v, decay, state, z, heads=h, groups=g)
        out.append([t.clone() for t in (y, last, dq, dkey, dval, state, z)])
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_states_past_4_gb():
    """A step whose slots lie far into a pool."""
    import torch
    import paper_2112_02752_amd as emb
    say("far states")
    g, dk, dv, slots = 2, 128, 128, 40000                    # 5.2 GB
    pool = torch.empty((slots, g, dk, dv), device=DEV)
    where = torch.tensor([slots - 1, 0, 33000], dtype=torch.int32, device=DEV)
    torch.manual_seed(3)
    start = torch.randn((3, g, dk, dv), device=DEV)
    pool[where.long()] = start
    q, k, v = (torch.randn((3, g * 128), device=DEV) for _ in range(3))
    decay = torch.tensor([0.9, 0.5], device=DEV)
    y, y2, small = torch.empty((3, g * dv), device=DEV), torch.empty((3, g * dv), device=DEV), start.clone()
    emb.linear_attention_step(q, k, v, decay, pool, y, heads=g, slots=where)
    emb.linear_attention_step(q, k, v, decay, small, y2, heads=g)
    assert torch.equal(y, y2) and torch.equal(pool[where.long()], small)


def test_logits_far_apart():
    import torch
    import paper_2112_02752_amd as emb
    say("far rows: logits")
    torch.manual_seed(4)
    near = torch.randn((3, 5000), device=DEV).bfloat16()
    far = _far(near, (1 << 30) + 64)
    ids = torch.tensor([0, 4999, 17], device=DEV)
    w, wh = torch.randn(3, device=DEV), torch.randn(3, device=DEV)
    answer = emb.LogProbs(3, 5000, top=4)
    out = []
    for x in (near, far):
        logp, top, tl, dx = torch.empty(3, device=DEV), torch.empty((3, 4), dtype=torch.int32, device=DEV), \
            torch.empty((3, 4), device=DEV), torch.empty_like(near)
        answer.forward(x, ids, logp, top_ids=top, top_logp=tl)
        answer.backward(x, ids, w, dx, dentropy=wh)
        one = torch.empty_like(near)
        answer.train(x, ids, None, w, one)
        out.append((logp, top, tl, dx, one))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    other = _far(near, (1 << 30) + 64)
    answer.train(near, ids, None, w, other)
    answer.train(far, ids, None, w, far)
    assert torch.equal(other, out[0][4]) and torch.equal(far, out[0][4])
