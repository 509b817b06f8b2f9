"""The operators of a model's block run together with those over sequences, as a
model's training step and its serving would: token rows, norm, projection to
queries, keys and values, linear attention, projection back, dropout and residual,
norm, logits, log probabilities of the next tokens, and all the way back to the
table's rows, against the same model in 64 bits by autograd; then prompts and
single tokens of the model against whole sequences.

Tolerance: no stage adds more than 512 terms into a value, so that each of the
twelve stages is off by at most 512 u of what it adds; a result is held to
12 * 512 u of the largest value of its tensor."""
import numpy as np
import pytest

from .block_plain import DEV, U, host, kept, keep_scale, say

pytestmark = pytest.mark.gpu

ROWS, DIM, HEADS, GROUPS, DK, DV, SEQS = 300, 64, 4, 2, 24, 16, 5
SCALE, DROP, EPS, NEAR = 0.7, 0.2, 1e-5, 12 * 512 * U


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _close(got, want, what):
    off, most = np.abs(host(got) - want.detach().double().numpy()).max(), float(want.detach().abs().max())
    assert off <= NEAR * most, (what, off, most)


class Model:
    """One block over the tables, fp32."""

    def __init__(self, seed):
        import torch
        import paper_2112_02752_amd as emb
        torch.manual_seed(seed)
        new = lambda *s: torch.randn(s, device=DEV) / s[0] ** 0.5  # noqa: E731
        self.cols = HEADS * DK, GROUPS * DK, GROUPS * DV
        self.table = torch.randn((ROWS, DIM), device=DEV)
        self.tables = emb.Tables(self.table, [0, ROWS])
        self.w1, self.w2 = 1 + 0.2 * torch.randn(DIM, device=DEV), 1 + 0.2 * torch.randn(DIM, device=DEV)
        self.mix, self.back, self.out = new(DIM, sum(self.cols)), new(HEADS * DV, DIM), new(DIM, ROWS)
        self.decay = torch.tensor([0.9, 0.99], device=DEV)

    def parameters(self):
        return dict(table=self.table, w1=self.w1, w2=self.w2, mix=self.mix, back=self.back, out=self.out)

    def parts(self, m):
        import paper_2112_02752_amd as emb
        at = (0, self.cols[0], self.cols[0] + self.cols[1])
        return [emb.Mat(m, cols=c, first=a) for a, c in zip(at, self.cols)]


def _batch(seed, lens):
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(seed)
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    n = int(offs[-1])
    ids = rng.integers(0, ROWS, n)
    targets = np.concatenate([ids[1:], [-1]])
    targets[offs[1:][offs[1:] > 0] - 1] = -1          # a sequence's last token has no next one
    weights = (-rng.random(n) / n).astype(np.float32)
    put = lambda t: torch.from_numpy(t).to(DEV)  # noqa: E731
    return emb.Batch(put(offs), put(ids), len(lens)), put(targets), put(weights), offs, ids, targets, weights


def test_a_training_step():
    import torch
    import paper_2112_02752_amd as emb
    say("training step of a block")
    m = Model(3)
    lens = [100, 0, 1, 130, 69]
    batch, targets, weights, offs, ids, ht, hw = _batch(4, lens)
    n, seed = int(offs[-1]), 77
    new = lambda *s: torch.empty(s, device=DEV)  # noqa: E731
    first = torch.randn((SEQS, GROUPS, DK, DV), device=DEV)
    tokens = emb.TokenLayer(m.tables, scale=SCALE, max_tokens=n, max_seqs=SEQS)
    norm1, norm2 = emb.Norm(m.w1, eps=EPS, max_rows=n), emb.Norm(m.w2, eps=EPS, drop=DROP, max_rows=n)
    attention = emb.LinearAttention(n, SEQS, HEADS, GROUPS, DK, DV)
    answers = emb.LogProbs(n, ROWS, scale=1.25)
    # forward
    rows, y1, proj, y = new(n, DIM), new(n, DIM), new(n, sum(m.cols)), new(n, HEADS * DV)
    tokens.forward(batch, rows)
    norm1.forward(rows, y1)
    torch.mm(y1, m.mix, out=proj)
    heads = emb.Heads(batch.offsets, *m.parts(proj), m.decay, heads=HEADS, groups=GROUPS, scale=DK ** -0.5, first=first)
    last = new(SEQS, GROUPS, DK, DV)
    attention.forward(heads, y, last)
    total, y2, logits = new(n, DIM), new(n, DIM), new(n, ROWS)
    norm2.forward(y @ m.back, y2, residual=rows, total=total, seed=seed)
    torch.mm(y2, m.out, out=logits)
    logp, entropy = new(n), new(n)
    # backward of sum(weights * logp), and the same in two calls with an entropy bonus below
    plain_logits = logits.clone()
    answers.train(logits, targets, logp, weights, logits, entropy=entropy)
    dlogits = logits
    dw = {k: torch.zeros_like(t) for k, t in m.parameters().items()}
    torch.mm(y2.t(), dlogits, out=dw["out"])
    dtotal, dbranch = new(n, DIM), new(n, DIM)
    norm2.backward(total, dlogits @ m.out.t(), dtotal, branch=dbranch, dweight=dw["w2"], seed=seed)
    torch.mm(y.t(), dbranch, out=dw["back"])
    dproj, dlast, dfirst = new(n, sum(m.cols)), torch.randn_like(last), torch.empty_like(first)
    attention.backward(heads, dbranch @ m.back.t(), *m.parts(dproj), dlast=dlast, dfirst=dfirst)
    torch.mm(y1.t(), dproj, out=dw["mix"])
    drows = new(n, DIM)
    norm1.backward(rows, dproj @ m.mix.t(), drows, arriving=dtotal, dweight=dw["w1"])
    tokens.table_grad(batch, drows, dw["table"])
    bonus = 0.01 * torch.randn(n, device=DEV)
    answers.forward(plain_logits, targets, logp, entropy=entropy)
    dlogits2 = new(n, ROWS)
    answers.backward(plain_logits, targets, weights, dlogits2, dentropy=bonus)
    torch.cuda.synchronize()

    # the same in 64 bits
    p = {k: t.detach().cpu().double().requires_grad_() for k, t in m.parameters().items()}
    s0 = first.cpu().double().requires_grad_()
    decay = m.decay.cpu().double()
    x = SCALE * p["table"][torch.from_numpy(ids)]
    rms = lambda t: t / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)  # noqa: E731
    q, k, v = torch.split(p["w1"] * rms(x) @ p["mix"], m.cols, 1)
    q, k, v = q.reshape(n, GROUPS, -1, DK), k.reshape(n, GROUPS, DK), v.reshape(n, GROUPS, DV)
    out, lasts = [], []
    for i in range(SEQS):
        s = s0[i]
        for t in range(offs[i], offs[i + 1]):
            s = decay[:, None, None] * s + k[t][:, :, None] * v[t][:, None]
            out.append(DK ** -0.5 * (q[t] @ s).reshape(1, -1))
        lasts.append(s)
    wide_y, wide_last = torch.cat(out), torch.stack(lasts)
    keep = torch.from_numpy(kept(n, DIM, DROP, seed)) * keep_scale(DROP)
    z = p["w2"] * rms(x + keep * (wide_y @ p["back"])) @ p["out"]
    l = torch.log_softmax(1.25 * z, 1)
    real = torch.from_numpy(ht >= 0)
    want = torch.where(real, l.gather(1, torch.from_numpy(np.maximum(ht, 0))[:, None])[:, 0], 0.0)
    want_h = -(l.exp() * l).sum(1)
    loss = (want * torch.from_numpy(hw).double()).sum() + (wide_last * dlast.cpu().double()).sum()
    grads = torch.autograd.grad(loss, list(p.values()) + [s0], retain_graph=True)
    for got, wide, what in ((y, wide_y, "y"), (last, wide_last, "last"), (logp, want, "logp"), (entropy, want_h, "entropy")):
        _close(got, wide, what)
    for (name, got), wide in zip(list(dw.items()) + [("first", dfirst)], grads):
        _close(got, wide, name)
    again = torch.autograd.grad((want * torch.from_numpy(hw).double()).sum() + (want_h * bonus.cpu().double()).sum(), z)
    _close(dlogits2, again[0], "dlogits with a bonus")


def test_prompts_and_single_tokens():
    """Sequences read as prompts and continued token by token in slots of a pool give the logits' alternatives that the
    whole sequences give."""
    import torch
    import paper_2112_02752_amd as emb
    m = Model(5)
    lens, more = [70, 1, 33, 200, 64], 4
    batch, _, _, offs, ids, _, _ = _batch(6, [x + more for x in lens])
    norm1, norm2 = emb.Norm(m.w1, eps=EPS), emb.Norm(m.w2, eps=EPS)
    tokens = emb.TokenLayer(m.tables, scale=SCALE)
    answers = emb.LogProbs(512, ROWS, top=3)

    def before(b):
        n = int(b.indices.numel())
        rows, y1 = torch.empty((n, DIM), device=DEV), torch.empty((n, DIM), device=DEV)
        tokens.forward(b, rows)
        norm1.forward(rows, y1)
        return rows, y1 @ m.mix

    def after(rows, y):
        n = rows.shape[0]
        y2 = torch.empty((n, DIM), device=DEV)
        norm2.forward(y @ m.back, y2, residual=rows)
        top, lp = torch.empty((n, 3), dtype=torch.int32, device=DEV), torch.empty((n, 3), device=DEV)
        answers.forward(y2 @ m.out, None, None, top_ids=top, top_logp=lp)
        return top, lp

    def whole(b, state=None):
        rows, proj = before(b)
        y = torch.empty((rows.shape[0], HEADS * DV), device=DEV)
        h = emb.Heads(b.offsets, *m.parts(proj), m.decay, heads=HEADS, groups=GROUPS, scale=DK ** -0.5)
        emb.LinearAttention(rows.shape[0], SEQS, HEADS, GROUPS, DK, DV, train=False).forward(h, y, state)
        return after(rows, y)

    want, want_lp = whole(batch)
    short = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    part = np.concatenate([ids[offs[i]:offs[i] + lens[i]] for i in range(SEQS)])
    put = lambda t: torch.from_numpy(t).to(DEV)  # noqa: E731
    state = torch.empty((SEQS, GROUPS, DK, DV), device=DEV)
    whole(emb.Batch(put(short), put(part), SEQS), state)
    pool = torch.full((9, GROUPS, DK, DV), 7.0, device=DEV)
    slots = np.array([8, 0, 3, 5, 1], dtype=np.int32)
    pool[put(slots).long()] = state
    one = put(np.arange(SEQS + 1, dtype=np.int32))
    for j in range(more):
        at = np.array([offs[i] + lens[i] + j for i in range(SEQS)])
        rows, proj = before(emb.Batch(one, put(ids[at]), SEQS))
        y = torch.empty((SEQS, HEADS * DV), device=DEV)
        emb.linear_attention_step(*m.parts(proj), m.decay, pool, y, heads=HEADS, groups=GROUPS, scale=DK ** -0.5,
                                  slots=put(slots))
        top, lp = after(rows, y)
        # (alternatives nearer to one another than both forms' error may change places: none are here)
        assert torch.equal(top, want[put(at)])
        assert float((lp - want_lp[put(at)]).abs().max()) <= 2 * NEAR * float(want_lp.abs().max())
    untouched = [i for i in range(9) if i not in slots]
    assert (pool[untouched] == 7.0).all()


def test_refusals_of_the_binding():
    """Tensors that do not fit their call, are of other types, or lie elsewhere."""
    import torch
    import paper_2112_02752_amd as emb
    x = lambda *shape: torch.zeros(shape, device="cuda")  # noqa: E731
    norm = emb.Norm(x(16), max_rows=4)
    for call in (lambda: norm.forward(x(4, 15), x(4, 16)), lambda: norm.forward(x(4, 16), x(3, 16)),
                 lambda: norm.forward(x(4, 16), x(4, 16).cpu()), lambda: norm.forward(x(4, 16), x(4, 32)[:, ::2]),
                 lambda: norm.forward(x(4, 16).half(), x(4, 16).half()),
                 lambda: norm.backward(x(5, 16), x(5, 16), dweight=x(16)),
                 lambda: norm.backward(x(4, 16), x(4, 16), dweight=x(15)),
                 lambda: norm.backward(x(4, 16), x(4, 16), dweight=x(16).cpu()),
                 lambda: norm.backward(x(4, 16), x(4, 16), dweight=x(16).double()),
                 lambda: emb.dropout(x(4, 16), x(4, 17), 0.5, 1)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: norm.forward(x(4, 16)), lambda: norm.forward(x(4, 16), x(4, 16).bfloat16()),
                 lambda: norm.forward(x(4, 16), x(4, 16), residual=x(4, 16).bfloat16()),
                 lambda: norm.forward(x(4, 16), x(4, 16), first_row=-1),
                 lambda: emb.dropout(x(4, 16), x(4, 16), 1.0, 1)):
        with pytest.raises(emb.EmbError):
            call()

    offsets = torch.tensor([0, 40, 70], dtype=torch.int32, device="cuda")
    q, k, v, decay, states = x(70, 32), x(70, 16), x(70, 24), x(2), x(2, 2, 8, 12)
    new = lambda **kw: emb.Heads(**{**dict(offsets=offsets, q=q, k=k, v=v, decay=decay, heads=4, groups=2), **kw})  # noqa: E731
    for kw in (dict(heads=3), dict(groups=3), dict(q=x(70, 31)), dict(q=x(69, 32)), dict(v=x(69, 24)), dict(k=x(70, 15)),
               dict(decay=x(3)), dict(decay=decay.cpu()), dict(decay=decay.double()), dict(first=x(3, 2, 8, 12)),
               dict(first=states.cpu()), dict(offsets=offsets.long())):
        with pytest.raises(ValueError):
            new(**kw)
    h = new()
    att, small, served = (emb.LinearAttention(t, 2, 4, 2, 8, 12, train=train)
                          for t, train in ((70, True), (69, True), (70, False)))
    y = x(70, 48)
    for call in (lambda: small.forward(h, y), lambda: att.forward(h, x(70, 47)), lambda: att.forward(h, y, last=x(1, 2, 8, 12)),
                 lambda: att.forward(h, y.cpu()), lambda: att.forward(h, y, last=states.cpu()),
                 lambda: att.backward(h, y, x(70, 32), x(70, 16), x(70, 24))):     # no forward yet
        with pytest.raises(ValueError):
            call()
    with pytest.raises(emb.EmbError):
        att.forward(h, y.bfloat16())
    att.forward(h, y)
    served.forward(h, y)
    with pytest.raises(ValueError, match="train"):
        served.backward(h, y, x(70, 32), x(70, 16), x(70, 24))
    with pytest.raises(ValueError):
        att.backward(h, y, x(70, 32), x(70, 16), x(70, 23))
    with pytest.raises(ValueError):
        att.backward(h, y, x(70, 32), x(70, 16), x(70, 24), dlast=x(2, 2, 8, 11))
    with pytest.raises(emb.EmbError):
        att.backward(h, y, q, x(70, 16), x(70, 24))          # over its queries

    one = lambda **kw: emb.linear_attention_step(**{**dict(  # noqa: E731
        q=x(3, 32), k=x(3, 16), v=x(3, 24), decay=decay, state=x(5, 2, 8, 12), y=x(3, 48), heads=4, groups=2), **kw})
    slots = torch.arange(3, dtype=torch.int32, device="cuda")
    one(slots=slots)
    for kw in (dict(slots=slots[:2]), dict(slots=slots.long()), dict(slots=slots.float()), dict(slots=slots.cpu()),
               dict(state=x(2, 2, 8, 12)), dict(state=x(5, 2, 8, 11)), dict(decay=x(1)), dict(y=x(3, 47)), dict(q=x(2, 32))):
        with pytest.raises(ValueError):
            one(**kw)
    torch.cuda.synchronize()
