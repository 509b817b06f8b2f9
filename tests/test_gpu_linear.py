"""Linear attention with a decay for each key head against the recurrence in 64
bits: forward, backward, single tokens; ragged and empty sequences, one
position to several segments, shared heads, odd widths, strides.

Tolerances (u = 2^-24).  Every result is a sum of terms, each the product of
rows and powers of the decay; with |.| for the same sums of magnitudes:
 - a term of fp32 rows is rounded when its products and sums are formed: at
   most T sums over the positions and one width over the columns, on the matrix
   units, whose inner sums need not round to nearest (2 u each), and two
   roundings (power, product) for each chunk of 32 or 64 positions: (T + width + 32) 2u |.|
   with T the longest sequence and the wider head;
 - bf16 rows: a term within a chunk has its weight rounded to bf16, one from
   before it the state, 2^-8 |.|; that has got rows times weights with 16 bits
   since the segment's begin, 2^-16 |.|; the result is rounded, 2^-8 of it.  States that are
   kept get weighted rows with 24 bits: as fp32, u more.
"""
import numpy as np
import pytest

from .block_plain import DEV, HALF, U, dt, host, linear, linear_back, say, strided, untouched, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _offsets(rng, n, m, empty=0.0):
    cuts = np.sort(rng.integers(0, n + 1, m - 1))
    for i in np.nonzero(rng.random(m - 1) < empty)[0]:
        cuts[i] = cuts[i - 1] if i else 0
    return np.concatenate([[0], cuts, [n]]).astype(np.int32)


def _decay(groups):
    """Rates from forgetting at once to never."""
    return np.array([0.97, 0.0, 1.0, 0.5, 0.998, 0.9, 0.75, 0.99])[np.arange(groups) % 8]


class Batch:
    def __init__(self, kind, n, offs, heads, groups, dk, dv, gap=0, shift=0, first=True, seed=0, pad=0):
        import torch
        import paper_2112_02752_amd as emb
        rng = np.random.default_rng(seed)
        self.kind, self.n, self.offs, self.sizes = kind, n, offs, (heads, groups, dk, dv)
        m, rows = len(offs) - 1, n + pad
        self.scale = 1 / np.sqrt(dk)
        put = lambda cols: strided(torch.from_numpy(  # noqa: E731
            rng.standard_normal((rows, cols)).astype(np.float32)).to(dt(kind)), gap, shift, dt(kind))
        (self.q, _), (self.k, _), (self.v, _) = put(heads * dk), put(groups * dk), put(groups * dv)
        (self.y, self.ybuf), (self.dy, _) = put(heads * dv), put(heads * dv)
        (self.dq, self.qbuf), (self.dk, self.kbuf), (self.dv, self.vbuf) = (put(heads * dk), put(groups * dk),
                                                                          put(groups * dv))
        state = lambda std: torch.from_numpy(  # noqa: E731
            (std * rng.standard_normal((m, groups, dk, dv))).astype(np.float32)).to(DEV)
        self.first, self.dlast = (state(2.0), state(1.0)) if first else (None, None)
        self.last, self.dfirst = state(9.0), state(9.0)
        self.decay = torch.from_numpy(_decay(groups).astype(np.float32)).to(DEV)
        self.heads = emb.Heads(torch.from_numpy(offs).to(DEV), self.q, self.k, self.v, self.decay, heads=heads,
                               groups=groups, scale=self.scale, first=self.first)
        self.attention = emb.LinearAttention(rows, m, heads, groups, dk, dv)
        self.gap, self.shift = gap, shift

    def run(self, stream=None):
        self.attention.forward(self.heads, self.y, self.last, stream=stream)
        self.attention.backward(self.heads, self.dy, self.dq, self.dk, self.dv, dlast=self.dlast, dfirst=self.dfirst,
                                stream=stream)

    def outputs(self):
        return [t.clone() for t in (self.y, self.last, self.dq, self.dk, self.dv, self.dfirst)]

    def check(self):
        h, g, dk, dv = self.sizes
        n, r = self.n, h // g
        scale, decay = float(np.float32(self.scale)), host(self.decay)
        q, k, v = host(self.q)[:n].reshape(n, g, r, dk), host(self.k)[:n].reshape(n, g, dk), \
            host(self.v)[:n].reshape(n, g, dv)
        dy = host(self.dy)[:n].reshape(n, g, r, dv)
        first, dlast = (host(t) if t is not None else None for t in (self.first, self.dlast))
        mag = lambda t: np.abs(t) if t is not None else None  # noqa: E731
        y, last, every = linear(self.offs, q, k, v, decay, scale, first)
        dq, dkey, dval, dfirst = linear_back(self.offs, q, k, v, decay, scale, every, dy, dlast)
        ya, lasta, everya = linear(self.offs, mag(q), mag(k), mag(v), decay, scale, mag(first))
        dqa, dka, dva, dfirsta = linear_back(self.offs, mag(q), mag(k), mag(v), decay, scale, everya, mag(dy), mag(dlast))
        longest = int((self.offs[1:] - self.offs[:-1]).max()) if len(self.offs) > 1 else 0
        near = (longest * r + max(dk, dv) + 32) * 2 * U
        low = self.kind == "bf16"
        for got, want, size, name in ((self.y, y, ya, "y"), (self.dq, dq, dqa, "dq"), (self.dk, dkey, dka, "dk"),
                                      (self.dv, dval, dva, "dv")):
            bound = (near + (2.0 ** -8 + 2.0 ** -16 if low else 0)) * size + HALF[self.kind] * np.abs(want)
            within(host(got)[:n].reshape(want.shape), want, bound, name)
        for got, want, size, name in ((self.last, last, lasta, "last"), (self.dfirst, dfirst, dfirsta, "dfirst")):
            within(got, want, (near + U) * size, name)
        for t, buf in ((self.y, self.ybuf), (self.dq, self.qbuf), (self.dk, self.kbuf), (self.dv, self.vbuf)):
            assert untouched(t, buf, self.gap, self.shift)


SIZES = [
    # tokens, sequences, heads, groups, dk, dv, gap, shift
    (1, 1, 1, 1, 1, 1, 0, 0), (5, 3, 2, 1, 8, 8, 0, 0), (63, 1, 2, 2, 16, 24, 0, 0), (64, 1, 1, 1, 32, 64, 8, 0),
    (65, 2, 1, 1, 64, 65, 0, 0), (130, 2, 4, 2, 40, 72, 0, 0), (257, 1, 1, 1, 65, 8, 0, 1), (700, 3, 3, 3, 64, 128, 0, 0),
    (600, 1, 1, 1, 17, 5, 1, 0), (1200, 5, 8, 2, 128, 128, 0, 0), (530, 2, 2, 1, 256, 256, 0, 0),
    (300, 2, 2, 1, 200, 33, 0, 0), (290, 1, 4, 1, 24, 250, 0, 0), (1501, 23, 6, 2, 40, 72, 0, 0),
    (100, 100, 2, 1, 16, 16, 0, 0), (513, 1, 1, 1, 8, 8, 0, 0), (0, 3, 2, 1, 8, 16, 0, 0)]


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("n,m,heads,groups,dk,dv,gap,shift", SIZES)
def test_linear_attention(n, m, heads, groups, dk, dv, gap, shift, kind):
    say("linear attention", kind, n, m, heads, groups, dk, dv, gap, shift)
    rng = np.random.default_rng(n + dk)
    b = Batch(kind, n, _offsets(rng, n, m, 0.2), heads, groups, dk, dv, gap, shift, first=(n + dk) % 2 == 0, seed=n)
    b.run()
    b.check()


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_longer_segments(kind):
    """So many key heads and tokens that the segments grow."""
    say("longer segments", kind)
    b = Batch(kind, 9000, np.array([0, 8, 8500, 8500, 9000], dtype=np.int32), 64, 64, 8, 8, seed=2)
    b.run()
    b.check()


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_rows_behind_the_last_sequence(kind):
    b = Batch(kind, 300, np.array([0, 290, 300], dtype=np.int32), 2, 1, 16, 16, pad=500, seed=3)
    for t in (b.q, b.k, b.v, b.dy):
        t[300:] = float("nan")
    held = [t[300:].clone() for t in (b.y, b.dq, b.dk, b.dv)]
    b.run()
    b.check()
    for t, h in zip((b.y, b.dq, b.dk, b.dv), held):
        assert (t[300:] == h).all()


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_infinities_stay_in_their_sequence(kind):
    import torch
    offs = np.array([0, 200, 201, 700, 900], dtype=np.int32)
    b = Batch(kind, 900, offs, 4, 2, 32, 32, seed=4)
    b.run()
    want = b.outputs()
    b.q[250], b.k[300, 3], b.v[400, 7], b.dy[690] = float("nan"), float("inf"), float("-inf"), float("nan")
    b.run()
    for x, y in zip(want, b.outputs()):
        if x.dim() == 2:
            assert torch.equal(x[:201], y[:201]) and torch.equal(x[700:], y[700:])
        else:
            assert torch.equal(x[[0, 1, 3]], y[[0, 1, 3]])
    # and results before the chunk of the first of them are as they were
    assert torch.equal(want[0][201:201 + 32], b.y[201:201 + 32])


def test_gradients_against_differences():
    n, offs, h, g, dk, dv = 9, np.array([0, 6, 6, 9], dtype=np.int32), 2, 1, 3, 2
    b = Batch("fp32", n, offs, h, g, dk, dv, seed=6)
    b.run()
    shape = lambda t, *s: host(t).reshape(s)  # noqa: E731
    args = [shape(b.q, n, g, h // g, dk), shape(b.k, n, g, dk), shape(b.v, n, g, dv), host(b.first)]
    dy, dlast, decay = shape(b.dy, n, g, h // g, dv), host(b.dlast), host(b.decay)

    def loss(q, k, v, first):
        y, last, _ = linear(offs, q, k, v, decay, float(np.float32(b.scale)), first)
        return (y * dy).sum() + (last * dlast).sum()

    for i, got in enumerate((b.dq, b.dk, b.dv, b.dfirst)):
        got = host(got).reshape(args[i].shape)
        for at in np.ndindex(got.shape):
            ends = []
            for d in (1e-4, -1e-4):
                moved = [a.copy() for a in args]
                moved[i][at] += d
                ends.append(loss(*moved))
            # (the loss is of degree one in each input: differences are exact but for 1e-15 / 1e-4; fp32 gradients of
            # about 10 are off by some u each of 9 positions)
            assert abs(got[at] - (ends[0] - ends[1]) / 2e-4) < 2e-5, (i, at)


def _step_batch(kind, n, slots, heads, groups, dk, dv, gap, shift, seed):
    import torch
    rng = np.random.default_rng(seed)
    put = lambda cols: strided(torch.from_numpy(  # noqa: E731
        rng.standard_normal((n, cols)).astype(np.float32)).to(dt(kind)), gap, shift, dt(kind))
    pool = torch.from_numpy((3 * rng.standard_normal((slots, groups, dk, dv))).astype(np.float32)).to(DEV)
    where = rng.permutation(slots)[:n].astype(np.int32)
    where[rng.random(n) < 0.2] = -1
    if n > 2:
        where[1] = slots            # just outside
        where[2] = np.int32(2 ** 31 - 1)
    return put(heads * dk)[0], put(groups * dk)[0], put(groups * dv)[0], put(heads * dv), pool, where


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("n,slots,heads,groups,dk,dv,gap,shift", [
    (1, 1, 1, 1, 1, 1, 0, 0), (5, 9, 2, 1, 8, 8, 0, 0), (17, 40, 12, 12, 128, 128, 0, 0), (9, 9, 6, 2, 40, 72, 8, 0),
    (7, 8, 8, 1, 64, 33, 1, 3), (6, 6, 4, 1, 256, 256, 0, 0), (3, 5, 7, 1, 200, 250, 0, 1), (130, 131, 2, 2, 16, 4, 0, 0),
    (0, 3, 2, 1, 8, 8, 0, 0)])
def test_single_tokens(n, slots, heads, groups, dk, dv, gap, shift, kind):
    """One step: sums of dk products, 2 u each and as many for the state's two roundings."""
    import torch
    import paper_2112_02752_amd as emb
    say("single tokens", kind, n, slots, heads, groups, dk, dv)
    q, k, v, (y, buf), pool, where = _step_batch(kind, n, slots, heads, groups, dk, dv, gap, shift, n + dk)
    decay = torch.from_numpy(_decay(groups).astype(np.float32)).to(DEV)
    r, before, scale = heads // groups, host(pool), 0.3
    emb.linear_attention_step(q, k, v, decay, pool, y, heads=heads, groups=groups, scale=scale,
                              slots=torch.from_numpy(where).to(DEV))
    torch.cuda.synchronize()
    hq, hk, hv, g = host(q).reshape(n, groups, r, dk), host(k).reshape(n, groups, dk), host(v).reshape(n, groups, dv), host(decay)
    after, after_size = before.copy(), np.abs(before)
    want, size = np.zeros((n, groups, r, dv)), np.zeros((n, groups, r, dv))
    for i, a in enumerate(where):
        if 0 <= a < slots:
            outer = hk[i][:, :, None] * hv[i][:, None]
            after[a] = g[:, None, None] * before[a] + outer
            after_size[a] = g[:, None, None] * np.abs(before[a]) + np.abs(outer)
            want[i] = np.float32(scale) * (hq[i] @ after[a])
            size[i] = np.float32(scale) * (np.abs(hq[i]) @ after_size[a])
    within(pool, after, 3 * U * after_size, "state")
    assert np.array_equal(host(pool)[~np.isin(np.arange(slots), where)], before[~np.isin(np.arange(slots), where)])
    within(host(y).reshape(want.shape), want, (dk + 8) * 2 * U * size + HALF[kind] * np.abs(want), "y")
    assert untouched(y, buf, gap, shift)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_tokens_one_by_one_continue_a_prompt(kind):
    """Prompts by the whole form, then tokens one by one, as the whole form of all of them: y within both forms' bounds,
    of which the whole one's is the larger (the single steps' is for 300 positions of state)."""
    import torch
    import paper_2112_02752_amd as emb
    n, extra, h, g, dk, dv = 300, 5, 4, 2, 32, 64
    b = Batch(kind, n + extra, np.array([0, n + extra], dtype=np.int32), h, g, dk, dv, first=False, seed=7)
    b.run()
    whole = b.y.clone()
    short = emb.Heads(torch.tensor([0, n], dtype=torch.int32, device=DEV), b.q[:n], b.k[:n], b.v[:n], b.decay, heads=h,
                      groups=g, scale=b.scale)
    state = torch.empty((1, g, dk, dv), device=DEV)
    b.attention.forward(short, b.y[:n], state)
    assert torch.equal(b.y[:n], whole[:n])
    q, k, v = (host(t) for t in (b.q, b.k, b.v))
    _, _, every = linear(np.array([0, n + extra]), np.abs(q).reshape(-1, g, h // g, dk), np.abs(k).reshape(-1, g, dk),
                         np.abs(v).reshape(-1, g, dv), host(b.decay), 1.0)
    for i in range(n, n + extra):
        y = torch.empty((1, h * dv), dtype=dt(kind), device=DEV)
        emb.linear_attention_step(b.q[i:i + 1], b.k[i:i + 1], b.v[i:i + 1], b.decay, state, y, heads=h, groups=g,
                                  scale=b.scale)
        size = b.scale * (np.abs(q[i]).reshape(g, h // g, dk) @ every[i]).reshape(1, -1)
        near = 2 * (305 + 64 + 32) * 2 * U + (2.0 ** -8 + 2.0 ** -16 if kind == "bf16" else 0)
        within(y, host(whole[i:i + 1]), near * size + 2 * HALF[kind] * np.abs(host(whole[i:i + 1])), i)


def test_streams_objects_and_graphs():
    import torch
    torch.manual_seed(1)
    offs = np.array([0, 600, 700, 1300], dtype=np.int32)
    a, b = (Batch("bf16", 1300, offs, 4, 2, 64, 64, seed=s) for s in (8, 9))
    a.run()
    b.run()
    want = a.outputs(), b.outputs()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):             # two at once
        for x in (a, b):
            for t in (x.y, x.dq, x.dk, x.dv, x.last, x.dfirst):
                t.fill_(5)
        torch.cuda.synchronize()
        a.run()
        b.run(stream=side)
        torch.cuda.synchronize()
        for x, w in zip((a, b), want):
            assert all(torch.equal(s, t) for s, t in zip(x.outputs(), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for i in range(3):
        a.q.copy_(torch.randn_like(a.q.float()))
        a.run()
        eager = a.outputs()
        for t in (a.y, a.dq, a.dk, a.dv, a.last, a.dfirst):
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(eager, a.outputs())), i
