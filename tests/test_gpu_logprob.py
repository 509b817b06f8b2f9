"""Log probabilities of given tokens, entropy, top alternatives and the logits'
gradient against plain forms in 64 bits: a few columns to more than registers
hold, odd widths, strides, masked tokens, ties, rows without a target or
without any token.

Tolerances (u = 2^-24), z' = scale (x - largest x):
 - z' (to the base of two) is rounded once, as is what it is multiplied with, its
   reference point is the same for a row, and the exponential is off by 2 u: e is off
   by (4 |z'| + 4) u of itself; a sum adds at most 16 * 8 values of a lane, 6
   exchanges and 16 wavefronts, and is referred to another point twice, by 5 u.  Where
   registers do not hold the row, a lane adds cols / 1024 values and is referred to
   another point at most once a vector of four (5 u): A = 160 + 2.25 cols / 1024
   roundings.  The logarithm of the sum is then off by B = sum of p (4 |z'| + 8) u +
   A u, and by 2 u of itself.
 - the entropy's second sum errs by its terms' (4 |z'| + 8 + 2 A) u.
 - a probability is off by R = (4 |z'| + 16) u + B of itself, and below 2^-126 is zero.
bf16 gradients are rounded: 2^-8 of them."""
import numpy as np
import pytest

from .block_plain import DEV, HALF, U, answers, answers_back, dt, host, say, strided, untouched, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _logits(rng, n, d, kind, gap, shift, masked=0.0, std=3.0):
    import torch
    x = torch.from_numpy((std * rng.standard_normal((n, d))).astype(np.float32)).to(dt(kind))
    if masked:
        out = torch.from_numpy(rng.random((n, d)) < masked)
        out[:, 0] = False
        x[out] = -float("inf")
    return strided(x, gap, shift, dt(kind))


class Bounds:
    def __init__(self, x, scale, every, entropy):
        with np.errstate(invalid="ignore"):
            z = np.abs(scale * (x - x.max(1, keepdims=True)))
        self.p = np.exp(every)
        self.z = np.where(self.p > 0, z, 0.0)
        adds = 160 + 2.25 * x.shape[1] / 1024
        log_sum = np.abs(every.max(1))
        self.log = (self.p * (4 * self.z + 8)).sum(1) * U + adds * U + 2 * U * log_sum
        self.entropy = self.log + (self.p * self.z * (4 * self.z + 8 + 2 * adds)).sum(1) * U + 4 * U * (entropy + log_sum)
        self.scale = scale
        self.every = np.where(self.p > 0, every, 0.0)
        self.h = entropy

    def logp(self, every, z):
        return self.log + 3 * U * np.abs(z) + 2 * U * np.abs(every)

    def grad(self, ids, dlogp, dentropy):
        share = (4 * self.z + 16) * U + self.log[:, None]
        real = (ids >= 0) & (ids < self.p.shape[1])
        dl = np.where(real, np.abs(dlogp), 0.0)[:, None]
        b = dl * (self.p * share + 1e-37) + dl * 2 * U * (np.arange(self.p.shape[1]) == ids[:, None])
        if dentropy is not None:
            dh = np.abs(dentropy)[:, None]
            b = b + dh * self.p * np.abs(self.every + self.h[:, None]) * share
            b = b + dh * (self.p * (2 * self.entropy[:, None] + 4 * U * (np.abs(self.every) + self.h[:, None] + self.z)) + 1e-35)
        return self.scale * b


# columns at the borders of the variants (vectors of 4 or 8 values; 128, 512, 2048, 4096, 8192, 16384 of them)
SIZES = [(1, 1, 0, 0), (3, 2, 1, 0), (5, 7, 0, 1), (9, 100, 0, 0), (4, 505, 0, 0), (3, 1001, 0, 3), (2, 1024, 8, 0),
         (3, 2040, 1, 0), (5, 4088, 0, 0), (2, 4099, 0, 1), (3, 8185, 0, 0), (2, 16001, 1, 0), (3, 16390, 8, 0),
         (2, 32761, 0, 0), (2, 40003, 0, 5), (3, 65530, 0, 0), (2, 70001, 0, 0), (2, 131071, 0, 0), (2, 150001, 1, 0),
         (300, 33, 0, 0), (0, 50, 0, 0)]


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("n,d,gap,shift", SIZES)
def test_log_probabilities(n, d, gap, shift, kind):
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(n * 13 + d)
    scale, top, bits = [1.0, 0.8, 1.25][d % 3], min(d, [0, 5, 32, 1][(n + d) % 4]), [32, 64][d % 2]
    say("log probabilities", kind, n, d, gap, shift, scale, top, bits)
    x, _ = _logits(rng, n, d, kind, gap, shift, masked=[0.0, 0.3, 0.9][n % 3])
    hx = host(x)
    ids = rng.integers(0, d, n)
    ids[1::4] = [-1, d, d + 5, -(2 ** 31)][(n + d) % 4]
    if n:
        ids[0] = 0
    dev_ids = torch.from_numpy(ids.astype(np.int32 if bits == 32 else np.int64)).to(DEV)
    dlogp, dentropy = rng.standard_normal(n), rng.standard_normal(n)
    dl, dh = (torch.from_numpy(t.astype(np.float32)).to(DEV) for t in (dlogp, dentropy))
    dlogp, dentropy = host(dl), host(dh)
    answer = emb.LogProbs(max(n, 1), d, top=top, scale=scale)
    f32 = float(np.float32(scale))
    logp, entropy, logp2, entropy2 = (torch.full((n,), 7.0, device=DEV) for _ in range(4))
    top_ids, top_logp = torch.full((n, top), -7, dtype=torch.int32, device=DEV), torch.full((n, top), 7.0, device=DEV)
    answer.forward(x, dev_ids, logp, entropy=entropy, top_ids=top_ids, top_logp=top_logp)
    dx, buf = _logits(rng, n, d, kind, gap, shift)
    answer.backward(x, dev_ids, dl, dx, dentropy=dh)
    dx2, buf2 = _logits(rng, n, d, kind, gap + 1, shift)     # rows that lie otherwise
    answer.train(x, dev_ids, logp2, dl, dx2, entropy=entropy2)
    torch.cuda.synchronize()
    if n == 0:
        return
    want, want_h, every, order = answers(hx, ids, f32, top)
    bounds = Bounds(hx, f32, every, want_h)
    real = (ids >= 0) & (ids < d)
    with np.errstate(invalid="ignore"):
        z = f32 * (hx - hx.max(1, keepdims=True))
    at = (np.arange(n), np.where(real, ids, 0))
    gone = real & np.isinf(z[at])
    assert np.array_equal(host(logp)[gone], np.full(gone.sum(), -np.inf))
    sure = ~gone
    # (gradients that lie otherwise take another variant, whose sums have another order)
    for l, h, name in ((logp, entropy, "forward"), (logp2, entropy2, "train")):
        within(host(l)[sure], want[sure], np.where(real, bounds.logp(every[at], z[at]), 0)[sure], f"logp, {name}")
        within(h, want_h, bounds.entropy, f"entropy, {name}")
    if top:
        assert np.array_equal(top_ids.cpu().numpy(), order)
        rows = np.arange(n)[:, None]
        got, wl, zl = host(top_logp), every[rows, order], z[rows, order]
        some = ~np.isinf(wl)
        assert (got[~some] == -np.inf).all()
        limit = bounds.log[:, None] + 3 * U * np.abs(zl) + 2 * U * np.abs(wl)
        within(got[some], wl[some], limit[some], "top logp")
    # in place
    other = x.clone() if gap == 0 else _logits(rng, n, d, kind, gap, shift)[0].copy_(x)
    answer.train(x, dev_ids, None, dl, x)
    answer.backward(other, dev_ids, dl, other, dentropy=dh)
    torch.cuda.synchronize()
    for got, g, name in ((dx, dentropy, "dlogits"), (dx2, None, "dlogits of one pass"), (other, dentropy, "in place"),
                         (x, None, "of one pass in place")):
        grad = answers_back(every, ids, want_h, f32, dlogp, g)
        within(got, grad, bounds.grad(ids, dlogp, g) + HALF[kind] * np.abs(grad), name)
    assert untouched(dx, buf, gap, shift) and untouched(dx2, buf2, gap + 1, shift)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [50, 3000, 20000, 300000])
def test_rows_of_special_logits(d, kind):
    """No token that can be, one, ties everywhere, infinities, NaN: each row for itself."""
    import torch
    import paper_2112_02752_amd as emb
    inf, nan = float("inf"), float("nan")
    x = torch.zeros((7, d), device=DEV)
    x[0] = -inf
    x[1] = -inf
    x[1, d - 1] = 2.0
    x[2] = 1.5
    x[3, 10] = inf
    x[4, 20] = nan
    x[5] = -inf
    x[5, 30] = nan
    x[6, 3], x[6, 7] = -0.0, 5.0
    x = x.to(dt(kind))
    ids = torch.tensor([3, d - 1, 4, 5, 6, 7, 7], device=DEV)
    logp, entropy = torch.empty(7, device=DEV), torch.empty(7, device=DEV)
    top_ids, top_logp = torch.empty((7, 4), dtype=torch.int32, device=DEV), torch.empty((7, 4), device=DEV)
    answer = emb.LogProbs(7, d, top=4)
    answer.forward(x, ids, logp, entropy=entropy, top_ids=top_ids, top_logp=top_logp)
    dx, dx2 = torch.empty_like(x), torch.empty_like(x)
    one = torch.ones(7, device=DEV)
    answer.backward(x, ids, one, dx, dentropy=one)
    answer.train(x, ids, None, one, dx2)
    logp, entropy, top_ids, top_logp, dx, dx2 = (t.cpu().float() for t in (logp, entropy, top_ids, top_logp, dx, dx2))
    assert logp[0] == -inf and entropy[0] == 0 and (dx[0] == 0).all() and (dx2[0] == 0).all()
    assert top_ids[0].tolist() == [0, 1, 2, 3] and (top_logp[0] == -inf).all()
    assert logp[1] == 0 and entropy[1] == 0 and (dx[1] == 0).all() and (dx2[1] == 0).all()
    assert top_ids[1].tolist() == [d - 1, 0, 1, 2] and top_logp[1].tolist() == [0, -inf, -inf, -inf]
    # (adding equal values: 160 + 2.25 d / 1024 roundings)
    near = (170 + 2.25 * d / 1024) * U
    assert abs(logp[2] + np.log(d)) < near + 2 * U * np.log(d) and abs(entropy[2] - np.log(d)) < near + 2 * U * np.log(d)
    assert top_ids[2].tolist() == [0, 1, 2, 3]
    for i in (3, 4, 5):
        assert torch.isnan(logp[i]) and torch.isnan(entropy[i]) and torch.isnan(dx[i]).all() and torch.isnan(dx2[i]).all()
    assert top_ids[3, 0] == 10 and top_ids[4].tolist() == [20, 0, 1, 2] and top_ids[5].tolist() == [30, 0, 1, 2]
    assert top_ids[6].tolist() == [7, 0, 1, 2]


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [40, 900, 30000])
def test_most_alternatives_among_ties(d, kind):
    """32 alternatives of rows of few different values, rising, falling."""
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(d)
    x = torch.from_numpy(rng.integers(0, 3, (6, d)).astype(np.float32))
    x[1] = torch.arange(d) / 8.0
    x[2] = -torch.arange(d) / 8.0
    x[3] = torch.from_numpy((rng.random(d) < 20 / d).astype(np.float32))
    x[4, :] = torch.where(torch.arange(d) % 64 == 5, 3.0, -1.0)        # all in one lane's columns, or few
    x = x.to(dt(kind)).to(DEV)
    top_ids, top_logp = torch.empty((6, 32), dtype=torch.int32, device=DEV), torch.empty((6, 32), device=DEV)
    emb.LogProbs(6, d, top=32).forward(x, None, None, top_ids=top_ids, top_logp=top_logp)
    want = np.argsort(-host(x), axis=1, kind="stable")[:, :32]
    assert np.array_equal(top_ids.cpu().numpy(), want)


def test_gradients_against_differences():
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(4)
    n, d, scale = 3, 6, 0.75
    x, dl, dh = rng.standard_normal((n, d)), rng.standard_normal(n), rng.standard_normal(n)
    x, dl, dh = (t.astype(np.float32).astype(np.float64) for t in (x, dl, dh))
    ids = np.array([2, -1, 5])
    put = lambda t: torch.from_numpy(t.astype(np.float32)).to(DEV)  # noqa: E731
    answer = emb.LogProbs(n, d, scale=scale)
    logp, dx, one = torch.empty(n, device=DEV), torch.empty((n, d), device=DEV), torch.empty((n, d), device=DEV)
    dev = torch.from_numpy(ids).to(DEV)
    answer.forward(put(x), dev, logp)
    answer.backward(put(x), dev, put(dl), dx, dentropy=put(dh))
    answer.train(put(x), dev, None, put(dl), one)
    answer.forward(put(x), dev, logp)
    only = torch.empty((n, d), device=DEV)
    answer.backward(put(x), None, None, only, dentropy=put(dh))

    def loss(x, dl, dh):
        l, h, _, _ = answers(x, ids, scale)
        return (dl * l).sum() + (dh * h).sum()

    for got, a, b in ((dx, dl, dh), (one, dl, 0 * dh), (only, 0 * dl, dh)):
        got = host(got)
        for at in np.ndindex(x.shape):
            ends = []
            for e in (1e-4, -1e-4):
                moved = x.copy()
                moved[at] += e
                ends.append(loss(moved, a, b))
            # (1e-8 of a third derivative below 10, 1e-15 / 1e-4; fp32: 100 u of values of about one)
            assert abs(got[at] - (ends[0] - ends[1]) / 2e-4) < 1e-5


def test_streams_and_graphs():
    import torch
    import paper_2112_02752_amd as emb
    torch.manual_seed(2)
    n, d = 40, 5001
    x = (3 * torch.randn((n, d), device=DEV)).bfloat16()
    ids = torch.randint(0, d, (n,), device=DEV)
    w, wh = -torch.rand(n, device=DEV), torch.randn(n, device=DEV)
    answer = emb.LogProbs(n, d, top=3)

    def step():
        out = [torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty((n, 3), dtype=torch.int32, device=DEV),
               torch.empty((n, 3), device=DEV), torch.empty_like(x), torch.empty_like(x)]
        answer.forward(x, ids, out[0], entropy=out[1], top_ids=out[2], top_logp=out[3])
        answer.backward(x, ids, w, out[4], dentropy=wh)
        answer.train(x, ids, None, w, out[5])
        return out

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(3 * torch.randn((n, d), device=DEV))
        eager = step()
        for t in held:
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), i


def test_binding_refusals():
    import torch
    import paper_2112_02752_amd as emb
    x, ids, v = torch.zeros((4, 10), device=DEV), torch.zeros(4, dtype=torch.long, device=DEV), torch.zeros(4, device=DEV)
    a = emb.LogProbs(4, 10, top=2)
    with pytest.raises(ValueError, match="follows"):
        a.backward(x, ids, v, x)
    with pytest.raises(ValueError, match="top"):
        a.forward(x, ids, v)
    a = emb.LogProbs(4, 10)
    for bad in (ids[:3], ids.float(), ids[None], ids.cpu(), torch.zeros(8, dtype=torch.long, device=DEV)[::2],
                ids.to(torch.int16)):
        with pytest.raises(ValueError):
            a.forward(x, bad, v)
    for bad in (v.double(), v[:3], v.cpu()):
        with pytest.raises(ValueError):
            a.forward(x, ids, bad)
    with pytest.raises(ValueError):
        a.forward(x[:, :9], ids, v)
    with pytest.raises(ValueError, match="more rows"):
        a.forward(torch.zeros((5, 10), device=DEV), None, None)
    with pytest.raises(emb.EmbError):
        a.forward(x, None, v)
