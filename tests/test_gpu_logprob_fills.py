"""Log probabilities where logits are masked by large finite numbers, as masks often are: a few tokens left, rows of
nothing but the fill, the fill in a part of a row that one wavefront or one lane has, large logits of either sign, and
the largest and smallest scales.

Tolerances are those of test_gpu_logprob.py (Bounds): z' = scale (x - largest x) has at most four roundings (of the
difference, of its product, two of scale log2(e)), and a power that does not underflow is off by (4 |z'| + 4) u; what a
power of zero multiplies adds nothing.  The 64-bit form takes the same differences, so a filled token's probability
is zero there too.  Where scale times a logit is past fp32's range, so are finite log probabilities: minus infinity is
the nearest."""
import numpy as np
import pytest

from .block_plain import DEV, HALF, U, answers_back, dt, host, say, strided, within
from .test_gpu_logprob import Bounds

pytestmark = pytest.mark.gpu

F32 = float(np.finfo(np.float32).max)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def answers(x, ids, scale, top):
    """As the other files', of differences: 1e15 + log d has not the digits of log d in 64 bits either."""
    z = scale * (x - x.max(1, keepdims=True))
    every = z - np.log(np.exp(z).sum(1, keepdims=True))
    p = np.exp(every)
    real = (ids >= 0) & (ids < x.shape[1])
    logp = np.where(real, every[np.arange(len(ids)), np.where(real, ids, 0)], 0.0)
    return logp, -np.where(p > 0, p * every, 0.0).sum(1), every, np.argsort(-x, axis=1, kind="stable")[:, :top]


def _rows(rng, d, fill):
    """Ordinary rows of which tokens are filled: all but a few, all but one, all, the first ones, the last ones, every
    64th eight (a lane's share), all but every 64th eight, and rows whose ordinary logits lie about the fill's negative."""
    at = np.arange(d)
    x = 3 * rng.standard_normal((9, d))
    few = rng.permutation(d)[:5]
    x[0, ~np.isin(at, few)] = fill
    x[1, at != few[0]] = fill
    x[2] = fill
    x[3, at < d // 2] = fill
    x[4, at >= d // 2] = fill
    x[5, at // 8 % 64 == 3] = fill
    x[6, at // 8 % 64 != 0] = fill
    x[7, at // 512 % 16 == 1] = fill          # (a wavefront's share of eights)
    x[8] = -fill
    x[8, at % 3 == 1] = fill
    return x


def _check(hx, x, ids, scale, top, kind, gap):
    """Forward, backward and both in one pass against 64 bits."""
    import torch
    import paper_2112_02752_amd as emb
    n, d = hx.shape
    rng = np.random.default_rng(d)
    # (gradients of the logits below about 64, whatever the scale)
    unit = 2.0 ** min(0, 6 - int(np.ceil(np.log2(scale))))
    dl, dh = (torch.from_numpy((unit * rng.standard_normal(n)).astype(np.float32)).to(DEV) for _ in range(2))
    dev_ids = torch.from_numpy(ids).to(DEV)
    answer = emb.LogProbs(n, d, top=top, scale=scale)
    scale = float(np.float32(scale))
    logp, entropy, logp2, entropy2 = (torch.full((n,), 7.0, device=DEV) for _ in range(4))
    top_ids, top_logp = torch.full((n, top), -7, dtype=torch.int32, device=DEV), torch.full((n, top), 7.0, device=DEV)
    answer.forward(x, dev_ids, logp, entropy=entropy, top_ids=top_ids, top_logp=top_logp)
    dx, dx2 = torch.empty_like(x), strided(hx, gap + 1, 0, dt(kind))[0]
    answer.backward(x, dev_ids, dl, dx, dentropy=dh)
    answer.train(x, dev_ids, logp2, dl, dx2, entropy=entropy2)
    same = strided(hx, gap, 0, dt(kind))[0]
    answer.train(same, dev_ids, None, dl, same)
    torch.cuda.synchronize()
    want, want_h, every, order = answers(hx, ids, scale, top)
    bounds = Bounds(hx, scale, every, want_h)
    z = scale * (hx - hx.max(1, keepdims=True))
    real = (ids >= 0) & (ids < d)
    at = (np.arange(n), np.where(real, ids, 0))

    def logs(got, want, z, limit, what):
        got, past = host(got), want < -F32 * (1 - 2 * U)
        assert not np.isnan(got).any(), what
        assert (got[past] <= -F32 * (1 - 8 * U)).all(), what
        within(got[~past], want[~past], limit[~past], what)

    for l, h, name in ((logp, entropy, "forward"), (logp2, entropy2, "train")):
        logs(l, want, z[at], np.where(real, bounds.logp(every[at], z[at]), 0), f"logp, {name}")
        within(h, want_h, bounds.entropy, f"entropy, {name}")
    assert np.array_equal(top_ids.cpu().numpy(), order)
    rows = np.arange(n)[:, None]
    wl, zl = every[rows, order], z[rows, order]
    logs(top_logp, wl, zl, bounds.log[:, None] + 3 * U * np.abs(zl) + 2 * U * np.abs(wl), "top logp")
    dlogp, dentropy = host(dl), host(dh)
    for got, g, name in ((dx, dentropy, "dlogits"), (dx2, None, "of one pass, lying otherwise"),
                         (same, None, "of one pass in place")):
        grad = answers_back(every, ids, want_h, scale, dlogp, g)
        within(got, grad, bounds.grad(ids, dlogp, g) + HALF[kind] * np.abs(grad), name)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("fill", [-1e9, -1e10, -1e15, -1e30, "lowest"])
@pytest.mark.parametrize("d,gap", [(7, 0), (700, 0), (3000, 1), (5000, 8), (20000, 0), (50001, 1), (70000, 0), (120000, 0),
                                   (210000, 8)])
def test_finite_masks(d, gap, fill, kind):
    import torch
    scale = [0.8, 1.0, 1.25][(d + len(str(fill))) % 3]
    say("finite masks", kind, d, gap, fill, scale)
    rng = np.random.default_rng(d)
    value = float(torch.finfo(dt(kind)).min) if fill == "lowest" else fill
    x = _rows(rng, d, value)
    view, _ = strided(torch.from_numpy(np.clip(x, -F32, F32).astype(np.float32)).to(dt(kind)), gap, 0, dt(kind))
    hx = host(view)
    ids = np.concatenate([hx[:7].argmax(1), [0, d - 1]]).astype(np.int64)
    ids[3], ids[5] = d // 2, -1
    _check(hx, view, ids, scale, min(d, 4), kind, gap)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [700, 3000, 50001, 210000])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 100.0, 1e10, 3e38])
def test_scales(d, scale, kind):
    import torch
    say("scales", kind, d, scale)
    rng = np.random.default_rng(d + 1)
    x = np.round(8 * rng.standard_normal((3, d))) / 4
    x[1] *= 2.0 ** 40
    x[2, 1:] = -1e30
    x[2, 0] = 5
    view, _ = strided(torch.from_numpy(x.astype(np.float32)).to(dt(kind)), 0, 0, dt(kind))
    hx = host(view)
    _check(hx, view, np.array([hx[0].argmax(), 1, 0], dtype=np.int64), scale, 3, kind, 0)
