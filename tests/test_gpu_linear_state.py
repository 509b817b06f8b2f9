"""Linear attention of bf16 rows where results are small against what they are
summed from: large states, keys and values with a common component (as a trained
model's activations have), queries across it; and many sequences some of which
have several segments.

Tolerances (u = 2^-24).  Of bf16 rows nothing is rounded but
 - the state where rows are multiplied with it, weights within a chunk, and what
   the state gets of a row: each is held in two parts of bf16.  The first is off by
   at most 2^-8 of the value, the second by 2^-8 of what the first leaves: 2^-16.  A
   term that comes through the state has two of these, one within a chunk one;
 - fp32 sums: (T + width + 32) 2 u |.|, T being the most positions (times heads) that
   add into one value, |.| the same sum of magnitudes;
 - the result, to bf16.
So an element is off by at most (T + width + 32) 2 u |.| + 2^-15 |.| + 2^-8 of itself.

Where only the sum over many elements is looked at: rounding errors of different values
are independent, so the root mean square of what precedes the result's own
rounding is at most that of 2^-16 sqrt(sum over d of q_d^2 S_d^2), S the state after the
position, once for the operand and once for what S is made of.  That is where the state
outweighs a chunk's own weights, as the long sums here do."""
import numpy as np
import pytest

from .block_plain import DEV, HALF, U, dt, host, linear, linear_back, say, within
from .test_gpu_linear import Batch, _offsets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _put(t, x):
    import torch
    t.copy_(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV))


def _across(rng, rows, cols):
    """Rows whose neighbouring columns cancel."""
    x = rng.standard_normal((rows, cols))
    x[:, 1::2] = -x[:, ::2]
    return x


def _parts(b):
    h, g, dk, dv = b.sizes
    n, r = b.n, h // g
    q, k, v, dy = (host(t)[:n] for t in (b.q, b.k, b.v, b.dy))
    return q.reshape(n, g, r, dk), k.reshape(n, g, dk), v.reshape(n, g, dv), dy.reshape(n, g, r, dv)


def _results(b, f=lambda t: t):
    q, k, v, dy = map(f, _parts(b))
    scale, decay = float(np.float32(b.scale)), host(b.decay)
    first, dlast = (f(host(t)) if t is not None else None for t in (b.first, b.dlast))
    y, last, every = linear(b.offs, q, k, v, decay, scale, first)
    return (y, *linear_back(b.offs, q, k, v, decay, scale, every, dy, dlast)[:3]), every


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("n,m,heads,groups,dk,dv,gap,shift", [
    (1, 1, 1, 1, 16, 16, 0, 0), (40, 2, 2, 1, 16, 32, 0, 0), (70, 1, 1, 1, 24, 40, 0, 0), (70, 2, 2, 2, 64, 64, 0, 0),
    (70, 1, 1, 1, 18, 34, 1, 1), (66, 1, 1, 1, 128, 128, 0, 0), (66, 1, 1, 1, 256, 200, 0, 0), (66, 1, 1, 1, 250, 202, 0, 0)])
def test_results_that_cancel_in_a_large_state(n, m, heads, groups, dk, dv, gap, shift, kind):
    say("large states", kind, n, m, heads, groups, dk, dv, gap, shift)
    rng = np.random.default_rng(dk)
    b = Batch(kind, n, _offsets(rng, n, m), heads, groups, dk, dv, gap, shift, seed=n)
    for t in (b.first, b.dlast):
        _put(t, 30 + rng.standard_normal(tuple(t.shape)))
    for t in (b.q, b.k, b.v, b.dy):
        _put(t, _across(rng, *t.shape))
    b.run()
    b.check()
    want, _ = _results(b)
    size, _ = _results(b, np.abs)
    near = (n * (heads // groups) + max(dk, dv) + 32) * 2 * U + (2.0 ** -15 if kind == "bf16" else 0)
    for got, w, s, name in zip((b.y, b.dq, b.dk, b.dv), want, size, ("y", "dq", "dk", "dv")):
        within(host(got).reshape(w.shape), w, near * s + HALF[kind] * np.abs(w), name)


@pytest.mark.parametrize("common", [0.0, 1.0, 3.0])
def test_rows_with_a_common_component(common):
    """The error's root mean square is the result's own rounding's, and three times (the independence's margin) what the
    parts leave."""
    import torch
    say("rows with a common component", common)
    n, dk, dv = 2048, 128, 128
    rng = np.random.default_rng(9)
    b = Batch("bf16", n, np.array([0, n], dtype=np.int32), 1, 1, dk, dv, first=False, seed=5)
    b.decay.fill_(1 - 1 / 512)
    _put(b.q, _across(rng, n, dk))
    _put(b.dy, _across(rng, n, dv))
    for t in (b.k, b.v):
        _put(t, common + rng.standard_normal(tuple(t.shape)))
    b.run()
    (y, dq, _, _), every = _results(b)
    q, k, v, dy = _parts(b)
    scale, s2 = float(np.float32(b.scale)), every[:, 0] ** 2
    for got, w, left in ((b.y, y, (q[:, 0] ** 2 @ s2)), (b.dq, dq, (dy[:, 0] ** 2 @ np.swapaxes(s2, 1, 2)))):
        w = w.reshape(n, -1)
        rms = lambda t: float(np.sqrt((t ** 2).mean()))  # noqa: E731
        own = rms(host(torch.from_numpy(w).to(torch.bfloat16)) - w)
        parts = 2 * 2.0 ** -16 * scale * float(np.sqrt(left.mean()))
        off = rms(host(got) - w)
        assert off <= own + 3 * parts, (off, own, parts, rms(w))


def test_weights_within_a_chunk():
    """Sequences shorter than a chunk, no state before them: y's error is its rounding's, and what two parts of the
    weights leave, 2^-16 sqrt(sum over j of p_j^2 v_j^2) in its root mean square (three times: its margin)."""
    import torch
    n, m, dk, dv = 1500, 50, 64, 64
    offs = np.arange(0, n + 1, n // m).astype(np.int32)
    b = Batch("bf16", n, offs, 1, 1, dk, dv, first=False, seed=11)
    b.run()
    q, k, v, _ = _parts(b)
    want, left = np.zeros((n, dv)), np.zeros((n, dv))
    for i in range(m):
        a, e = offs[i], offs[i + 1]
        at = np.arange(e - a)
        w = np.tril(float(host(b.decay)[0]) ** np.abs(at[:, None] - at)) * (q[a:e, 0, 0] @ k[a:e, 0].T) * b.scale
        want[a:e] = w @ v[a:e, 0]
        left[a:e] = w ** 2 @ v[a:e, 0] ** 2
    rms = lambda t: float(np.sqrt((t ** 2).mean()))  # noqa: E731
    own = rms(host(torch.from_numpy(want).to(torch.bfloat16)) - want)
    off = rms(host(b.y) - want)
    assert off <= own + 3 * 2.0 ** -16 * float(np.sqrt(left.mean())), (off, own)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_a_prompt_and_single_tokens_agree(kind):
    """Sequences of one token each by the whole form and as single tokens: both are sums of dk products with the same
    state, whose operand the whole form holds in two parts."""
    import torch
    import paper_2112_02752_amd as emb
    n, h, g, dk, dv = 70, 4, 2, 64, 32
    rng = np.random.default_rng(2)
    b = Batch(kind, n, np.arange(n + 1, dtype=np.int32), h, g, dk, dv, seed=3)
    _put(b.first, 30 + rng.standard_normal(tuple(b.first.shape)))
    _put(b.q, _across(rng, *b.q.shape))
    b.attention.forward(b.heads, b.y, b.last)
    pool, y = b.first.clone(), torch.empty_like(b.y)
    emb.linear_attention_step(b.q, b.k, b.v, b.decay, pool, y, heads=h, groups=g, scale=b.scale)
    size, _ = _results(b, np.abs)
    size = size[0].reshape(n, -1)
    near = 2 * (dk + 32) * 2 * U + (2.0 ** -15 if kind == "bf16" else 0)
    within(b.y, host(y), near * size + 2 * HALF[kind] * np.abs(host(y)) * (1 + HALF[kind]), "y")
    within(b.last, host(pool), 8 * U * (np.abs(host(pool)) + 60), "states")


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("m", [63, 64, 65, 200])
def test_many_sequences_some_of_several_segments(m, kind):
    """Boundaries between segments found among so many offsets that no wavefront holds them all: sequences of one
    position, empty ones, and long ones first, in between and last."""
    say("many sequences", kind, m)
    lens = np.ones(m, dtype=np.int64)
    lens[::3] = 0
    lens[[1, m // 2, m - 1]] = 300, 450, 200
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    b = Batch(kind, int(offs[-1]), offs, 2, 1, 16, 24, seed=m)
    b.run()
    b.check()
