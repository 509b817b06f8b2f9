"""Residual addition with dropout and norm, and dropout, against plain forms in
64 bits: odd widths, strides and alignments, one row to many, both types.

Tolerances (u = 2^-24): t is a product and a sum, 2 u of |residual| + |scaled x|
and its type's rounding; the sum of a row's squares adds at most 8 * 4 values of
a lane, 6 exchanges and 8 wavefronts one after another, 46 u of a sum of
positive numbers, so 1 / root is off by 23 u, and by 4 u more for mean, eps,
root and reciprocal: y is within 32 u.  The backward's second sum errs by 47 u of its terms'
magnitudes and what it is multiplied with by 32 u: 96 u of the gradient's parts
holds both.  A weight gradient adds the rows of a wavefront (one in 256 or
more), 4 wavefronts, 32 blocks' rows and 16 partial sums one after another.
Results are then rounded to their type: half a step."""
import numpy as np
import pytest

from .block_plain import (DEV, HALF, U, dropped, dt, host, kept, keep_scale, norm_parts, say, strided, untouched, within)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _data(rng, n, d, dtype, gap, shift, std=1.0):
    import torch
    x = torch.from_numpy((rng.standard_normal((n, d)) * std).astype(np.float32)).to(dt(dtype))
    return strided(x, gap, shift, dt(dtype))


# widths at each variant's borders, odd ones, the widest
SIZES = [(1, 1, 0, 0), (1, 8, 0, 0), (5, 3, 1, 0), (3, 512, 0, 0), (70, 513, 0, 1), (9, 520, 8, 0), (33, 1024, 8, 8),
         (6, 1030, 0, 0), (64, 1536, 0, 0), (5, 2048, 0, 0), (4, 2049, 0, 3), (3, 2056, 0, 0), (7, 4096, 0, 0),
         (3, 4100, 0, 0), (2, 8192, 0, 0), (3, 8200, 8, 0), (2, 16384, 0, 0), (2, 16383, 0, 0), (3001, 40, 0, 0),
         (2500, 264, 8, 0), (0, 64, 0, 0),
         # several rows a wavefront, the last ones of a block not there
         (57, 64, 0, 0), (58, 63, 0, 1), (3, 24, 8, 8), (1025, 13, 0, 0), (61, 65, 3, 0), (129, 128, 0, 0), (2101, 120, 8, 1),
         (37, 127, 0, 1), (66, 129, 0, 0), (41, 250, 6, 1), (43, 256, 0, 3), (47, 257, 0, 0)]


@pytest.mark.parametrize("types", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("n,d,gap,shift", SIZES)
def test_norm(n, d, gap, shift, types):
    import torch
    import paper_2112_02752_amd as emb
    kind, stream = types
    drop = [0.0, 0.1, 0.5][(n + d) % 3]
    say("norm", n, d, gap, shift, types, drop)
    rng = np.random.default_rng(n * 7 + d)
    seed, first_row, eps = 12345 + d, 7 * (n % 2), 1e-6
    x, _ = _data(rng, n, d, kind, gap, shift)
    res, _ = _data(rng, n, d, stream, gap, shift, 2.0)
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)).to(DEV)
    total, tbuf = _data(rng, n, d, stream, gap, shift)
    y, ybuf = _data(rng, n, d, kind, gap, shift)
    saved = emb.Checkpoint(n, d)
    norm = emb.Norm(w, eps=eps, drop=drop, max_rows=max(n, 1))
    norm.forward(x, y, residual=res, total=total, saved=saved, seed=seed, first_row=first_row)
    torch.cuda.synchronize()
    branch = dropped(host(x), drop, seed, first_row)
    want = host(res) + branch
    within(total, want, 2 * U * (np.abs(host(res)) + np.abs(branch)) + HALF[stream] * np.abs(want), "total")
    t, wide = host(total), host(w)
    dy, _ = _data(rng, n, d, kind, gap, shift, 0.3)
    inv, nn, grad, size = norm_parts(t, wide, eps, host(dy))
    within(y, nn * wide, (32 * U + HALF[kind]) * np.abs(nn * wide), "y")
    assert untouched(total, tbuf, gap, shift) and untouched(y, ybuf, gap, shift)
    again = emb.Checkpoint(n, d)
    again.pack(y)
    assert torch.equal(saved.codes, again.codes) and torch.equal(saved.exps, again.exps)

    arriving, _ = _data(rng, n, d, stream, gap, shift, 0.3)
    dtotal, dbuf = _data(rng, n, d, stream, gap, shift)
    branch_grad, bbuf = _data(rng, n, d, kind, gap, shift)
    dw = torch.full((d,), 3.0, device=DEV)
    norm.backward(total, dy, dtotal, branch=branch_grad, arriving=arriving, dweight=dw, seed=seed, first_row=first_row)
    torch.cuda.synchronize()
    want, off = host(arriving) + grad, 96 * U * size + 2 * U * np.abs(host(arriving))
    within(dtotal, want, off + HALF[stream] * np.abs(want), "dtotal")
    scaled = dropped(want, drop, seed, first_row)
    within(branch_grad, scaled, (off * keep_scale(drop) + (U + HALF[kind]) * np.abs(scaled)) * (scaled != 0), "dbranch")
    assert untouched(dtotal, dbuf, gap, shift) and untouched(branch_grad, bbuf, gap, shift)
    terms = host(dy) * nn
    depth = n / 256 + 4 + 32 + 16 + 34
    within(dw, terms.sum(0), depth * U * np.abs(terms).sum(0), "dweight")
    # added to what is there
    dw2 = torch.full((d,), 3.0, device=DEV)
    norm.backward(total, dy, dweight=dw2, add=True, seed=seed, first_row=first_row)
    torch.cuda.synchronize()
    assert torch.equal(dw2, dw + 3.0)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_norm_alone(kind):
    """No residual, no kept total, in place."""
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(5)
    x, _ = _data(rng, 37, 200, kind, 0, 0)
    w = torch.ones(200, device=DEV)
    norm = emb.Norm(w, eps=1e-5)
    want = host(x) / np.sqrt((host(x) ** 2).mean(1, keepdims=True) + 1e-5)
    y = torch.empty_like(x)
    norm.forward(x, y)
    within(y, want, (32 * U + HALF[kind]) * np.abs(want), "y")
    saved = emb.Checkpoint(37, 200)
    norm.forward(x, saved=saved)
    back = torch.empty_like(x)
    saved.unpack(back)
    again = emb.Checkpoint(37, 200)
    again.pack(y)
    assert torch.equal(saved.codes, again.codes) and torch.equal(saved.exps, again.exps)
    # total over the residual's rows, y over x's
    res, _ = _data(rng, 37, 200, kind, 0, 0)
    total, y2 = torch.empty_like(x), torch.empty_like(x)
    norm.forward(x, y2, residual=res, total=total)
    norm.forward(x, x, residual=res, total=res)
    torch.cuda.synchronize()
    assert torch.equal(res, total) and torch.equal(x, y2)
    # gradients over what arrives
    dy, _ = _data(rng, 37, 200, kind, 0, 0)
    arriving, _ = _data(rng, 37, 200, kind, 0, 0)
    dtotal, branch = torch.empty_like(x), torch.empty_like(x)
    norm.backward(total, dy, dtotal, branch=branch, arriving=arriving)
    norm.backward(total, dy, arriving, branch=dy, arriving=arriving)
    torch.cuda.synchronize()
    assert torch.equal(arriving, dtotal) and torch.equal(dy, branch)


def test_norm_extreme_rows():
    """Rows of zeros, of tiny and huge values, with infinities: each keeps to itself."""
    import torch
    import paper_2112_02752_amd as emb
    x = torch.zeros((6, 96), device=DEV)
    x[1] = 1e-30
    x[2] = 1e18
    x[3, 5] = float("inf")
    x[4, 7] = float("nan")
    x[5] = 2.0
    y = torch.empty_like(x)
    saved = emb.Checkpoint(6, 96)
    emb.Norm(torch.ones(96, device=DEV), eps=1e-6).forward(x, y, saved=saved)
    y = y.cpu()
    assert (y[0] == 0).all()
    assert torch.allclose(y[1], torch.tensor(1e-27), rtol=1e-5, atol=0)
    assert torch.allclose(y[2], torch.ones(96), rtol=32 * U) and torch.allclose(y[5], torch.ones(96), rtol=1e-6)
    assert torch.isnan(y[3, 5]) and (y[3, :5] == 0).all() and torch.isnan(y[4]).all()
    assert saved.exps.cpu()[3].tolist()[0] == 255 and (saved.exps.cpu()[4] == 255).all()


@pytest.mark.parametrize("d", [40, 61, 136, 250, 264, 1000, 1029, 4104])
def test_infinities_at_a_rows_end(d):
    """They keep to their row, where lanes past its end read them again."""
    import torch
    import paper_2112_02752_amd as emb
    n = 21
    rng = np.random.default_rng(d)
    total, dy = (torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(DEV) for _ in range(2))
    total[4, d - 1], total[11, d - 2], dy[7, d - 1], dy[13, d - 3] = (float(v) for v in ("inf", "nan", "inf", "nan"))
    bad = {4, 7, 11, 13}
    norm = emb.Norm(torch.ones(d, device=DEV), max_rows=n)
    y, kept_total, dtotal, dbranch = (torch.empty_like(dy) for _ in range(4))
    norm.forward(total, y, total=kept_total)
    norm.backward(kept_total, dy, dtotal=dtotal, branch=dbranch)
    t, g = host(total), host(dy)
    with np.errstate(all="ignore"):
        inv = 1 / np.sqrt((t * t).mean(1, keepdims=True) + 1e-6)
        along = (g * t * inv).mean(1, keepdims=True)
        want_y, want_d = t * inv, inv * (g - t * inv * along)
    for i in range(n):
        if i in (4, 11):
            assert np.array_equal(np.isfinite(host(y)[i]), np.isfinite(want_y[i])), i
        else:       # a sum of d terms, in at most 64 of a lane and 12 of lanes
            within(y[i], want_y[i], (2 * 80) * U * np.abs(want_y[i]), i)
        if i in bad:
            assert not np.isfinite(host(dtotal)[i]).any() or i == 4, i
        else:
            near = 4 * 80 * U * inv[i] * (np.abs(g[i]) + np.abs(t[i] * inv[i]) * np.abs(g[i] * t[i] * inv[i]).mean())
            within(dtotal[i], want_d[i], near, i)
            assert torch.equal(dbranch[i], dtotal[i])


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("n,d,gap,shift", SIZES)
def test_dropout(n, d, gap, shift, kind):
    import torch
    import paper_2112_02752_amd as emb
    drop = [0.1, 0.5, 0.999][(n + d) % 3]
    say("dropout", n, d, gap, shift, kind, drop)
    rng = np.random.default_rng(n + 3 * d)
    x, _ = _data(rng, n, d, kind, gap, shift)
    y, buf = _data(rng, n, d, kind, gap, shift)
    seed, first_row = (1 << 63) + 11 * d, (1 << 40) * (d % 2)
    emb.dropout(x, y, drop, seed, first_row)
    torch.cuda.synchronize()
    keep = kept(n, d, drop, seed, first_row)
    scale = float(np.float32(keep_scale(drop)))
    want = torch.where(torch.from_numpy(keep), x.cpu().float() * scale, torch.tensor(0.0)).to(dt(kind))
    assert torch.equal(y.cpu(), want)
    assert untouched(y, buf, gap, shift)
    emb.dropout(x, x, drop, seed, first_row)
    assert torch.equal(x.cpu(), want)


def test_dropout_of_parts_is_that_of_the_whole():
    import torch
    import paper_2112_02752_amd as emb
    x = torch.randn((100, 50), device=DEV)
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    emb.dropout(x, whole, 0.3, 99)
    for a, b in ((0, 1), (1, 60), (60, 100)):
        emb.dropout(x[a:b], parts[a:b], 0.3, 99, first_row=a)
    assert torch.equal(whole, parts)
    assert 0.2 < float((whole == 0).float().mean()) < 0.4
    other = torch.empty_like(x)
    emb.dropout(x, other, 0.3, 100)
    assert not torch.equal(whole == 0, other == 0)
    emb.dropout(x, other, 0.0, 100)
    assert torch.equal(other, x)


def test_dropped_infinities_are_zeros():
    import torch
    import paper_2112_02752_amd as emb
    x = torch.full((4, 64), float("inf"), device=DEV)
    y = torch.empty_like(x)
    emb.dropout(x, y, 0.5, 1)
    keep = torch.from_numpy(kept(4, 64, 0.5, 1))
    assert (y.cpu()[keep] == float("inf")).all() and (y.cpu()[~keep] == 0).all()


def test_norm_gradients_against_differences():
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(8)
    n, d, eps, drop, seed = 3, 11, 0.1, 0.3, 4
    x, res, dy, w = (rng.standard_normal(s) for s in ((n, d), (n, d), (n, d), (d,)))
    put = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV)  # noqa: E731
    w32 = put(w)
    norm = emb.Norm(w32, eps=eps, drop=drop, max_rows=n)
    total, y, dtotal, branch = (torch.empty((n, d), device=DEV) for _ in range(4))
    dw = torch.empty(d, device=DEV)
    norm.forward(put(x), y, residual=put(res), total=total, seed=seed)
    norm.backward(total, put(dy), dtotal, branch=branch, dweight=dw, seed=seed)

    def loss(x, res, w):
        t = res + dropped(x, drop, seed)
        return (dy * w * t / np.sqrt((t * t).mean(1, keepdims=True) + eps)).sum()

    for name, got, i in (("dx", branch, 0), ("dres", dtotal, 1), ("dw", dw, 2)):
        args, got = [x, res, w], host(got)
        for at in np.ndindex(args[i].shape):
            ends = []
            for h in (1e-5, -1e-5):
                moved = args[i].copy()
                moved[at] += h
                ends.append(loss(*(moved if j == i else a for j, a in enumerate(args))))
            # (differences: 1e-10 of the third derivative, 1e-16 / 1e-5 of the loss; fp32: inputs rounded to u)
            assert abs(got[at] - (ends[0] - ends[1]) / 2e-5) < 2e-5, (name, at)


def test_norm_on_streams_and_in_graphs():
    import torch
    import paper_2112_02752_amd as emb
    torch.manual_seed(3)
    n, d = 300, 264
    x, res, dy, arr = (torch.randn((n, d), device=DEV).bfloat16() for _ in range(4))
    norm = emb.Norm(torch.ones(d, device=DEV), drop=0.2, max_rows=n)

    def step(seed=6):
        out = [torch.empty_like(x) for _ in range(4)] + [torch.empty(d, device=DEV)]
        norm.forward(x, out[1], residual=res, total=out[0], seed=seed)
        norm.backward(out[0], dy, out[2], branch=out[3], arriving=arr, dweight=out[4], seed=seed)
        return out

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(torch.randn((n, d), device=DEV))
        eager = step()
        for t in held:
            t.fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, held):
            assert torch.equal(a, b), i
