"""Alternatives of rows that share a block (a wavefront each): a row's result is its own, whatever the rows beside it
hold.  Columns are compared as such, and log probabilities with those of the same rows in other places, bit for bit
where a row lies alike in its 16 bytes.  Where it begins elsewhere in them, other lanes have its columns: every power of
the sum is the same, and only the order differs in which A = 160 + 2.25 cols / 1024 roundings (u = 2^-24) at most are
made, so logarithms of the two sums differ by 2 A u, and the rounded logarithms (of at most log cols) and results by
2 u of them each."""
import numpy as np
import pytest

from .block_plain import DEV, U, dt, host, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _row(what, d, rng):
    """Rows of few candidates for the alternatives, of more than a list holds, and of most columns."""
    x = 3 * rng.standard_normal(d)
    if what == "tied":
        x[:] = 1.5
    elif what == "few":
        x = rng.integers(0, 3, d).astype(float)
    elif what == "masked":
        x[rng.permutation(d)[20:]] = -np.inf
    elif what == "nan":
        x[d // 2] = np.nan
    return x


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [200, 1000, 2043, 4088])
@pytest.mark.parametrize("top", [8, 32])
def test_rows_of_a_block(d, top, kind):
    import torch
    import paper_2112_02752_amd as emb
    say("rows of a block", d, top, kind)
    rng = np.random.default_rng(d + top)
    kinds = ["plain", "tied", "few", "masked", "nan"]
    # every pair of kinds in every two places of four rows, the rest ordinary; then blocks at random
    blocks = [[a if p == i else b if p == j else "plain" for p in range(4)]
              for i in range(4) for j in range(4) if i != j for a in ("plain", "few") for b in kinds[1:]]
    blocks += [[kinds[k] for k in rng.integers(0, 5, 4)] for _ in range(400)]
    rows = [what for block in blocks for what in block]
    x = torch.from_numpy(np.stack([_row(what, d, rng) for what in rows]).astype(np.float32)).to(dt(kind)).to(DEV)
    n = len(rows)
    want = np.argsort(np.where(np.isnan(host(x)), -np.inf, -host(x)), axis=1, kind="stable")[:, :top]
    answer = emb.LogProbs(n, d, top=top)

    def run(x):
        ids, logp = torch.empty((len(x), top), dtype=torch.int32, device=DEV), torch.empty((len(x), top), device=DEV)
        answer.forward(x, None, None, top_ids=ids, top_logp=logp)
        return ids, logp

    ids, logp = run(x)
    # the rows moved on by one place in their blocks
    ids2, logp2 = run(torch.roll(x, 1, 0))
    torch.cuda.synchronize()
    for got in (ids, torch.roll(ids2, -1, 0)):
        bad = np.nonzero((got.cpu().numpy() != want).any(1))[0]
        assert len(bad) == 0, [(int(i), int(i) % 4, rows[i], rows[i // 4 * 4:i // 4 * 4 + 4]) for i in bad[:4]]
    a, b = logp, torch.roll(logp2, -1, 0)
    same = (a == b) | (a.isnan() & b.isnan())
    if d * x.element_size() % 16:
        a, b = a.double(), b.double()
        same |= (a - b).abs() <= U * (2 * (160 + 2.25 * d / 1024) + 2 * np.log(d) + 2 * (a.abs() + b.abs()))
    assert same.all()


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [9, 100, 600, 3001, 20000, 300000])
@pytest.mark.parametrize("top", [1, 5, 32])
def test_nan_is_the_largest_from_column_zero_on(d, top, kind):
    """Rows of NaN in the first column, the first few, the last and first, and all: lowest columns first, then the numbers."""
    import torch
    import paper_2112_02752_amd as emb
    top = min(top, d)
    x = torch.arange(d, dtype=torch.float32).remainder(7).repeat(6, 1)
    x[0, 0] = x[1, :3] = x[2, 0] = x[2, d - 1] = x[3] = np.nan
    x[4, d - 1] = np.nan
    x = x.to(dt(kind)).to(DEV)
    x[5, 0] = -torch.full((), np.nan, device=DEV)       # its sign is nothing
    ids, logp = torch.full((6, top), -7, dtype=torch.int32, device=DEV), torch.zeros((6, top), device=DEV)
    emb.LogProbs(6, d, top=top).forward(x, None, None, top_ids=ids, top_logp=logp)
    want = np.argsort(np.where(np.isnan(host(x)), -np.inf, -host(x)), axis=1, kind="stable")[:, :top]
    assert np.array_equal(ids.cpu().numpy(), want)
    assert logp.isnan().all()
