"""The forms that only larger calls take: outputs stored past the caches, chains
of many spans over several slices, rows of a table's gradient beside its zeros,
large tiles of a weight gradient; with tolerances as in test_gpu_sequence."""
import numpy as np
import pytest

from tests import test_gpu_sequence as small
from tests.test_gpu_sequence import U, _dt, _np, _plain_backward, _plain_forward, _saved_plain, _steps

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("table,out,n,D", [("bf16", "bf16", 8203, 2056), ("fp32", "bf16", 16501, 1028),
                                           ("bf16", "fp32", 4111, 2056), ("fp32", "fp32", 70001, 132)])
def test_lookup_past_the_caches(table, out, n, D):
    import torch
    import paper_2112_02752_amd as emb
    t = {"bf16": torch.bfloat16, "fp32": torch.float32}
    g = torch.Generator(device=DEV).manual_seed(n)
    W = torch.randn((701, D), generator=g, device=DEV).to(t[table])
    ids = torch.randint(0, 701, (n,), generator=g, device=DEV)
    batch = emb.Batch(torch.tensor([0, n], dtype=torch.int32, device=DEV), ids, 1)
    y = torch.empty((n, D), dtype=t[out], device=DEV)
    assert y.numel() * y.element_size() > 32 << 20
    emb.token_fwd(emb.Tables(W, [0, 701]), batch, y, scale=0.7, pad_row=5)
    want = W.float()[ids] * torch.tensor(0.7, device=DEV)
    want[ids == 5] = 0
    assert torch.equal(y, want.to(t[out]))


@pytest.mark.parametrize("dy_type", ["bf16", "fp32"])
def test_table_gradient_past_the_caches(dy_type):
    """9001 rows, of which a few hundred are named, some by hundreds of tokens."""
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(2)
    R, D, n = 9001, 1028, 6001
    key = (rng.random(n) ** 4 * 900).astype(np.int64) * 9 + 3
    key[rng.random(n) < 0.05] = R - 1
    dy = torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).to(
        torch.bfloat16 if dy_type == "bf16" else torch.float32)
    tables = emb.Tables(torch.zeros((R, D), device=DEV), [0, R])
    batch = emb.Batch(torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.from_numpy(key).to(DEV), 1)
    layer = emb.TokenLayer(tables, scale=0.3, pad_row=R - 1, max_tokens=n, max_seqs=1)
    grad = torch.full((R, D), 7.0, device=DEV)
    layer.table_grad(batch, dy.to(DEV), grad)
    want, mag = np.zeros((R, D)), np.zeros((R, D))
    keep = key != R - 1
    rows = dy.double().numpy()[keep] * np.float32(0.3)
    np.add.at(want, key[keep], rows)
    np.add.at(mag, key[keep], np.abs(rows))
    assert (np.abs(_np(grad) - want) <= 67 * U * mag).all()
    assert (_np(grad)[mag.sum(1) == 0] == 0).all()


# so many positions and columns that a wavefront takes a chunk's positions (n, D, rows, gap, shift, hottest's share, sequences)
MANY = [(33001, 48, [300, 2000], 3, 0, 0.2, 11), (9001, 1028, [4000], 0, 1, 0.1, 9), (3701, 4104, [50, 900], 8, 0, 0.3, 2)]


@pytest.mark.parametrize("dy_type", ["fp32", "bf16"])
@pytest.mark.parametrize("case", MANY)
def test_token_gradient_of_many(case, dy_type):
    small.test_token_gradient_layouts(case, dy_type)


@pytest.mark.parametrize("opt", ["sgd", "adagrad", "adagrad_ew"])
@pytest.mark.parametrize("table,dy_type", [("fp32", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("case", MANY)
def test_token_update_of_many(case, table, dy_type, opt):
    small.test_token_update(case, table, dy_type, opt)


def _check_scan(rng, offs, D, dtype):
    """Forward and backward over the given sequences with every optional part,
    against the plain form."""
    import torch
    import paper_2112_02752_amd as emb
    n, M, t = int(offs[-1]), len(offs) - 1, _dt(dtype)
    v = [torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).to(t) for _ in range(4)]
    x, f, o, dy = (m.double().numpy() for m in v)
    xv, fv, ov, dyv = (m.to(DEV) for m in v)
    bias = np.linspace(-2, 4, D).astype(np.float32)
    h0, dhl = rng.standard_normal((2, M, D)).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    scan = emb.Scan(dev(offs), xv, fv, ov, bias=dev(bias), h0=dev(h0))
    rec = emb.Recurrence(n, M, D)
    y, last = torch.empty_like(xv), torch.empty((M, D), device=DEV)
    rec.forward(scan, y, last)
    a, q, before, h, y_w, last_w = _plain_forward(offs, x, f, o, bias, h0)
    steps = _steps(int(max(offs[1:] - offs[:-1])), q)
    top = max(np.abs(x).max(), np.abs(h0).max())
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    tol = 32 * U * steps * top
    assert (np.abs(_np(y) - y_w) <= tol + half * np.abs(y_w)).all()
    assert (np.abs(_np(last) - last_w) <= tol).all()
    dx, df, do = (torch.empty_like(xv) for _ in range(3))
    db, dh0 = torch.empty(D, device=DEV), torch.empty((M, D), device=DEV)
    rec.backward(scan, dyv, dx, df, do, dbias=db, dh_last=dev(dhl), dh0=dh0)
    dh, dx_w, df_w, do_w, db_w, dh0_w = _plain_backward(offs, x, a, q, before, h, o, dy, dhl)
    gtop = max(1.0, np.abs(dh).max())
    tol_g, tol_f = 32 * U * steps * gtop, 4 * 32 * U * steps * gtop * max(top, 1.0)
    assert (np.abs(_np(dx) - dx_w) <= tol_g + half * np.abs(dx_w)).all()
    assert (np.abs(_np(df) - df_w) <= tol_f + half * np.abs(df_w)).all()
    assert (np.abs(_np(do) - do_w) <= tol_f + half * np.abs(do_w)).all()
    assert (np.abs(_np(db) - db_w) <= 2 * tol_f + (70 * U) * np.abs(df_w).sum(0) + tol_f * np.sqrt(n + 1)).all()
    assert (np.abs(_np(dh0) - dh0_w) <= tol_g).all()
    again = [torch.empty_like(m) for m in (y, dx, df, do)]
    rec.forward(scan, again[0])
    rec.backward(scan, dyv, *again[1:], dh_last=dev(dhl))
    assert all(torch.equal(p, q) for p, q in zip(again, (y, dx, df, do)))


@pytest.mark.parametrize("dtype,n,D", [("bf16", 8500, 2052), ("fp32", 8500, 1030)])
def test_scan_past_the_caches(dtype, n, D):
    """67 spans forward and 133 backward in each of 17 slices; a long sequence,
    an empty one and some short ones."""
    rng = np.random.default_rng(D)
    lens = [n - 1300, 0, 1, 700, 64, 535]
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    assert offs[-1] == n and n * D * (2 if dtype == "bf16" else 4) > 32 << 20
    _check_scan(rng, offs, D, dtype)


def test_weight_gradient_large_tiles():
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(11)
    n, K, F = 2100, 1500, 4002
    x = torch.from_numpy(rng.standard_normal((n, K)).astype(np.float32)).to(DEV)
    ck = emb.Checkpoint(n, K)
    ck.pack(x)
    back = _saved_plain(x.double().cpu().numpy())[2]
    dy = torch.from_numpy(rng.standard_normal((n, F)).astype(np.float32)).bfloat16()
    dw = torch.full((K, F), 5.0, device=DEV)
    ck.weight_grad(dy.to(DEV), dw)
    y = dy.double().numpy()
    want, mag = back.T @ y, np.abs(back).T @ np.abs(y)
    assert (np.abs(_np(dw) - want) <= (n + 8) * 2 * U * mag).all()
    first = dw.clone()
    ck.weight_grad(dy.to(DEV), dw)
    assert torch.equal(dw, first)


@pytest.mark.parametrize("dtype,n,D", [("bf16", 2100, 1602), ("bf16", 1900, 803), ("fp32", 1900, 801)])
def test_scan_of_many_blocks(dtype, n, D):
    """Above 96 blocks of long spans, below 32 MB."""
    rng = np.random.default_rng(D)
    lens = [1, 0, n - 800, 127, 129, 543]
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    assert offs[-1] == n
    _check_scan(rng, offs, D, dtype)


def test_matrices_of_more_than_four_gigabytes():
    """Rows 8 MB apart: the last ones lie beyond 2^32 bytes (and 2^32 / 2 elements)."""
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(4)
    n, D, F = 700, 96, 200
    base = torch.empty((n, 1 << 22), dtype=torch.bfloat16, device=DEV)
    view = [base[:, 1000 * i: 1000 * i + D] for i in range(9)]
    near = [torch.empty((n, D), dtype=torch.bfloat16, device=DEV) for _ in range(9)]
    for k in range(4):
        near[k].copy_(torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)))
        view[k].copy_(near[k])
    offs = torch.tensor([0, 3, 3, 650, n], dtype=torch.int32, device=DEV)
    bias = torch.linspace(-1, 3, D, device=DEV)
    sums = []
    for v in (near, view):
        rec, db = emb.Recurrence(n, 4, D), torch.empty(D, device=DEV)
        scan = emb.Scan(offs, v[0], v[1], v[2], bias=bias)
        rec.forward(scan, v[4])
        rec.backward(scan, v[3], v[5], v[6], v[7], dbias=db)
        sums.append(db)
    assert torch.equal(*sums)
    for k in (4, 5, 6, 7):
        assert torch.equal(view[k], near[k])
    state = [torch.ones((n, D), device=DEV) for _ in range(2)]
    for v, st in zip((near, view), state):
        emb.scan_step(v[0], v[1], v[2], st, v[8], bias=bias)
    assert torch.equal(view[8], near[8]) and torch.equal(*state)
    ck = [emb.Checkpoint(n, D) for _ in range(2)]
    back = [near[8], view[8]]
    for c, v, b in zip(ck, (near, view), back):
        c.pack(v[0])
        c.unpack(b)
    assert torch.equal(*back)
    wide = torch.from_numpy(rng.standard_normal((n, F)).astype(np.float32)).bfloat16().to(DEV)
    base[:, 20000:20000 + F] = wide
    dw = [torch.empty((D, F), device=DEV) for _ in range(2)]
    ck[0].weight_grad(wide, dw[0])
    ck[0].weight_grad(base[:, 20000:20000 + F], dw[1])
    assert torch.equal(*dw)


def test_tables_of_more_than_four_gigabytes():
    import torch
    import paper_2112_02752_amd as emb
    R, D, n = 600_001, 2048, 301
    rng = np.random.default_rng(6)
    key = np.concatenate([rng.integers(R - 2000, R, n - 3), [0, R - 1, R - 1]])
    ids = torch.from_numpy(key).to(DEV)
    W = torch.zeros((R, D), device=DEV)
    W[ids] = torch.arange(n, device=DEV, dtype=torch.float32)[:, None] + 1
    W[R - 1] = 77
    batch = emb.Batch(torch.tensor([0, n], dtype=torch.int32, device=DEV), ids, 1)
    tables = emb.Tables(W, [0, R])
    y = torch.empty((n, D), device=DEV)
    layer = emb.TokenLayer(tables, opt="sgd", lr=0.5, max_tokens=n, max_seqs=1)
    layer.forward(batch, y)
    assert torch.equal(y, W[ids])
    dy = torch.full((n, D), 0.25, device=DEV)
    grad = torch.full((R, D), 3.0, device=DEV)
    layer.table_grad(batch, dy, grad)
    count = torch.zeros(R, device=DEV).index_add_(0, ids, torch.full((n,), 0.25, device=DEV))
    assert bool((grad == count[:, None]).all())
    want = W[ids] - 0.5 * count[ids][:, None]
    layer.update(batch, dy)
    assert torch.equal(W[ids], want)


@pytest.mark.parametrize("n,K,F", [(2100, 2048, 6146), (8200, 1024, 2050)])
def test_weight_gradient_large_tiles_whole_and_in_parts(n, K, F):
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(n)
    x = torch.from_numpy(rng.standard_normal((n, K)).astype(np.float32)).to(DEV)
    ck = emb.Checkpoint(n, K)
    ck.pack(x)
    back = _saved_plain(x.double().cpu().numpy())[2]
    dy = torch.from_numpy(rng.standard_normal((n, F)).astype(np.float32)).bfloat16()
    y = dy.double().numpy()
    want, mag = back.T @ y, np.abs(back).T @ np.abs(y)
    dw = torch.full((K, F), 5.0, device=DEV)
    ck.weight_grad(dy.to(DEV), dw)
    assert (np.abs(_np(dw) - want) <= (n + 8) * 2 * U * mag).all()
    first = dw.clone()
    ck.weight_grad(dy.to(DEV), dw, add=True)
    assert (np.abs(_np(dw) - 2 * want) <= (2 * n + 20) * 2 * U * mag + 4 * U * np.abs(want)).all()
    ck.weight_grad(dy.to(DEV), dw)
    assert torch.equal(dw, first)
