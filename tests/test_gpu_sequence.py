"""Operators over sequences of tokens against plain implementations in 64 bits:
token lookup and its gradient by sorted tokens, the gated recurrence forward,
backward and by single tokens, activations in 8 bits and the weight gradient
from them; at the sizes, strides and contents where they can go wrong.

Tolerances (u = 2^-24, half a unit of fp32's last place):
 - a lookup is one fp32 product, rounded once more for bf16: equal bit for bit;
 - a gradient sum adds at most 64 fp32 values one after another, pieces of 64
   in double, and scales once: (64 + 3) u times the sum of magnitudes;
 - codes and restored values of a checkpoint are exact;
 - a gate sigmoid(z) of |z| <= 16 is within 24 u (exponent's product: 16 log2(e)
   ln 2 u, exponential, sum, reciprocal: 2 u each), so a step of the recurrence
   errs by at most 32 u of the largest state, and as many steps add up as the
   slowest gate remembers: min(T, 1 / (1 - a)); gradients are sums over the same
   steps of products of at most three such values;
 - a weight gradient adds N products in fp32: (N + 8) 2u times the sum of their
   magnitudes (twice u: the matrix units' inner sums need not round to nearest);
 - bf16 results: 2^-8 of their magnitude more.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _say(*a):
    print(*a, flush=True)


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _strided(x, gap, shift, dtype):
    """x on the GPU as columns of a wider matrix (gap columns after them, shift
    elements before the first), the rest filled with 77."""
    import torch
    n, d = x.shape
    buf = torch.full((n * (d + gap) + shift + 8,), 77.0, dtype=dtype, device=DEV)
    view = buf[shift:shift + n * (d + gap)].view(n, d + gap)[:, :d] if n else buf[:0].view(0, d)
    view.copy_(torch.as_tensor(x).to(DEV))
    return view, buf


def _np(t):
    return t.detach().cpu().double().numpy()


# ---------------------------------------------------------------- tokens

def _token_batch(rng, rows, n, per_table, bits, hot=0.0, bad=0):
    """offsets, ids (table by table) and global keys of a batch over tables of
    `rows` rows each, `per_table` sequences a table."""
    T = len(rows)
    cuts = np.sort(rng.integers(0, n + 1, T * per_table - 1)) if T * per_table > 1 else np.array([], dtype=int)
    offs = np.concatenate([[0], cuts, [n]]).astype(np.int32)
    table = np.zeros(n, dtype=np.int64)
    for t in range(T):
        table[offs[t * per_table]:offs[(t + 1) * per_table]] = t
    size = np.array(rows)[table] if n else np.zeros(0)
    ids = np.floor(rng.random(n) ** 2 * size).astype(np.int64)
    ids[rng.random(n) < hot] = 0
    start = np.concatenate([[0], np.cumsum(rows)])
    key = start[table] + ids if n else np.zeros(0, dtype=np.int64)
    return offs, ids.astype(np.int32 if bits == 32 else np.int64), key, start


def _tables(rng, rows, D, dtype):
    import torch
    import paper_2112_02752_amd as emb
    start = np.concatenate([[0], np.cumsum(rows)])
    W = torch.from_numpy(rng.standard_normal((int(start[-1]), D)).astype(np.float32)).to(_dt(dtype))
    return W, emb.Tables(W.to(DEV), [int(s) for s in start])


@pytest.mark.parametrize("table,out", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,D,rows,gap,shift,bits", [
    (1, 8, [5], 0, 0, 32), (63, 16, [100], 8, 0, 64), (65, 64, [1000], 1, 0, 32), (1000, 200, [50, 7, 300], 0, 1, 64),
    (257, 1024, [400], 24, 0, 32), (70, 2048, [60], 0, 3, 64), (5, 4104, [9, 1], 8, 0, 32), (9000, 24, [77], 0, 0, 64),
    (0, 16, [10], 0, 0, 32)])
def test_token_lookup(table, out, n, D, rows, gap, shift, bits):
    import torch
    import paper_2112_02752_amd as emb
    _say("token lookup", table, out, n, D, rows)
    rng = np.random.default_rng(n * 31 + D)
    offs, ids, key, start = _token_batch(rng, rows, n, 3, bits)
    W, tables = _tables(rng, rows, D, table)
    pad = int(key[0]) if n else -1
    batch = emb.Batch(torch.from_numpy(offs).to(DEV), torch.from_numpy(ids).to(DEV), 3)
    y, buf = _strided(np.zeros((n, D)), gap, shift, _dt(out))
    emb.token_fwd(tables, batch, y, scale=1.7, pad_row=pad)
    torch.cuda.synchronize()
    want = W[torch.from_numpy(key)].float() * torch.tensor(1.7, dtype=torch.float32)
    want[torch.from_numpy(key == pad)] = 0
    assert torch.equal(y.cpu(), want.to(_dt(out)))
    rest = torch.ones_like(buf, dtype=torch.bool)
    if n:
        rest[shift:shift + n * (D + gap)].view(n, D + gap)[:, :D] = False
    assert bool((buf[rest] == 77.0).all())      # nothing outside the columns is written


def test_token_lookup_of_ids_outside_the_table_gives_zeros():
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(1)
    _, tables = _tables(rng, [10, 5], 16, "fp32")
    ids = torch.tensor([0, 10, -1, 4, 5, 2], dtype=torch.int32, device=DEV)   # table 0: 0 10 -1, table 1: 4 5 2
    batch = emb.Batch(torch.tensor([0, 3, 6], dtype=torch.int32, device=DEV), ids, 1)
    y = torch.ones(6, 16, device=DEV)
    emb.token_fwd(tables, batch, y)
    y = y.cpu()
    assert bool((y[[1, 2, 4]] == 0).all())
    assert torch.equal(y[[0, 3, 5]], tables.weights.cpu()[[0, 14, 12]])


GRAD_CASES = [
    # n, D, rows, gap, shift, share of the hottest token, sequences a table
    (1, 8, [5], 0, 0, 0.0, 1), (64, 64, [40], 0, 0, 0.0, 4), (65, 16, [1], 1, 0, 0.0, 2), (129, 100, [3, 50], 0, 0, 0.3, 3),
    (700, 256, [90], 8, 0, 0.5, 5), (1500, 260, [5], 0, 1, 0.0, 7), (5000, 1024, [4000], 0, 0, 0.1, 9),
    (12001, 48, [300, 200], 3, 0, 0.2, 11), (9000, 64, [2], 0, 0, 0.97, 1), (200, 4104, [20], 8, 0, 0.4, 2),
]


def _grad_setup(case, table, dy_type, bits=32):
    import torch
    import paper_2112_02752_amd as emb
    n, D, rows, gap, shift, hot, per = case
    if table == "bf16" and D % 8:
        D = (D + 7) // 8 * 8
    rng = np.random.default_rng(n + 7 * D)
    offs, ids, key, start = _token_batch(rng, rows, n, per, bits, hot)
    W, tables = _tables(rng, rows, D, table)
    dy = torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).to(_dt(dy_type))
    dyv, _ = _strided(dy, gap, shift, _dt(dy_type))
    batch = emb.Batch(torch.from_numpy(offs).to(DEV), torch.from_numpy(ids).to(DEV), per)
    return rng, D, W, tables, batch, key, dy.double().numpy(), dyv, int(start[-1])


def _sums(key, dy, R, scale, pad):
    keep = key != pad
    g, mag = np.zeros((R, dy.shape[1])), np.zeros((R, dy.shape[1]))
    np.add.at(g, key[keep], dy[keep] * np.float32(scale))
    np.add.at(mag, key[keep], np.abs(dy[keep]) * np.float32(scale))
    return g, mag


@pytest.mark.parametrize("dy_type", ["fp32", "bf16"])
@pytest.mark.parametrize("case", GRAD_CASES)
def test_token_gradient_layouts(case, dy_type):
    import torch
    import paper_2112_02752_amd as emb
    _say("token gradient", case, dy_type)
    rng, D, W, tables, batch, key, dy, dyv, R = _grad_setup(case, "fp32", dy_type)
    n = len(key)
    for pad in (-1, int(np.bincount(key).argmax())):
        layer = emb.TokenLayer(tables, scale=0.3, pad_row=pad, max_tokens=n, max_seqs=batch.bags_per_table * 2)
        want, mag = _sums(key, dy, R, 0.3, pad)
        tol = 67 * U * mag
        whole = torch.full((R, D), 5.0, device=DEV)
        layer.table_grad(batch, dyv, whole)
        assert (np.abs(_np(whole) - want) <= tol).all()
        assert (_np(whole)[mag.sum(1) == 0] == 0).all()
        added = torch.full((R, D), 5.0, device=DEV)
        layer.table_grad(batch, dyv, added, add=True)
        assert (np.abs(_np(added) - 5 - want) <= tol + 2 * U * (5 + mag)).all()
        assert (_np(added)[mag.sum(1) == 0] == 5).all()
        rows = torch.full((n + 3, D), 5.0, device=DEV)
        layer.row_grads(batch, dyv, rows)
        u = int(layer.dedup.num_unique.item())
        keys = layer.dedup.unique_keys[:u].cpu().numpy().astype(np.int64)
        assert np.array_equal(keys, np.unique(key))
        assert np.array_equal(rows[:u].cpu().numpy(), whole.cpu().numpy()[keys])   # the same sums, bit for bit
        assert (rows[u:].cpu().numpy() == 5).all()
        again = torch.empty_like(whole)
        layer.table_grad(batch, dyv, again)
        assert torch.equal(again, whole)
        layer.check()


@pytest.mark.parametrize("opt", ["sgd", "adagrad", "adagrad_ew"])
@pytest.mark.parametrize("table,dy_type", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("case", GRAD_CASES)
def test_token_update(case, table, dy_type, opt):
    """Updated rows within 1e-5 of their largest value (bf16: one unit of the
    last place, 2^-8), accumulators within 1e-5, as the pooled layer's."""
    import torch
    import paper_2112_02752_amd as emb
    _say("token update", case, table, dy_type, opt)
    rng, D, W, tables, batch, key, dy, dyv, R = _grad_setup(case, table, dy_type, 64)
    n, pad = len(key), int(np.bincount(key).argmax()) if len(np.unique(key)) > 1 else -1
    h0 = rng.random((R,) if opt == "adagrad" else (R, D)).astype(np.float32) + 0.5
    state = torch.from_numpy(h0).to(DEV) if opt != "sgd" else None
    layer = emb.TokenLayer(tables, scale=0.3, pad_row=pad, opt=opt, lr=0.05, eps=1e-8, state=state, max_tokens=n,
                           max_seqs=batch.bags_per_table * 2)
    layer.update(batch, dyv)
    g, _ = _sums(key, dy, R, 0.3, pad)
    lr = float(np.float32(0.05))
    W0 = W.double().numpy()
    if opt == "sgd":
        want = W0 - lr * g
    elif opt == "adagrad":
        h = h0 + (g * g).mean(1)
        want = W0 - lr * g / (np.sqrt(h) + 1e-8)[:, None]
    else:
        h = h0 + g * g
        want = W0 - lr * g / (np.sqrt(h) + 1e-8)
    got = _np(tables.weights)
    tol = (1e-5 if table == "fp32" else 2.0 ** -8 + 1e-5) * np.abs(want).max(1, keepdims=True)
    assert (np.abs(got - want) <= tol).all()
    touched = np.zeros(R, dtype=bool)
    touched[key[key != pad]] = True
    assert np.array_equal(got[~touched], W0[~touched])
    if opt != "sgd":
        assert (np.abs(_np(state) - h) <= 1e-5 * h).all()
        assert np.array_equal(_np(state)[~touched], h0.astype(np.float64)[~touched])
    layer.check()


def test_token_update_stochastic_rounding_is_a_neighbour_and_follows_the_seed():
    import torch
    import paper_2112_02752_amd as emb
    got = []
    for seed in (3, 3, 4):
        rng, D, W, tables, batch, key, dy, dyv, R = _grad_setup((700, 256, [90], 8, 0, 0.5, 5), "bf16", "bf16")
        layer = emb.TokenLayer(tables, opt="sgd", lr=0.01, max_tokens=len(key), max_seqs=8, rounding="stochastic",
                               seed=seed)
        layer.update(batch, dyv)
        got.append(tables.weights.clone())
    g, _ = _sums(key, dy, R, 1.0, -1)
    want = W.double().numpy() - float(np.float32(0.01)) * g
    assert (np.abs(_np(got[0]) - want) <= 2.0 ** -7 * np.abs(want) + 1e-5 * np.abs(want).max(1, keepdims=True)).all()
    assert torch.equal(got[0], got[1]) and not torch.equal(got[0], got[2])


def test_token_gradient_of_an_empty_batch():
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(0)
    _, tables = _tables(rng, [70], 16, "fp32")
    batch = emb.Batch(torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV), 2)
    layer = emb.TokenLayer(tables, opt="sgd", lr=0.1, max_tokens=4, max_seqs=2)
    dy, before = torch.zeros((0, 16), device=DEV), tables.weights.clone()
    grad = torch.ones((70, 16), device=DEV)
    layer.table_grad(batch, dy, grad, add=True)
    assert bool((grad == 1).all())
    layer.table_grad(batch, dy, grad)
    assert bool((grad == 0).all())
    layer.update(batch, dy)
    assert torch.equal(before, tables.weights)


def test_token_gradient_after_a_failed_dedup_touches_no_row():
    """The dedup's error bit is set from the host between the two calls."""
    import torch
    import paper_2112_02752_amd as emb
    rng, D, W, tables, batch, key, dy, dyv, R = _grad_setup((700, 256, [90], 8, 0, 0.5, 5), "fp32", "fp32")
    n = len(key)
    d = emb.DedupBuffers(DEV, n, 8, D)
    emb.unique_ids(tables, batch, d.unique_keys, d.counts, d.seg_offsets, d.sort_perm, d.num_unique, d.ws)
    at = emb.workspace_error_offset()
    words = d.ws[:256].view(torch.int32)
    words[at // 4 + 1] = words[0]       # the call's generation
    words[at // 4] = 1                  # a wait of the dedup ran out
    before = tables.weights.clone()
    emb.token_grad(tables, batch, dyv, d, opt="sgd", lr=0.1)
    assert torch.equal(before, tables.weights)
    grad = torch.ones((R, D), device=DEV)
    emb.token_grad(tables, batch, dyv, d, grad=grad, layout="table_add")
    assert bool((grad == 1).all())
    emb.token_grad(tables, batch, dyv, d, grad=grad, layout="table")
    assert bool((grad == 0).all())
    rows = torch.ones((n, D), device=DEV)
    emb.token_grad(tables, batch, dyv, d, grad=rows, layout="rows")
    assert bool((rows == 0).all())


# ---------------------------------------------------------------- recurrence

def _sigmoid(z):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-z))


def _plain_forward(offs, x, f, o, bias, h0, keep=None):
    """States before and after each position, y and last states; `keep`: another
    pass's states before every 64th position, from which this one goes on."""
    n, D = x.shape
    M = len(offs) - 1
    z = f + (bias if bias is not None else 0)
    a, q = _sigmoid(z), _sigmoid(-z)
    before, h = np.zeros((n, D)), np.zeros((n, D))
    last = np.zeros((M, D))
    for m in range(M):
        s = h0[m].copy() if h0 is not None else np.zeros(D)
        for t in range(offs[m], offs[m + 1]):
            if keep is not None and t % 64 == 0 and t > offs[m]:
                s = keep[t]
            before[t] = s
            s = a[t] * s + q[t] * x[t]
            h[t] = s
        last[m] = s
    y = h * _sigmoid(o) if o is not None else h.copy()
    return a, q, before, h, y, last


def _plain_backward(offs, x, a, q, before, h, o, dy, dh_last):
    n, D = x.shape
    M = len(offs) - 1
    s = _sigmoid(o) if o is not None else np.ones((n, D))
    dh, dh0 = np.zeros((n, D)), np.zeros((M, D))
    for m in range(M):
        back = dh_last[m].copy() if dh_last is not None else np.zeros(D)
        for t in range(offs[m + 1] - 1, offs[m] - 1, -1):
            dh[t] = s[t] * dy[t] + back
            back = a[t] * dh[t]
        dh0[m] = back
    dx = q * dh
    df = dh * (before - x) * a * q
    do = dy * h * s * (1 - s)
    return dh, dx, df, do, df.sum(0), dh0


def _lengths(kind, rng):
    return {
        "one": [1], "two": [2], "edge": [15, 16, 17, 63, 64, 65, 1], "span": [64, 128, 64], "long": [700],
        "ragged": list(rng.integers(1, 90, 12)), "empties": [0, 0, 5, 0, 70, 0, 0, 64, 0],
        "many_empties": [3] + [0] * 200 + [40, 0, 0, 30] + [0] * 70 + [1] * 40, "ones": [1] * 150,
        "first_empty": [0] * 130 + [20], "nothing": [0, 0, 0], "tail": [100, 27]}[kind]


def _scan_inputs(kind, D, dtype, seed, gated=True, gap=0, shift=0, wide=False):
    import torch
    rng = np.random.default_rng(seed)
    lens = _lengths(kind, rng)
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    n, M = int(offs[-1]), len(lens)
    mats, views = [], []
    for i in range(4):
        v = torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32) * (1.5 if i == 1 else 1.0)).to(_dt(dtype))
        views.append(_strided(v, gap, shift, _dt(dtype))[0])
        mats.append(v.double().numpy())
    bias = (np.linspace(-2, 5, D) if D > 1 else np.array([1.0])).astype(np.float32)
    h0, dhl = rng.standard_normal((2, M, D)).astype(np.float32)
    if not gated:
        mats[2] = views[2] = None
    return rng, offs, n, M, mats, views, bias, h0, dhl


def _steps(T, q):
    """How many steps' errors add up: as many as the slowest gate remembers."""
    return 1.0 + (min(float(T), float(1 / q.min())) if q.size else 0.0)


def _check_scan(kind, D, dtype, gated, with_all, gap=0, shift=0, saved=False):
    import torch
    import paper_2112_02752_amd as emb
    _say("scan", kind, D, dtype, gated, with_all, gap, shift, saved)
    rng, offs, n, M, (x, f, o, dy), (xv, fv, ov, dyv), bias, h0, dhl = _scan_inputs(kind, D, dtype, D + 13, gated, gap,
                                                                                   shift)
    if not with_all:
        bias = h0 = dhl = None
    dev = lambda v: torch.from_numpy(v).to(DEV) if v is not None else None  # noqa: E731
    t = _dt(dtype)
    scan = emb.Scan(dev(offs), xv, fv, ov, bias=dev(bias), h0=dev(h0))
    rec = emb.Recurrence(n, M, D)
    y, ybuf = _strided(np.zeros((n, D)), gap, shift, t)
    last = torch.full((M, D), 9.0, device=DEV)
    rec.forward(scan, y, last)
    a, q, before, h, y_w, last_w = _plain_forward(offs, x, f, o, bias, h0)
    T = int(max(offs[1:] - offs[:-1]))
    steps = _steps(T, q)
    top = max(1e-30, *(np.abs(v).max() for v in (x, h0) if v is not None and v.size)) if n else 1.0
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    tol = 32 * U * steps * top
    assert (np.abs(_np(y) - y_w) <= tol + half * np.abs(y_w)).all()
    assert (np.abs(_np(last) - last_w) <= tol).all()
    back = scan
    if saved:
        cks = []
        for v in (xv, fv, ov):
            if v is None:
                cks.append(None)
                continue
            ck = emb.Checkpoint(n, D)
            ck.pack(v)
            cks.append(ck)
        x, f, o = (_saved_plain(v)[2] if v is not None else None for v in (x, f, o))
        a, q, before, h, _, _ = _plain_forward(offs, x, f, o, bias, h0, keep=before)
        back = emb.Scan(dev(offs), *(c.columns(0, D) if c else None for c in cks), bias=dev(bias), h0=dev(h0))
        steps = _steps(T, q)
    dx, df, do = (_strided(np.zeros((n, D)), gap, shift, t)[0] for _ in range(3))
    db, dh0 = torch.full((D,), 9.0, device=DEV), torch.full((M, D), 9.0, device=DEV)
    rec.backward(back, dyv, dx, df, do if gated else None, dbias=db, dh_last=dev(dhl), dh0=dh0)
    dh, dx_w, df_w, do_w, db_w, dh0_w = _plain_backward(offs, x, a, q, before, h, o, dy, dhl)
    gtop = max(1.0, np.abs(dh).max()) if n else 1.0
    tol_g = 32 * U * steps * gtop
    tol_f = 4 * 32 * U * steps * gtop * max(top, 1.0)
    assert (np.abs(_np(dx) - dx_w) <= tol_g + half * np.abs(dx_w)).all()
    assert (np.abs(_np(df) - df_w) <= tol_f + half * np.abs(df_w)).all()
    if gated:
        assert (np.abs(_np(do) - do_w) <= tol_f + half * np.abs(do_w)).all()
    assert (np.abs(_np(db) - db_w) <= 2 * tol_f + (70 * U) * np.abs(df_w).sum(0) + tol_f * np.sqrt(n + 1)).all()
    if n == 0 or M:
        assert (np.abs(_np(dh0) - dh0_w) <= tol_g).all()
    # the same again, bit for bit
    y2, last2 = torch.empty_like(y), torch.empty_like(last)
    rec.forward(scan, y2, last2)
    assert torch.equal(y2, y) and torch.equal(last2, last)


KINDS = ["one", "two", "edge", "span", "long", "ragged", "empties", "many_empties", "ones", "first_empty", "nothing",
         "tail"]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_scan(kind, dtype):
    _check_scan(kind, 130, dtype, True, True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D,gated,with_all,gap,shift", [
    (1, True, True, 0, 0), (2, False, True, 0, 0), (3, True, False, 5, 0), (64, False, False, 0, 1), (100, True, True, 3, 0),
    (128, True, False, 2, 2), (257, True, True, 1, 1)])
def test_scan_widths_and_strides(D, gated, with_all, gap, shift, dtype):
    for kind in ("ragged", "empties"):
        _check_scan(kind, D, dtype, gated, with_all, gap, shift)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind,D,gated", [("edge", 64, True), ("ragged", 100, True), ("long", 31, False),
                                          ("many_empties", 160, True)])
def test_scan_backward_from_checkpoints(kind, D, gated, dtype):
    _check_scan(kind, D, dtype, gated, True, saved=True)


def test_scan_of_a_long_sequence():
    """20001 steps with gates that remember up to 400 of them."""
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(5)
    n, D = 20001, 66
    x, f, o = rng.standard_normal((3, n, D)).astype(np.float32)
    bias = np.linspace(-1, 6, D).astype(np.float32)
    offs = np.array([0, n], dtype=np.int32)
    dev = lambda v: torch.from_numpy(v).to(DEV)  # noqa: E731
    rec = emb.Recurrence(n, 1, D, train=False)
    y, last = torch.empty(n, D, device=DEV), torch.empty(1, D, device=DEV)
    rec.forward(emb.Scan(dev(offs), dev(x), dev(f), dev(o), bias=dev(bias)), y, last)
    a, q, before, h, y_w, last_w = _plain_forward(offs, *(v.astype(np.float64) for v in (x, f, o, bias)), None)
    tol = 32 * U * _steps(n, q) * np.abs(x).max()
    assert (np.abs(_np(y) - y_w) <= tol).all() and (np.abs(_np(last) - last_w) <= tol).all()


def test_scan_gradient_against_differences():
    """The gradient along random directions against central differences of the
    64-bit forward: an error of (1e-4)^2 times third derivatives of a few units,
    and the fp32 gradient's own over about a thousand values."""
    import torch
    import paper_2112_02752_amd as emb
    rng, offs, n, M, (x, f, o, _), _, bias, h0, dhl = _scan_inputs("edge", 24, "fp32", 3)
    w, wl = rng.standard_normal((n, 24)), dhl.astype(np.float64)
    parts = [v.astype(np.float64) for v in (x, f, o, bias, h0)]

    def loss(v):
        out = _plain_forward(offs, *v)
        return (out[4] * w).sum() + (out[5] * wl).sum()

    dev = lambda v: torch.from_numpy(np.asarray(v, dtype=np.float32)).to(DEV)  # noqa: E731
    rec = emb.Recurrence(n, M, 24)
    scan = emb.Scan(torch.from_numpy(offs).to(DEV), dev(x), dev(f), dev(o), bias=dev(bias), h0=dev(h0))
    g = [torch.empty(n, 24, device=DEV) for _ in range(3)] + [torch.empty(24, device=DEV),
                                                                torch.empty(M, 24, device=DEV)]
    rec.forward(scan, torch.empty(n, 24, device=DEV))
    rec.backward(scan, dev(w), g[0], g[1], g[2], dbias=g[3], dh_last=dev(wl), dh0=g[4])
    for i in range(5):
        v = rng.standard_normal(parts[i].shape)
        up, down = list(parts), list(parts)
        up[i], down[i] = parts[i] + 1e-4 * v, parts[i] - 1e-4 * v
        diff = (loss(up) - loss(down)) / 2e-4
        along = (_np(g[i]) * v).sum()
        size = np.abs(_np(g[i]) * v).sum()
        assert abs(diff - along) <= 1e-5 * size, (i, diff, along)


def test_scan_keeps_infinities_and_nan_within_their_sequence_and_column():
    import torch
    import paper_2112_02752_amd as emb
    n, D, M = 200, 6, 4
    offs = np.array([0, 70, 130, 130, n], dtype=np.int32)
    rng = np.random.default_rng(8)
    x, f, o, dy = rng.standard_normal((4, n, D)).astype(np.float32)
    clean = [v.copy() for v in (x, f, o, dy)]
    x[75, 1], f[80, 2], o[90, 3], dy[100, 4] = np.nan, np.nan, np.nan, np.inf
    x[60, 5] = np.inf
    f[10:20, 0], f[140:150, 0] = np.inf, -np.inf     # gates shut and open for good: finite
    clean[1][10:20, 0], clean[1][140:150, 0] = np.inf, -np.inf

    def go(x, f, o, dy):
        d = lambda v: torch.from_numpy(v).to(DEV)  # noqa: E731
        rec = emb.Recurrence(n, M, D)
        scan = emb.Scan(d(offs), d(x), d(f), d(o))
        y, last = torch.empty(n, D, device=DEV), torch.empty(M, D, device=DEV)
        g = [torch.empty(n, D, device=DEV) for _ in range(3)]
        dh0 = torch.empty(M, D, device=DEV)
        rec.forward(scan, y, last)
        rec.backward(scan, d(dy), *g, dh0=dh0)
        return [v.cpu().numpy() for v in (y, last, *g, dh0)]

    got, want = go(x, f, o, dy), go(*clean)
    for v in want:
        assert np.isfinite(v).all()
    seq = np.repeat([0, 1, 3], [70, 60, 70])
    dirty = {(1, 1), (1, 2), (1, 3), (1, 4), (0, 5)}
    for v, w in zip(got, want):
        for m in range(M):
            for c in range(D):
                if (m, c) not in dirty:
                    rows = seq == m if v.shape[0] == n else np.arange(M) == m
                    assert np.array_equal(v[rows, c], w[rows, c]), (m, c)
    y = got[0]
    assert np.isnan(y[75:130, 1]).all() and np.isfinite(y[70:75, 1]).all()
    assert np.isnan(y[80:130, 2]).all() and np.isnan(y[90, 3]) and np.isfinite(y[91:130, 3]).all()
    assert not np.isfinite(y[60:70, 5]).any()
    assert np.isnan(got[1][1, 1]) and np.isnan(got[1][1, 2])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D,gated,gap", [(1, True, 0), (64, False, 0), (100, True, 1), (258, True, 2)])
def test_scan_step_follows_the_scan(D, gated, gap, dtype):
    """Five tokens of each of seven sequences one by one, in slots in any order,
    against the whole sequences: the same gates and products, within two more
    roundings a step."""
    import torch
    import paper_2112_02752_amd as emb
    rng = np.random.default_rng(D)
    M, T = 7, 5
    t = _dt(dtype)
    mats = [torch.from_numpy(rng.standard_normal((M * T, D)).astype(np.float32)).to(t) for _ in range(3)]
    bias = torch.from_numpy(rng.standard_normal(D).astype(np.float32)).to(DEV)
    h0 = torch.from_numpy(rng.standard_normal((M, D)).astype(np.float32)).to(DEV)
    offs = torch.arange(0, M * T + 1, T, dtype=torch.int32, device=DEV)
    rec = emb.Recurrence(M * T, M, D, train=False)
    y, last = torch.empty(M * T, D, dtype=t, device=DEV), torch.empty(M, D, device=DEV)
    d = [m.to(DEV) for m in mats]
    rec.forward(emb.Scan(offs, d[0], d[1], d[2] if gated else None, bias=bias, h0=h0), y, last)
    pool = torch.full((12, D), 3.0, device=DEV)
    order = torch.from_numpy(rng.permutation(12)[:M].astype(np.int32)).to(DEV)
    pool[order.long()] = h0
    for k in range(T):
        rows = [_strided(m[k::T], gap, 0, t)[0] for m in mats]
        yk, _ = _strided(np.zeros((M, D)), gap, 0, t)
        emb.scan_step(rows[0], rows[1], rows[2] if gated else None, pool, yk, bias=bias, slots=order)
        tol = 4 * U * T * 4 + (2.0 ** -8 if dtype == "bf16" else 0) * np.abs(_np(y[k::T]))
        assert (np.abs(_np(yk) - _np(y[k::T])) <= tol).all()
    assert (np.abs(_np(pool[order.long()]) - _np(last)) <= 4 * U * T * 4).all()
    others = [i for i in range(12) if i not in order.tolist()]
    assert bool((pool[others] == 3.0).all())


def test_scan_step_without_a_slot():
    import torch
    import paper_2112_02752_amd as emb
    x, f, o = torch.randn(3, 5, 8, device=DEV)
    state, y = torch.ones(4, 8, device=DEV), torch.full((5, 8), 7.0, device=DEV)
    emb.scan_step(x, f, o, state, y, slots=torch.tensor([2, -1, 4, 0, 1 << 30], dtype=torch.int32, device=DEV))
    assert bool((y[[1, 2, 4]] == 0).all()) and bool((y[[0, 3]] != 0).all())
    assert bool((state[[1, 3]] == 1).all()) and bool((state[[0, 2]] != 1).all())
    emb.scan_step(x[:0], f[:0], o[:0], state, y[:0])


# ---------------------------------------------------------------- checkpoints

def _saved_plain(x):
    """Codes, exponents and restored values of a float64 array."""
    n, d = x.shape
    groups = (d + 31) // 32
    p = np.zeros((n, groups * 32))
    p[:, :d] = x
    p = p.reshape(n, groups, 32)
    top = np.abs(p).max(2)
    fine = np.isfinite(top)
    with np.errstate(invalid="ignore"):
        part, e = np.frexp(np.where(fine, top, 1.0) / 127)
    e = np.clip(np.where(part == 0.5, e - 1, e), -120, 121)
    e = np.where(top == 0, -120, e)
    unit = np.ldexp(1.0, e)[:, :, None]
    with np.errstate(invalid="ignore"):
        codes = np.where(fine[:, :, None], np.clip(np.rint(p / unit), -127, 127), 0)
    back = np.where(fine[:, :, None], codes * unit, np.nan).reshape(n, -1)[:, :d]
    return codes.reshape(n, -1).astype(np.int8), np.where(fine, e + 127, 255).astype(np.uint8), back


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,D,gap,shift", [(1, 1, 0, 0), (3, 31, 0, 0), (5, 32, 0, 0), (64, 33, 7, 0), (100, 200, 0, 1),
                                           (33, 256, 8, 0), (1000, 100, 1, 0), (2, 2056, 0, 0)])
def test_saved_activations(n, D, gap, shift, dtype):
    import torch
    import paper_2112_02752_amd as emb
    _say("save", n, D, gap, shift, dtype)
    rng = np.random.default_rng(n + D)
    x = (rng.standard_normal((n, D)) * np.exp(3 * rng.standard_normal((n, 1)))).astype(np.float32)
    x[rng.random((n, D)) < 0.05] = 0
    xt = torch.from_numpy(x).to(_dt(dtype))
    codes, exps, back = _saved_plain(xt.double().numpy())
    v, _ = _strided(xt, gap, shift, _dt(dtype))
    ck = emb.Checkpoint(n, D)
    ck.codes.fill_(55)
    ck.pack(v)
    assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.exps.cpu().numpy(), exps)
    for out in ("fp32", "bf16"):
        r, buf = _strided(np.zeros((n, D)), gap, shift, _dt(out))
        ck.unpack(r)
        assert np.array_equal(_np(r), back)      # exact in both types
        assert int((buf == 77.0).sum()) >= buf.numel() - n * D - int((back == 77.0).sum())


def test_saved_activations_at_the_types_ends():
    import torch
    import paper_2112_02752_amd as emb
    big = float(np.finfo(np.float32).max)
    rows = np.zeros((10, 64), dtype=np.float32)
    rows[0, :3] = [big, -big, 1.0]                       # saturates at 127 * 2^121
    rows[1, :2] = [127.0, 0.5]                           # 127 * 2^0: ties of 0.5 to even
    rows[2, :4] = [127.0, 1.5, 2.5, -2.5]
    rows[3, :2] = [np.nextafter(np.float32(127.0), np.float32(200)), 1.0]   # just above: the next exponent
    rows[4, :2] = [1e-45, -1e-45]                        # below the smallest unit: zeros
    rows[5, :2] = [2.0 ** -120, 127 * 2.0 ** -120]
    rows[6, 5], rows[6, 40] = np.nan, 3.0                # one group lost, the other not
    rows[7, 63] = -np.inf
    rows[8, 0] = 2.0 ** -100
    codes, exps, back = _saved_plain(rows.astype(np.float64))
    ck = emb.Checkpoint(10, 64)
    ck.pack(torch.from_numpy(rows).to(DEV))
    assert np.array_equal(ck.codes.cpu().numpy(), codes) and np.array_equal(ck.exps.cpu().numpy(), exps)
    r = torch.empty(10, 64, device=DEV)
    ck.unpack(r)
    got = _np(r)
    assert np.array_equal(got, back, equal_nan=True)
    assert np.isnan(got[6, :32]).all() and got[6, 40] == 3.0 and np.isnan(got[7, 32:]).all()
    assert got[0, 0] == 127 * 2.0 ** 121 and np.isfinite(got[0, :32]).all()


# ---------------------------------------------------------------- weight gradient

@pytest.mark.parametrize("dy_type", ["bf16", "fp32"])
@pytest.mark.parametrize("n,K,F,gap,shift", [(1, 32, 8, 0, 0), (63, 64, 100, 0, 0), (64, 128, 128, 0, 0), (65, 33, 129, 0, 0),
                                             (300, 200, 7, 1, 0), (1000, 130, 260, 4, 0), (2500, 96, 64, 0, 1),
                                             (4100, 257, 384, 8, 0)])
def test_weight_gradient(n, K, F, gap, shift, dy_type):
    import torch
    import paper_2112_02752_amd as emb
    _say("weight gradient", n, K, F, gap, shift, dy_type)
    rng = np.random.default_rng(n + K + F)
    x = torch.from_numpy(rng.standard_normal((n, K)).astype(np.float32)).to(DEV)
    ck = emb.Checkpoint(n, K)
    ck.pack(x)
    back = _saved_plain(x.double().cpu().numpy())[2]
    dy = torch.from_numpy(rng.standard_normal((n, F)).astype(np.float32)).to(_dt(dy_type))
    dyv, _ = _strided(dy, gap, shift, _dt(dy_type))
    y = dy.double().numpy()
    dw = torch.full((K, F), 5.0, device=DEV)
    ck.weight_grad(dyv, dw)
    want, mag = back.T @ y, np.abs(back).T @ np.abs(y)
    tol = (n + 8) * 2 * U * mag
    assert (np.abs(_np(dw) - want) <= tol).all()
    # most of the error bound is never used: all together stay within 8 units of fp32 for the square root of n sums
    assert np.linalg.norm(_np(dw) - want) <= 8 * 2 * U * np.sqrt(n + 1) * np.linalg.norm(mag) / np.sqrt(n + 1)
    first = dw.clone()
    ck.weight_grad(dyv, dw, add=True)
    assert (np.abs(_np(dw) - 2 * _np(first)) <= 2 * U * np.abs(_np(first)) * 2).all()
    ck.weight_grad(dyv, dw)
    assert torch.equal(dw, first)


def test_weight_gradient_of_no_rows_and_of_infinities():
    import torch
    import paper_2112_02752_amd as emb
    ck = emb.Checkpoint(0, 40)
    dw = torch.ones(40, 24, device=DEV)
    ck.weight_grad(torch.zeros(0, 24, device=DEV), dw, add=True)
    assert bool((dw == 1).all())
    ck.weight_grad(torch.zeros(0, 24, device=DEV), dw)
    assert bool((dw == 0).all())
    x = torch.ones(70, 64, device=DEV)
    x[3, 40] = float("nan")
    ck = emb.Checkpoint(70, 64)
    ck.pack(x)
    for t in (torch.float32, torch.bfloat16):
        dy = torch.ones(70, 24, dtype=t, device=DEV)
        dy[5, 2] = float("inf")
        dw = torch.zeros(64, 24, device=DEV)
        ck.weight_grad(dy, dw)
        dw = dw.cpu()
        assert bool(torch.isnan(dw[32:]).all())             # the group that held a NaN
        assert bool((dw[:32, 2] == float("inf")).all())
        assert bool((dw[:32, :2] == 70).all()) and bool((dw[:32, 3:] == 70).all())


# ---------------------------------------------------------------- streams and graphs

def test_operators_on_another_stream_and_in_a_graph():
    """The recurrence both ways, a checkpoint and the weight gradient captured
    once, replayed with new inputs and eager work between, and run on a side
    stream: each equal to the eager result bit for bit."""
    import torch
    import paper_2112_02752_amd as emb
    n, D, F = 300, 96, 64
    offs = torch.tensor([0, 100, 100, 231, n], dtype=torch.int32, device=DEV)
    x, f, o, dy = (torch.randn(n, D, device=DEV).bfloat16() for _ in range(4))
    bias = torch.randn(D, device=DEV)
    rec, ck = emb.Recurrence(n, 4, D), emb.Checkpoint(n, D)
    scan = emb.Scan(offs, x, f, o, bias=bias)
    outs = [torch.empty_like(x) for _ in range(4)] + [torch.empty(4, D, device=DEV), torch.empty(D, device=DEV),
                                                       torch.empty(D, D, device=DEV)]

    def go(stream=None):
        rec.forward(scan, outs[0], outs[4], stream=stream)
        rec.backward(scan, dy, *outs[1:4], dbias=outs[5], stream=stream)
        ck.pack(x, stream=stream)
        ck.weight_grad(outs[1], outs[6], stream=stream)

    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    side = torch.cuda.Stream()
    for k in range(4):
        for v in (x, f, o, dy):
            v.copy_(torch.randn(n, D, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in outs]
        go()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), k
        for v in outs:
            v.zero_()
        side.wait_stream(torch.cuda.current_stream())
        go(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), k
