"""Operators over sequences where sizes, contents, streams or the caller's own
objects are at an edge; tolerances as in test_gpu_sequence."""
import numpy as np
import pytest

from tests.test_gpu_sequence import U, _dt, _np, _saved_plain

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


# ---------------------------------------------------------------- weight gradient

@pytest.mark.parametrize("n,K,F", [(8192, 64, 12800), (8192, 12800, 64), (32768, 32, 5400), (4099, 2080, 2313)])
def test_weight_gradient_of_large_tiles_that_the_matrix_ends_in(n, K, F):
    """Sizes whose tiles are large and whose last tile's second group of columns
    lies past the matrix."""
    import torch
    import paper_2112_02752_amd as emb
    g = torch.Generator(device=DEV).manual_seed(n + K)
    x = torch.randn((n, K), generator=g, device=DEV).bfloat16()
    dy = torch.randn((n, F), generator=g, device=DEV).bfloat16()
    ck = emb.Checkpoint(n, K)
    ck.pack(x)
    back = torch.empty((n, K), device=DEV)
    ck.unpack(back)
    dw = torch.full((K, F), 5.0, device=DEV)
    ck.weight_grad(dy, dw)
    b, y = back.double(), dy.double()
    want, mag = b.t().contiguous() @ y, b.abs().t().contiguous() @ y.abs()
    assert bool(((dw.double() - want).abs() <= (n + 8) * 2 * U * mag).all())
    assert float((dw.double() - want).norm()) <= 8 * 2 * U * float(mag.norm())


def test_weight_gradients_on_another_stream_keep_to_their_own_workspace():
    """Calls that cut the rows into parts, queued behind other work on a side
    stream, of few columns first and then of more: what the current stream
    allocates and fills meanwhile keeps its values, and the results are the
    current stream's."""
    import torch
    import paper_2112_02752_amd as emb
    n, K, widths = 4096, 256, (256, 640, 256)
    g = torch.Generator(device=DEV).manual_seed(3)
    ck = emb.Checkpoint(n, K)
    ck.pack(torch.randn((n, K), generator=g, device=DEV).bfloat16())
    dys = [torch.randn((n, w), generator=g, device=DEV).bfloat16() for w in widths]
    sizes = [emb.lib().emb_weight_grad_workspace_size(n, K, w) for w in widths]
    assert all(sizes) and sizes[1] > sizes[0]
    busy = torch.randn((8192, 8192), generator=g, device=DEV).bfloat16()
    for as_int in (False, True):
        outs = [torch.zeros((K, w), device=DEV) for w in widths]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(10):
                busy @ busy
        filled = []
        for dy, dw, size in zip(dys, outs, sizes):
            ck.weight_grad(dy, dw, stream=side.cuda_stream if as_int else side)
            filled += [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for _ in range(2)]
        torch.cuda.synchronize()
        assert all(bool((f == 7).all()) for f in filled)
        for dy, dw in zip(dys, outs):
            want = torch.empty_like(dw)
            ck.weight_grad(dy, want)
            assert torch.equal(dw, want)


def test_weight_gradient_of_any_nan():
    """A column of dy with a NaN of any bits gives NaN, the others sums of ones."""
    import torch
    import paper_2112_02752_amd as emb
    bits = [0x7f800001, 0x7f80ffff, 0xff800001 - 2 ** 32, 0x7fc00000, 0x7fbfffff, 0xffffffff - 2 ** 32]
    dy = torch.ones(70, 24, device=DEV)
    for i, b in enumerate(bits):
        dy.view(torch.int32)[11 * i, 2 * i] = b
    assert dy.isnan().sum() == len(bits)
    ck = emb.Checkpoint(70, 64)
    ck.pack(torch.ones(70, 64, device=DEV))
    dw = torch.zeros(64, 24, device=DEV)
    ck.weight_grad(dy, dw)
    dirty = torch.zeros(24, dtype=torch.bool, device=DEV)
    dirty[0:2 * len(bits):2] = True
    assert bool(dw[:, dirty].isnan().all()) and bool((dw[:, ~dirty] == 70).all())


# ---------------------------------------------------------------- the sequence layer

def _layer(opt, state, lens=(7, 0, 30, 1, 66), R=50, D=40, H=32, seed=4, **kw):
    import torch
    import paper_2112_02752_amd as emb
    g = torch.Generator().manual_seed(seed)
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    n, M = int(offs[-1]), len(lens)
    tables = emb.Tables(torch.randn((R, D), generator=g).to(DEV), [0, R])
    weight = (torch.randn((D, 3 * H), generator=g) * D ** -0.5).bfloat16().to(DEV)
    bias = torch.linspace(-1, 3, H, device=DEV)
    layer = emb.SequenceLayer(tables, weight, bias, n, M, opt=opt, lr=0.1, state=state, **kw)
    batch = emb.Batch(torch.from_numpy(offs).to(DEV), torch.randint(0, R, (n,), generator=g).to(DEV), M)
    dy = torch.randn((n, H), generator=g).bfloat16().to(DEV)
    y = torch.empty((n, H), dtype=torch.bfloat16, device=DEV)
    return layer, batch, y, dy


def test_a_refused_backward_runs_nothing_and_can_be_repeated():
    import torch
    import paper_2112_02752_amd as emb
    for opt in (None, "adagrad"):
        layer, batch, y, dy = _layer(opt, None)
        layer.forward(batch, y)
        dw, db = torch.full((40, 96), 5.0, device=DEV), torch.full((32,), 5.0, device=DEV)
        with pytest.raises(ValueError, match="optimizer|accumulators"):
            layer.backward(batch, dy, dw, db)
        torch.cuda.synchronize()
        assert bool((dw == 5).all()) and bool((db == 5).all())
        with pytest.raises(ValueError, match="optimizer|accumulators"):
            layer.tokens.update(batch, torch.zeros((dy.shape[0], 40), dtype=torch.bfloat16, device=DEV))
    layer, batch, y, dy = _layer("sgd", None)
    plain, batch2, y2, dy2 = _layer("sgd", None)
    layer.forward(batch, y)
    plain.forward(batch2, y2)
    fewer = emb.Batch(batch.offsets[:-1].contiguous(), batch.indices, 4)
    bad = [dict(dy=dy.float()), dict(dy=dy[:-1]), dict(dweight=dw[:-1]), dict(dbias=db[:-1]), dict(dweight=None),
           dict(dh_last=torch.zeros(4, 32, device=DEV)), dict(dh0=torch.zeros(5, 31, device=DEV)), dict(batch=fewer)]
    before = layer.tokens.tables.weights.clone()
    for kw in bad:
        args = dict(dict(batch=batch, dy=dy, dweight=dw, dbias=db), **kw)
        with pytest.raises(ValueError):
            layer.backward(**args)
    torch.cuda.synchronize()
    assert bool((dw == 5).all()) and bool((db == 5).all()) and torch.equal(before, layer.tokens.tables.weights)
    dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
    layer.backward(batch, dy, dw, db)
    plain.backward(batch2, dy2, dw2, db2)
    assert torch.equal(dw, dw2) and torch.equal(db, db2)
    assert torch.equal(layer.tokens.tables.weights, plain.tokens.tables.weights)


def test_gradients_of_two_batches_added():
    """With ``add`` the weights' and the bias's gradients both hold the sums (one
    more rounding of each: 2^-24, and the weights' sums meet what is there)."""
    import torch
    got = []
    for add in (False, True):
        sums = []
        layer, batch, y, dy = _layer("sgd", None)
        layer.tokens._updc.lr = 0.0
        dw, db = torch.zeros((40, 96), device=DEV), torch.zeros(32, device=DEV)
        for k in range(2):
            layer.forward(batch, y)
            layer.backward(batch, dy * (k + 1), dw, db, add=add)
            sums.append((dw.double().cpu(), db.double().cpu()))
        got.append(sums)
    for i in range(2):
        parts = [s[i] for s in got[0]]
        want = parts[0] + parts[1]
        mag = parts[0].abs() + parts[1].abs()
        assert bool(((got[1][1][i] - want).abs() <= 4 * U * mag).all())
    layer.forward(batch, y)
    layer.backward(batch, dy, dw, None, add=True)


def test_first_states_may_be_written_to_before_the_backward():
    """States carried from batch to batch in one buffer: the last states written
    over the first ones, or another batch's put there, change no gradient."""
    import torch
    got = []
    for kind in ("apart", "same", "later"):
        layer, batch, y, dy = _layer("sgd", None)
        state = torch.randn((5, 32), generator=torch.Generator().manual_seed(3)).to(DEV)
        last = state if kind == "same" else torch.empty_like(state)
        layer.forward(batch, y, last, h0=state)
        if kind == "later":
            state.copy_(last)
        dw, db, dh0 = (torch.empty(s, device=DEV) for s in ((40, 96), (32,), (5, 32)))
        layer.backward(batch, dy, dw, db, dh0=dh0)
        got.append((y, last, dw, db, dh0, layer.tokens.tables.weights))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_a_layer_keeps_checkpoints_alone():
    """What a layer holds, beside its workspaces, before a training forward
    (nothing) and until its backward (codes and exponents of most tokens)."""
    import torch
    import paper_2112_02752_amd as emb
    n, D, H = 4096, 64, 64
    kw = dict(R=50, D=D, H=H)
    warm = _layer("sgd", None, lens=(n,), **kw)
    warm[0].forward(warm[1], warm[2])

    def held(layer):
        parts = [layer.recurrence.ws, layer.recurrence.states, layer.tokens.dedup.ws]
        parts += [v for v in vars(layer.tokens.dedup).values() if v is not layer.tokens.dedup.ws]
        parts += [layer.tokens.tables.weights, layer.weight, layer.bias]
        return sum(-(-v.numel() * v.element_size() // 512) * 512 for v in parts)

    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    layer, batch, y, dy = _layer("sgd", None, lens=(n,), **kw)
    mine = sum(-(-v.numel() * v.element_size() // 512) * 512 for v in (batch.offsets, batch.indices, y, dy))
    full = 2 * n * (D + 3 * H)
    assert torch.cuda.memory_allocated() - before - mine - held(layer) < full // 16
    layer.forward(batch, y, train=False)
    assert torch.cuda.memory_allocated() - before - mine - held(layer) < full // 16
    layer.forward(batch, y)
    kept = n * (D + 3 * H) * 33 // 32
    assert kept <= torch.cuda.memory_allocated() - before - mine - held(layer) < kept + full // 16


def test_steps_of_changing_lengths_are_those_of_a_fresh_layer():
    import torch
    lens = [(60, 3), (5,), (40, 0, 1), (90,), (1,)]
    long = _layer("sgd", None, lens=(120,))[0]
    for some in lens:
        fresh, batch, y, dy = _layer("sgd", None, lens=some)
        long.tokens.tables.weights.copy_(fresh.tokens.tables.weights)
        long.weight.copy_(fresh.weight)
        out = []
        for layer in (fresh, long):
            dw, db = torch.empty((40, 96), device=DEV), torch.empty(32, device=DEV)
            layer.forward(batch, y)
            layer.backward(batch, dy, dw, db)
            out.append((y.clone(), dw, db, layer.tokens.tables.weights.clone()))
        assert all(torch.equal(a, b) for a, b in zip(*out)), some


# ---------------------------------------------------------------- tokens

@pytest.mark.parametrize("bits", [32, 64])
@pytest.mark.parametrize("rows", [[10], [10, 5]])
def test_lookup_of_ids_outside_the_table(rows, bits):
    """Zeros for them, whatever their low 32 bits are; so too where those are
    the padding row's."""
    import torch
    import paper_2112_02752_amd as emb
    W = torch.arange(1, 1 + sum(rows) * 8, dtype=torch.float32, device=DEV).view(-1, 8)
    big = [2 ** 32 + 3, -2 ** 32 + 3, 2 ** 63 - 1, -2 ** 63, 2 ** 31, 2 ** 40] if bits == 64 else [2 ** 31 - 1, -2 ** 31]
    one = [3, 0, 10, -1] + big
    ids = one + ([4, 5, -1, 0] + big if len(rows) > 1 else [])
    offs = [0, len(one)] + ([len(ids)] if len(rows) > 1 else [])
    batch = emb.Batch(torch.tensor(offs, dtype=torch.int32, device=DEV),
                      torch.tensor(ids, dtype=torch.int64 if bits == 64 else torch.int32, device=DEV), 1)
    start = [0] + list(np.cumsum(rows))
    for pad in (-1, 3):
        out = torch.full((len(ids), 8), 7.0, device=DEV)
        emb.token_fwd(emb.Tables(W, start), batch, out, pad_row=pad)
        for j, i in enumerate(ids):
            t = 0 if j < len(one) else 1
            key = start[t] + i if 0 <= i < rows[t] else -1
            want = W[key] if key >= 0 and key != pad else torch.zeros(8, device=DEV)
            assert torch.equal(out[j], want), (j, i)


# ---------------------------------------------------------------- recurrence

def _run_scan(offs, x, f, o, dy, bias=None, h0=None, dhl=None, per_seq=True):
    """y, last states, dx, df, do, dbias, dh0 of one forward and backward (numpy)."""
    import torch
    import paper_2112_02752_amd as emb
    dev = lambda v: torch.from_numpy(np.ascontiguousarray(v)).to(DEV) if v is not None else None  # noqa: E731
    n, D = x.shape
    M = len(offs) - 1
    rec = emb.Recurrence(n, M, D)
    scan = emb.Scan(dev(offs), dev(x), dev(f), dev(o), bias=dev(bias), h0=dev(h0))
    y, g = torch.empty(n, D, device=DEV), [torch.empty(n, D, device=DEV) for _ in range(3)]
    db = torch.empty(D, device=DEV)
    last, dh0 = (torch.empty(M, D, device=DEV) if per_seq else None for _ in range(2))
    rec.forward(scan, y, last)
    rec.backward(scan, dev(dy), *g, dbias=db, dh_last=dev(dhl), dh0=dh0)
    return [v.cpu().numpy() if v is not None else None for v in (y, last, *g, db, dh0)]


@pytest.mark.parametrize("run", [1, 2, 3, 4, 5, 6, 7, 8, 15, 16, 17, 1000])
def test_scan_past_runs_of_empty_sequences(run):
    """The same values as without the empty sequences, bit for bit, and theirs
    handed through."""
    D = 5
    rng = np.random.default_rng(run)
    lens = [1, 3, 12, 16, 1, 128, 64, 2, 300, 1]
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    n, M = int(offs[-1]), len(lens)
    x, f, o, dy = rng.standard_normal((4, n, D)).astype(np.float32)
    h0, dhl = rng.standard_normal((2, M, D)).astype(np.float32)
    want = _run_scan(offs, x, f, o, dy, None, h0, dhl)
    # runs of `run` and run // 2 empty sequences before, between and after them
    more, real = [], []
    for m in range(M):
        more += [0] * (run if m % 2 == 0 else run // 2)
        real.append(len(more))
        more.append(lens[m])
    more += [0] * run
    h0m, dhlm = rng.standard_normal((2, len(more), D)).astype(np.float32)
    h0m[real], dhlm[real] = h0, dhl
    got = _run_scan(np.concatenate([[0], np.cumsum(more)]).astype(np.int32), x, f, o, dy, None, h0m, dhlm)
    empty = np.setdiff1d(np.arange(len(more)), real)
    for i in (0, 2, 3, 4, 5):
        assert np.array_equal(got[i], want[i]), i
    assert np.array_equal(got[1][real], want[1]) and np.array_equal(got[6][real], want[6])
    assert np.array_equal(got[1][empty], h0m[empty]) and np.array_equal(got[6][empty], dhlm[empty])


def test_scan_past_millions_of_empty_sequences():
    """Thirty million of them where the span begins, ends and in the middle: the
    spans after them wait for no walk along them."""
    n, D = 500, 3
    rng = np.random.default_rng(2)
    x, f, o, dy = rng.standard_normal((4, n, D)).astype(np.float32)
    places = [0, 128, 130, 300, n]
    want = _run_scan(np.array(places, dtype=np.int32), x, f, o, dy, per_seq=False)
    offs = np.repeat(np.array(places, dtype=np.int32), [6_000_001, 6_000_000, 6_000_003, 6_000_000, 6_000_000])
    got = _run_scan(offs, x, f, o, dy, per_seq=False)
    for i in (0, 2, 3, 4, 5):
        assert np.array_equal(got[i], want[i]), i


def test_gradient_of_an_output_gate_that_is_nearly_open_or_shut():
    """do = dy h s (1 - s) to fp32's precision of each factor: for a gate of |z|
    the exponent's rounding gives (|z| + 8) u of either factor's smaller one, the
    state and the products 8 u; sequences of one position, where h = x / 2."""
    z = np.array([-80, -60, -30, -16, -8, -2, -1e-3, 0, 1e-3, 2, 8, 12, 16, 20, 30, 60, 80], dtype=np.float32)
    n, D = 70, len(z)
    rng = np.random.default_rng(9)
    x, dy = rng.standard_normal((2, n, D)).astype(np.float32)
    o = np.tile(z, (n, 1))
    got = _run_scan(np.arange(n + 1, dtype=np.int32), x, np.zeros_like(x), o, dy)
    zd = o.astype(np.float64)
    want = dy.astype(np.float64) * x / 2 / ((1 + np.exp(-zd)) * (1 + np.exp(zd)))
    assert (np.abs(got[4] - want) <= (np.abs(zd) + 24) * U * np.abs(want)).all()
    # ends of the type: no gradient, no NaN
    o[:, 0], o[:, 1], o[:, 2], o[:, 3] = np.inf, -np.inf, 3e38, -3e38
    got = _run_scan(np.arange(n + 1, dtype=np.int32), x, np.zeros_like(x), o, dy)
    assert (got[4][:, :4] == 0).all() and np.isfinite(got[4]).all()


@pytest.mark.parametrize("n", [100, 300, 3000])
def test_scan_keeps_an_infinite_state_past_products_that_underflow(n):
    """An infinity in a sequence stays one to its end (gates of a half: their
    products underflow after 150 positions), and so does one in the gradient to
    its beginning; the other columns are finite."""
    from tests.test_gpu_sequence import _plain_backward, _plain_forward
    D = 6
    rng = np.random.default_rng(n)
    x, f, o, dy = rng.standard_normal((4, n, D)).astype(np.float32)
    f[:, 2:4] -= 4
    x[20, 0], x[20, 2], dy[n - 10, 1], dy[n - 10, 3] = np.inf, -np.inf, np.inf, -np.inf
    offs = np.array([0, 5, n], dtype=np.int32)
    h0 = rng.standard_normal((2, D)).astype(np.float32)
    got = _run_scan(offs, x, f, o, dy, None, h0, None)
    xd, fd, od, dyd = (v.astype(np.float64) for v in (x, f, o, dy))
    with np.errstate(invalid="ignore"):
        a, q, before, h, y, last = _plain_forward(offs, xd, fd, od, None, h0.astype(np.float64))
        dh, dx, df, do, db, dh0 = _plain_backward(offs, xd, a, q, before, h, od, dyd, None)
    assert np.isinf(y[20:, 0]).all() and np.isinf(dx[5:n - 9, 1]).all()
    for v, w in zip(got, (y, last, dx, df, do, None, dh0)):
        if w is not None:
            assert np.array_equal(np.isnan(v), np.isnan(w)) and np.array_equal(np.isinf(v), np.isinf(w))
            assert np.array_equal(np.sign(v[np.isinf(w)]), np.sign(w[np.isinf(w)]))


# ---------------------------------------------------------------- the caller's objects

def test_descriptors_follow_their_tensors():
    """Tensors that get other memory (as an optimizer or a checkpoint's loading
    gives a parameter) are read and written there; what they had stays alive
    beside them and keeps its values."""
    import torch
    import paper_2112_02752_amd as emb
    g = torch.Generator(device=DEV).manual_seed(6)
    n, M, D = 90, 3, 64
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    offs = torch.tensor([0, 40, 50, n], dtype=torch.int32, device=DEV)
    t = dict(x=rnd(n, D), f=rnd(n, D), o=rnd(n, D), bias=rnd(D), h0=rnd(M, D), offsets=offs)
    y, last = torch.empty(n, D, device=DEV), torch.empty(M, D, device=DEV)
    scan = emb.Scan(t["offsets"], t["x"], t["f"], t["o"], bias=t["bias"], h0=t["h0"])
    y_mat, rec = emb.Mat(y), emb.Recurrence(200, 5, D)
    rec.forward(scan, y_mat, last)

    def follows():
        rec.forward(scan, y_mat, last)
        want, want_last = torch.empty_like(y), torch.empty_like(last)
        rec.forward(emb.Scan(*(t[k].clone() for k in ("offsets", "x", "f", "o")), bias=t["bias"].clone(),
                             h0=t["h0"].clone()), want, want_last)
        assert torch.equal(y, want) and torch.equal(last, want_last)

    kept = []
    for name, new in (("x", rnd(n, D)), ("f", rnd(n, D)), ("o", rnd(n, D)), ("bias", rnd(D)), ("h0", rnd(M, D)),
                      ("offsets", torch.tensor([0, 7, 7, n], dtype=torch.int32, device=DEV))):
        kept.append(t[name].detach().clone()), kept.append(t[name].detach())
        t[name].data = new
        follows()
    kept.append(y.detach()), kept.append(y.clone())
    y.data = torch.empty(n, D, device=DEV)
    t["x"].data = rnd(n, D)
    follows()
    for a, b in zip(kept[::2], kept[1::2]):
        assert torch.equal(a, b)
    # a wider or longer one by its own rows
    for name in ("x", "f", "o"):
        t[name].data = rnd(n + 5, 2 * D)[:, :D]
    t["offsets"].data = torch.tensor([0, 40, 50, n + 5], dtype=torch.int32, device=DEV)
    y.data = torch.empty(n + 5, D, device=DEV)
    follows()
    t["bias"].data = rnd(D - 1)
    with pytest.raises(ValueError, match="bias"):
        rec.forward(scan, y_mat, last)
    t["bias"].data = rnd(D)
    t["f"].data = rnd(n, D)
    with pytest.raises(ValueError, match="f has"):
        rec.forward(scan, y_mat, last)


def test_accumulators_that_move_are_followed():
    import torch
    import paper_2112_02752_amd as emb
    W = torch.ones(10, 16, device=DEV)
    state = torch.zeros(10, device=DEV)
    layer = emb.TokenLayer(emb.Tables(W, [0, 10]), opt="adagrad", lr=0.1, state=state, max_tokens=4, max_seqs=1)
    batch = emb.Batch(torch.tensor([0, 2], dtype=torch.int32, device=DEV), torch.tensor([3, 5], device=DEV), 1)
    dy = torch.ones(2, 16, device=DEV)
    layer.update(batch, dy)
    old = state.detach()
    state.data = torch.full((10,), 2.0, device=DEV)
    layer.update(batch, dy)
    assert old.tolist() == [0, 0, 0, 1, 0, 1, 0, 0, 0, 0] and state.tolist() == [2, 2, 2, 3, 2, 3, 2, 2, 2, 2]
    state.data = torch.zeros(9, device=DEV)
    with pytest.raises(ValueError, match="accumulators"):
        layer.update(batch, dy)


# ---------------------------------------------------------------- failures

def test_a_recurrences_record_of_waits():
    """Sound calls leave no record, whatever the workspace held; one that is there
    (put there from the host) is reported until the workspace is initialised."""
    import torch
    import paper_2112_02752_amd as emb
    n, D = 700, 70
    g = torch.Generator(device=DEV).manual_seed(1)
    x, f, o, dy = (torch.randn((n, D), generator=g, device=DEV) for _ in range(4))
    scan = emb.Scan(torch.tensor([0, n], dtype=torch.int32, device=DEV), x, f, o)
    rec = emb.Recurrence(n, 1, D)
    outs = [torch.empty_like(x) for _ in range(4)]

    def both():
        rec.forward(scan, outs[0])
        rec.backward(scan, dy, *outs[1:])
        return [v.clone() for v in outs]

    want = both()
    rec.check()
    at = emb.workspace_error_offset()
    words = rec.ws[:256].view(torch.int32)
    words[at // 4] = 8
    with pytest.raises(emb.StepFailed, match="recurrence"):
        rec.check()
    assert all(torch.equal(a, b) for a, b in zip(both(), want))
    with pytest.raises(emb.StepFailed, match="recurrence"):
        rec.check()
    emb.workspace_init(rec.ws)
    rec.check()
    rec.ws.fill_(255)      # no call needs it initialised
    assert all(torch.equal(a, b) for a, b in zip(both(), want))


def test_the_sequence_layers_check():
    import torch
    import paper_2112_02752_amd as emb
    layer, batch, y, dy = _layer("sgd", None)
    layer.forward(batch, y)
    layer.backward(batch, dy, torch.empty((40, 96), device=DEV), torch.empty(32, device=DEV))
    layer.check()
    layer.recurrence.ws[:256].view(torch.int32)[emb.workspace_error_offset() // 4] = 8
    with pytest.raises(emb.StepFailed):
        layer.check()


def test_a_record_is_read_behind_another_streams_work():
    """The status asked for on a busy side stream is that stream's, not what the
    current stream finds meanwhile."""
    import torch
    import paper_2112_02752_amd as emb
    tables = emb.Tables(torch.ones(10, 16, device=DEV), [0, 10])
    tokens = emb.TokenLayer(tables, opt="sgd", lr=0.1, max_tokens=4, max_seqs=1)
    pooled = emb.Layer(tables, "sum", "sgd", 0.1, max_indices=4, max_bags=1)
    rec = emb.Recurrence(10, 1, 16)
    busy = torch.randn((8192, 8192), device=DEV).bfloat16()
    for obj, ws in ((tokens, tokens.dedup.ws), (pooled, pooled.ws), (rec, rec.ws)):
        obj.check()
        ws[:256].view(torch.int32)[emb.workspace_error_offset() // 4] = 8
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(10):
                busy @ busy
        with pytest.raises(emb.StepFailed):
            obj.check(stream=side)


def test_columns_of_a_matrix():
    """Columns named by their first and number are those of a slice."""
    import torch
    import paper_2112_02752_amd as emb
    wide = torch.randn(40, 200, device=DEV).bfloat16()
    for t in (wide, wide.float(), wide[:1], wide[:0]):
        for first, cols in ((0, 200), (32, 64), (64, 1), (199, 1), (200, 0)):
            a, b = emb.Mat(t, cols=cols, first=first), emb.Mat(t[:, first:first + cols]) if cols else None
            if b is not None and t.shape[0]:
                assert (a.rows, a.cols, a.c().data, a.c().dtype) == (b.rows, b.cols, b.c().data, b.c().dtype)
                assert t.shape[0] == 1 or a.c().ld == b.c().ld
        for first, cols in ((-1, 3), (0, 201), (190, 11), (201, None)):
            with pytest.raises(ValueError, match="columns"):
                emb.Mat(t, cols=cols, first=first)
    ck = emb.Checkpoint(40, 200)
    ck.pack(wide)
    back = torch.empty(40, 200, device=DEV)
    ck.unpack(back)
    for first, cols in ((0, 200), (32, 64), (160, 40), (192, 8)):
        part, m = torch.empty(40, cols, device=DEV), ck.columns(first, cols)
        assert emb.lib().emb_restore(40, cols, m.ref, emb.Mat(part).ref, None) == 0
        torch.cuda.synchronize()
        assert torch.equal(part, back[:, first:first + cols])
