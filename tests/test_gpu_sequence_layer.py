"""The sequence layer as a program runs it: one training step against a 64-bit
model of the same step, and the training example."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def test_one_training_step_against_autograd_in_64_bits():
    """Lookup, projection, recurrence and their backward against PyTorch's
    autograd on the CPU in 64 bits.  Rows, projection and their gradients are
    rounded to bf16 (2^-9 of a value each) and their checkpoints to 7 bits (at
    most 2^-7 of a group's largest, about 0.7% of a spread of values): gradients
    agree within 4% of their norm, outputs within 2%."""
    import torch
    import paper_2112_02752_amd as emb
    rng = torch.Generator().manual_seed(4)
    R, D, H, lens = 50, 40, 32, [7, 0, 30, 1, 66]
    offs = np.concatenate([[0], np.cumsum(lens)])
    n, M = int(offs[-1]), len(lens)
    W = torch.randn((R, D), generator=rng)
    weight = (torch.randn((D, 3 * H), generator=rng) * D ** -0.5).bfloat16()
    bias = torch.linspace(-1, 3, H)
    ids = torch.randint(0, R, (n,), generator=rng)
    pad = int(ids[3])
    dy = torch.randn((n, H), generator=rng).bfloat16()
    dh_last, h0 = torch.randn((M, H), generator=rng), torch.randn((M, H), generator=rng)

    # 64 bits
    Wd, wd, bd, hd = (v.double().requires_grad_() for v in (W, weight, bias, h0))
    rows = Wd[ids] * 1.5 * (ids != pad).double()[:, None]
    x, f, o = (rows @ wd).split(H, 1)
    a = torch.sigmoid(f + bd)
    ys, lasts = [], []
    for m in range(M):
        h = hd[m]
        for t in range(offs[m], offs[m + 1]):
            h = a[t] * h + (1 - a[t]) * x[t]
            ys.append(torch.sigmoid(o[t]) * h)
        lasts.append(h)
    y_w, last_w = torch.stack(ys), torch.stack(lasts)
    ((y_w * dy.double()).sum() + (last_w * dh_last.double()).sum()).backward()

    tables = emb.Tables(W.clone().cuda(), [0, R])
    layer = emb.SequenceLayer(tables, weight.cuda(), bias.cuda(), n, M, scale=1.5, pad_row=pad, opt="sgd", lr=1.0)
    batch = emb.Batch(torch.from_numpy(offs.astype(np.int32)).cuda(), ids.cuda(), M)
    y, last = torch.empty((n, H), dtype=torch.bfloat16, device="cuda"), torch.empty((M, H), device="cuda")
    dw, db = torch.empty((D, 3 * H), device="cuda"), torch.empty(H, device="cuda")
    dh0 = torch.empty((M, H), device="cuda")
    layer.forward(batch, y, last, h0=h0.cuda())
    layer.backward(batch, dy.cuda(), dw, db, dh_last=dh_last.cuda(), dh0=dh0)

    def off(got, want):
        return float((got.double().cpu() - want.detach()).norm() / want.detach().norm())

    assert off(y, y_w) <= 0.02 and off(last, last_w) <= 0.02
    assert off(dw, wd.grad) <= 0.04 and off(db, bd.grad) <= 0.04 and off(dh0, hd.grad) <= 0.04
    step = W.double() - tables.weights.double().cpu()
    assert off(step, Wd.grad) <= 0.04
    assert bool((step[pad] == 0).all())
    with pytest.raises(ValueError):
        layer.backward(batch, dy.cuda(), dw, db)       # once a forward


def test_training_example_learns_and_serves():
    """120 steps bring the loss below half of guessing among eight markers, and
    the states token by token are those of the whole sequences (fp32, up to 60
    steps of a few units in the last place each; bf16 projections of other
    shapes may round differently: 2^-7)."""
    spec = importlib.util.spec_from_file_location("sequence_training",
                                                  os.path.join(ROOT, "examples", "sequence_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    layer, head, losses, g = example.train(120, say=lambda *a: print(*a, flush=True))
    assert np.mean(losses[:5]) > 1.5
    assert np.mean(losses[-10:]) < 0.5 * np.log(8)
    off, right = example.serve(layer, head.detach(), g, say=lambda *a: print(*a, flush=True))
    assert off <= 2.0 ** -7 * 8 and right >= 0.6
