"""One norm used by several threads, each with its own seed and rows: calls without a weight gradient need no order, so
each has its own mask.  Masks are read off whole numbers, exactly."""
import threading

import numpy as np
import pytest

from .block_plain import DEV, host, keep_scale, kept

pytestmark = pytest.mark.gpu

N, D, DROP = 40, 72, 0.5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _mask(seed, first_row):
    return kept(N, D, DROP, seed, first_row) * keep_scale(DROP)


class _Between:
    """The library, but what `then` does comes between a call's arguments and the call itself, once."""

    def __init__(self, real, name, then):
        self._real, self._name, self._then = real, name, then

    def __getattr__(self, name):
        fn = getattr(self._real, name)
        if name != self._name or self._then is None:
            return fn

        def call(*args):
            then, self._then = self._then, None
            other = threading.Thread(target=then)
            other.start()
            other.join()
            return fn(*args)
        return call


@pytest.mark.parametrize("way", ["forward", "backward"])
def test_a_call_between_anothers_arguments_and_itself(way, monkeypatch):
    import torch
    import paper_2112_02752_amd as emb
    from paper_2112_02752_amd import block
    norm = emb.Norm(torch.ones(D, device=DEV), drop=DROP)
    one, zero = torch.ones((N, D), device=DEV), torch.zeros((N, D), device=DEV)
    outs = [torch.full((N, D), 7.0, device=DEV) for _ in range(2)]
    calls = [(11, 0), (12, 1000)]

    def run(i):
        seed, row = calls[i]
        if way == "forward":
            norm.forward(one, torch.empty_like(one), total=outs[i], seed=seed, first_row=row)
        else:                   # (dy of zeros: the branch's gradient is what arrives, dropped)
            norm.backward(one, zero, branch=outs[i], arriving=one, seed=seed, first_row=row)

    real = block.lib()
    between = _Between(real, "emb_norm_fwd" if way == "forward" else "emb_norm_bwd", lambda: run(1))
    monkeypatch.setattr(block, "lib", lambda: between)
    run(0)
    torch.cuda.synchronize()
    for out, (seed, row) in zip(outs, calls):
        assert np.array_equal(host(out), _mask(seed, row)), (seed, row)


def test_threads_with_their_own_seeds():
    import torch
    import paper_2112_02752_amd as emb
    norm = emb.Norm(torch.ones(D, device=DEV), drop=DROP)
    one = torch.ones((N, D), device=DEV)
    outs = [[torch.full((N, D), 7.0, device=DEV) for _ in range(50)] for _ in range(4)]
    torch.cuda.synchronize()
    go = threading.Barrier(4)

    def run(i):
        y = torch.empty_like(one)
        go.wait()
        for k, out in enumerate(outs[i]):
            norm.forward(one, y, total=out, seed=100 * i + k, first_row=i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i, of in enumerate(outs):
        for k, out in enumerate(of):
            assert np.array_equal(host(out), _mask(100 * i + k, i)), (i, k)
