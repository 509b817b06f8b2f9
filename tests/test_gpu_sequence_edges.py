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
