"""What the binding of the operators over sequences refuses by itself, without a
GPU: arguments whose extent or type the C ABI cannot see."""
import pytest

import paper_2112_02752_amd as emb


def _tables(rows=10, dim=16):
    import torch
    return emb.Tables(torch.zeros(rows, dim), [0, rows])


@pytest.mark.parametrize("opt,shape", [("adagrad", (9,)), ("adagrad", (10, 16)), ("adagrad", (10, 2)), ("adagrad", ()),
                                       ("adagrad_ew", (10,)), ("adagrad_ew", (10, 15)), ("adagrad_ew", (9, 16)),
                                       ("adagrad_ew", (16, 10)), ("adagrad_ew", (159,))])
def test_accumulators_of_another_extent(opt, shape):
    import torch
    with pytest.raises(ValueError, match="accumulators"):
        emb.TokenLayer(_tables(), opt=opt, state=torch.zeros(shape))
    with pytest.raises(ValueError, match="accumulators"):
        emb.SequenceLayer(_tables(), torch.zeros((16, 96), dtype=torch.bfloat16), None, 0, 1, opt=opt,
                          state=torch.zeros(shape))


@pytest.mark.parametrize("opt,shape", [("adagrad", (10,)), ("adagrad_ew", (10, 16))])
def test_accumulators_of_another_kind(opt, shape):
    import torch
    for t in (torch.float64, torch.bfloat16, torch.int32):
        with pytest.raises(ValueError, match="accumulators"):
            emb.TokenLayer(_tables(), opt=opt, state=torch.zeros(shape, dtype=t))
    with pytest.raises(ValueError, match="accumulators"):
        emb.TokenLayer(_tables(), opt=opt, state=torch.zeros((shape[0], 32))[:, :shape[1]] if len(shape) > 1
                       else torch.zeros(20)[::2])
    with pytest.raises(ValueError, match="GPU"):
        emb.TokenLayer(_tables(), opt=opt, state=torch.zeros(shape))


def test_accumulators_of_a_single_call():
    import torch

    class Stub(emb.Mat):
        """A matrix without a GPU: the checks before any address is taken."""

        def __init__(self, rows, cols):
            self.tensor, self.exps, self.rows, self.cols = torch.zeros(rows, cols), None, rows, cols
            self._at = self.tensor.data_ptr()
            self._c = None

    batch = emb.Batch(torch.tensor([0, 3], dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 1)
    for opt, shape in (("adagrad", (9,)), ("adagrad_ew", (10,))):
        with pytest.raises(ValueError, match="accumulators"):
            emb.token_grad(_tables(), batch, Stub(3, 16), None, opt=opt, lr=0.1, state=torch.zeros(shape))


def test_no_accumulators_are_needed_without_adagrad():
    emb.TokenLayer(_tables(), opt="sgd")
    emb.TokenLayer(_tables())
    emb.TokenLayer(_tables(), opt="adagrad")      # looks up; an update asks for them


def test_a_layer_that_only_looks_up_has_no_backward_to_check():
    with pytest.raises(ValueError, match="only looks up"):
        emb.TokenLayer(_tables()).check()


def test_a_recurrence_off_the_gpu():
    with pytest.raises(ValueError, match="GPU"):
        emb.Recurrence(100, 1, 16, device="cpu")
