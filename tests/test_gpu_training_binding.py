"""What the binding of the training operators makes and refuses, where it takes a GPU to see it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,rows", [(64, 96), (1, 2), (500, 4000)])
def test_gradients_of_rows_that_nothing_selects_are_zeros(sa, T, rows):
    """Without an index the first T rows of src are combined; src may have more."""
    E = 32
    dy, src, gate = torch.ones(T, E, device="cuda"), torch.ones(rows, E, device="cuda"), torch.ones(T, device="cuda")
    nan = [torch.full((rows, E), float("nan"), device="cuda") for _ in range(8)]     # what memory holds that was in use before
    torch.cuda.synchronize()
    del nan
    dsrc, dgate, _ = sa.sa_combine_rows_backward(dy, src, max_rows=T, gate=gate)
    assert bool((dsrc[:T] == 1.0).all()) and bool((dsrc[T:] == 0.0).all()) and bool((dgate == E).all())
    keep = torch.full((rows, E), 5.0, device="cuda")         # a buffer that is given is left as it is there
    sa.sa_combine_rows_backward(dy, src, max_rows=T, gate=gate, dsrc=keep)
    assert bool((keep[:T] == 1.0).all()) and bool((keep[T:] == 5.0).all())


@pytest.mark.parametrize("T,rows,max_rows", [(96, 64, 64), (96, 96, 64), (96, 128, 96), (96, 128, 30)])
def test_zeros_of_either_side_that_is_longer(sa, T, rows, max_rows):
    """dsrc has the rows of src, dgate and dlogits those of dy: whichever is longer than max_rows ends in zeros."""
    E, n = 32, 2
    dy, src, gate = torch.ones(T, E, device="cuda"), torch.ones(rows, E, device="cuda"), torch.ones(T, device="cuda")
    logits = torch.tensor([[1.0, 0.0]], device="cuda").repeat(T, 1)
    nan = [torch.full(shape, float("nan"), device="cuda") for shape in ((rows, E), (T,), (T, n)) for _ in range(8)]
    torch.cuda.synchronize()
    del nan
    dsrc, dgate, dlogits = sa.sa_combine_rows_backward(dy, src, max_rows=max_rows, gate=gate, logits=logits)
    for t in (dsrc, dgate, dlogits):
        assert bool((t[:max_rows] != 0.0).all()) and bool(t[:max_rows].isfinite().all()) and bool((t[max_rows:] == 0.0).all())
