"""The balance loss with its gradient on the GPU, at logits that are not finite."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("n", [2, 3, 8])
@pytest.mark.parametrize("T", [1, 300, 5000])
@pytest.mark.parametrize("expert", [0, 1])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_logit_that_is_not_finite_shows_in_the_losses(sa, T, n, expert, value):
    """An overflow in the router: a softmax with an infinite logit has no value, and neither has a sum of it."""
    l, alpha, w = randn(1, T, n), torch.full((n,), 1.0 / n, device="cuda"), torch.ones(2, device="cuda")
    l[T // 2] = 1.0
    l[T // 2, expert] = value
    losses, sums, _, dl = sa.sa_moe_balance_loss_grad(l, alpha, 0.3, w)
    assert bool(losses.isnan().all()) and bool(sums.isnan().all()) and bool(dl.isnan().all())
    assert bool(sa.sa_moe_balance_loss(l, alpha, 0.3)[0].isnan().all())          # the value's own entry point says the same
    valid = torch.ones(T, dtype=torch.bool, device="cuda")
    valid[T // 2] = False                                    # of a padded token nothing is seen
    losses, sums, _, dl = sa.sa_moe_balance_loss_grad(l, alpha, 0.3, w, valid=valid)
    assert bool(losses.isfinite().all()) and bool(sums.isfinite().all()) and bool(dl.isfinite().all())
