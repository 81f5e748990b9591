"""The balance loss with its gradient on the GPU, at logits that are not finite and with experts that are hardly ever chosen."""
import pytest
import torch

import training_forms as tf

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


@pytest.mark.parametrize("T", [700, 5000])
@pytest.mark.parametrize("n", [2, 3, 8])
@pytest.mark.parametrize("std", [0.08, 0.13, 0.2, 0.5])
def test_load_of_experts_that_are_hardly_ever_chosen(sa, T, n, std):
    """One expert is far ahead for every token, so that the others' LOAD is made of distant tails: right relative to itself."""
    l, alpha = randn(T + n, T, n), torch.full((n,), 1.0 / n, device="cuda")
    l[:, 0] += 6.0 + l[:, 1:].abs().sum(1)
    std = float(torch.tensor(std, dtype=torch.float32))
    got = sa.sa_moe_balance_loss_grad(l, alpha, std, torch.ones(2, device="cuda"))[1][1, 1:].double().cpu()
    d = tf.f64(l)
    p = torch.softmax(d, 1)
    z = ((p - p.gather(1, tf.others(d))) / std)[:, 1:]
    q = 0.5 * torch.erfc(-z / 2.0 ** 0.5)
    want = q.sum(0) / n
    # As in training_forms.balance_off: of a probability its exponent's rounding, exp's own 2 units and a few more; of z three roundings.  That
    # counts by the density over the tail, which is less than (|z| + sqrt(z^2 + 4)) / 2.  The tail itself: its exponent z^2 / 2 is two
    # roundings of its size, as much again for the constant and the instruction, and 12 units for the rest.
    gap = d[:, :1] - d
    e_p = p * tf.U * (gap + (p * gap).sum(1, keepdim=True) + n + 10)
    e_z = (e_p[:, 1:] + e_p[:, :1]) / std + 3 * tf.U * z.abs()
    rel = e_z * (z.abs() + torch.sqrt(z * z + 4)) / 2 + (2 * z * z + 12) * tf.U
    bound = 1.01 * (q * rel).sum(0) / n + tf.U * want + 2.0 ** -126      # what is below the smallest normal number is 0
    err = (got - want).abs()
    assert bool((err <= bound).all()), (err / want, bound / want)


@pytest.mark.parametrize("E", [768, 4099, (1 << 18) + 5, (1 << 24) + 3])
@pytest.mark.parametrize("yt,st", [(torch.float32, torch.float32), (torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16)], ids=str)
def test_gate_of_long_rows_of_one_sign(sa, yt, st, E):
    """A dot product whose terms are all alike: what is added is rounded the same way again and again where it is small against the sum.
    Here 8 terms at a time are added up in fp32, those sums in fp64, and the up to 64 lanes' in fp32."""
    dy, src = torch.full((3, E), 0.3, device="cuda").to(yt), torch.full((3, E), 0.7, device="cuda").to(st)
    dgate = sa.sa_combine_rows_backward(dy, src, want_dsrc=False)[1]
    want = E * float(dy[0, 0]) * float(src[0, 0])
    assert bool(((dgate.double() - want).abs() <= (8 + 1 + 6) * tf.U * want).all()), (dgate.double() / want - 1) / tf.U
