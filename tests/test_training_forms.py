"""The 64-bit forms that the training operators are held to: their gradients are those of the formulas (autograd) and of differences."""
import pytest
import torch

import training_forms as tf


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def central(f, x, d):
    """df/dx along d by central differences."""
    h = 1e-5
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("T,E,n,residual", [(1, 1, 0, False), (1, 7, 2, True), (5, 12, 3, True), (9, 33, 8, False)])
def test_gradient_of_the_norm(T, E, n, residual):
    x, gamma, beta, dy = randn(1, T, E) * 2 + 0.5, 1 + 0.1 * randn(2, E), randn(3, E), randn(4, T, E)
    wg, bg = (randn(5, E, n), randn(6, n)) if n else (None, None)
    dl = randn(7, T, n) if n else None
    dres = randn(8, T, E) if residual else None
    leaves = [t.requires_grad_() for t in (x, gamma, beta) + ((wg, bg) if n else ())]

    def scalar(x, gamma, beta, wg=None, bg=None):
        y, _, _, logits = tf.norm(x, gamma, beta, 1e-3, wg, bg)
        s = (y * dy).sum()
        if n:
            s = s + (logits * dl).sum()
        return s + (x * dres).sum() if residual else s

    want = torch.autograd.grad(scalar(*leaves), leaves)
    leaves = [t.detach() for t in leaves]
    _, mean, rstd, _ = tf.norm(leaves[0], leaves[1], leaves[2], 1e-3)
    got = tf.norm_grad(dy, leaves[0], leaves[1], leaves[2], mean, rstd, dres, dl, leaves[3] if n else None)
    for g, w in zip(got, want):
        assert torch.allclose(g, w, rtol=1e-9, atol=1e-9)
    for i, leaf in enumerate(leaves):
        d = randn(20 + i, *leaf.shape)
        slope = central(lambda v: scalar(*(leaves[:i] + [v] + leaves[i + 1:])), leaf, d)
        assert torch.allclose((got[i] * d).sum(), slope, rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("T,n,padded", [(1, 2, False), (40, 2, True), (33, 5, False), (64, 8, True)])
def test_gradient_of_the_balance_loss(T, n, padded):
    l, alpha, w = randn(1, T, n), 0.5 + randn(2, n).abs(), torch.tensor([0.7, 1.3], dtype=torch.float64)
    valid = (randn(3, T) > -0.5) if padded else None
    keep = torch.ones(T, dtype=torch.bool) if valid is None else valid
    scalar = lambda v: (tf.balance_losses(v[keep], alpha, 0.3)[0] * w).sum()      # noqa: E731
    leaf = l.clone().requires_grad_()
    want, = torch.autograd.grad(scalar(leaf), leaf)
    losses, sums, counts, got = tf.balance(l, alpha, 0.3, w, valid)
    assert torch.allclose(got, want, rtol=1e-9, atol=1e-12) and int(counts.sum()) == int(keep.sum())
    d = randn(4, T, n)
    assert torch.allclose((got * d).sum(), central(scalar, l, d), rtol=1e-5, atol=1e-8)


def test_ties_go_to_the_lowest_index():
    l = torch.tensor([[1.0, 1.0, 0.0], [0.0, 2.0, 2.0], [3.0, 3.0, 3.0], [-1.0, 5.0, -1.0]], dtype=torch.float64)
    first, second = tf.ranks(l)
    assert first.tolist() == [0, 1, 0, 1] and second.tolist() == [1, 2, 1, 0]
    assert tf.others(l).tolist() == [[1, 0, 0], [1, 2, 1], [1, 0, 0], [1, 0, 1]]


@pytest.mark.parametrize("T,E,n", [(1, 1, 2), (20, 9, 3), (31, 16, 8)])
def test_gradient_of_the_combine(T, E, n):
    dy, src, l = randn(1, T, E), randn(2, T, E), randn(3, T, n)
    rows = torch.sort(tf.ranks(l)[0], stable=True).indices

    def scalar(src, l):
        gate = torch.softmax(l, 1).max(1).values
        y = torch.zeros_like(dy).index_copy(0, rows, gate[rows][:, None] * src)
        return (y * dy).sum()

    leaves = [src.clone().requires_grad_(), l.clone().requires_grad_()]
    want = torch.autograd.grad(scalar(*leaves), leaves)
    gate = torch.softmax(l, 1).max(1).values
    dsrc, dgate, dl = tf.combine_grad(dy, src, rows, gate, l)
    assert torch.allclose(dsrc, want[0]) and torch.allclose(dl, want[1][rows])
    d = randn(4, T, n) * 0.01
    assert torch.allclose((dl * d[rows]).sum(), central(lambda v: scalar(src, v), l, d), rtol=1e-5, atol=1e-8)
