"""The mixture half of a block trained as a program would: norm with router, dispatch, experts, gated combine, balance loss; then the
gradients of all of it, from the output back to the rows that entered, against autograd in 64 bits."""
import pytest
import torch

import training_forms as tf

pytestmark = pytest.mark.gpu

EPS, STD = 1e-6, 0.3


@pytest.mark.parametrize("T,E,n,captured", [(197, 192, 2, False), (197, 192, 2, True), (2000, 97, 4, False)])
def test_mixture_half(sa, T, E, n, captured):
    """Experts here are diagonal maps E_i(v) = v * w_i, so that what the library computes is all that matters; the loss is
    <y, dy> + 0.7 IMP + 0.4 LOAD with the residual stream x in y."""
    g = torch.Generator(device="cuda").manual_seed(T + E)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
    x, gamma, beta, wg, bg, w, dy = r(T, E), 1 + 0.1 * r(E), 0.1 * r(E), r(E, n) / E ** 0.5, 0.1 * r(n), r(n, E), r(T, E)
    alpha, weights = torch.full((n,), 1.0 / n, device="cuda"), torch.tensor([0.7, 0.4], device="cuda")
    state = {}

    def step():
        h, mean, rstd, logits = sa.sa_layernorm(x, gamma, beta, EPS, wg=wg, bg=bg)
        perm, expert_of, counts, gate = sa.sa_moe_dispatch(logits)
        rows = perm.long()
        chosen = w.index_select(0, expert_of.index_select(0, rows).long())
        src = h.index_select(0, rows) * chosen
        y = torch.empty_like(x)
        if E % 4 == 0:
            sa.sa_combine_rows(src, y, rows=perm, gate=gate)
        dsrc, dgate, dlogits = sa.sa_combine_rows_backward(dy, src, rows=perm, gate=gate, logits=logits)
        losses, sums, counted, dlogits = sa.sa_moe_balance_loss_grad(logits, alpha, STD, weights, dlogits=dlogits, accumulate=True)
        dh = torch.empty_like(h).index_copy_(0, rows, dsrc * chosen)
        grads = sa.sa_layernorm_backward(dh, x, gamma, beta, EPS, mean=mean, rstd=rstd, dres=dy, dlogits=dlogits, wg=wg)
        state.update(y=y, counts=counts, counted=counted, losses=losses, grads=grads)

    step()
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        held = dict(state)
        for k in range(3):
            x.copy_(r(T, E))
            graph.replay()
            torch.cuda.synchronize()
            replayed = [t.clone() for t in (held["y"], held["losses"]) + held["grads"]]
            step()
            assert all(torch.equal(a, b) for a, b in zip(replayed, (state["y"], state["losses"]) + state["grads"]))
    assert torch.equal(state["counts"], state["counted"])

    leaves = [tf.f64(t).requires_grad_() for t in (x, gamma, beta, wg, bg)]
    h, _, _, logits = tf.norm(leaves[0], leaves[1], leaves[2], EPS, leaves[3], leaves[4])
    first, second = tf.ranks(logits.detach())
    top2 = logits.detach().gather(1, torch.stack((first, second), 1))
    assert float((top2[:, 0] - top2[:, 1]).min()) > 1e-5     # no routing hangs on a rounding
    gate = torch.softmax(logits, 1).gather(1, first[:, None])
    y = gate * h * tf.f64(w)[first]
    losses = tf.balance_losses(logits, tf.f64(alpha), float(torch.tensor(STD, dtype=torch.float32)))[0]
    want = torch.autograd.grad(((y + leaves[0]) * tf.f64(dy)).sum() + (losses * tf.f64(weights)).sum(), leaves)
    # rows of 192 normal numbers: every step is a sum of up to E products of size 1, off by E * U of its magnitudes; columns sum T of them
    assert bool(((tf.f64(state["losses"]) - losses.detach()).abs() <= 1e-5 * (1 + losses.detach())).all())
    if E % 4 == 0:
        assert bool(((tf.f64(state["y"]) - y.detach()).abs() <= 64 * tf.U * (1 + E ** 0.5) * (1 + y.detach().abs())).all())
    for got, ref in zip(state["grads"], want):
        scale = float(ref.abs().max())
        assert float((tf.f64(got) - ref).abs().max()) <= tf.U * (tf.D + 2 * T ** 0.5) * 4 * (1 + scale), float((tf.f64(got) - ref).abs().max())
