"""The gradient of linear attention with a decay for each head: against 64 bits, against differences, and as a training step calls it."""
import pytest
import torch

from decay_forms import check, reference, sequences

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
LENGTHS = [[1], [16, 1, 17, 0, 15], [63, 64, 65], [700, 3, 90]]
HEADS = [(3, 3, 64, 64), (4, 2, 32, 24), (2, 1, 8, 128), (6, 2, 96, 72), (2, 2, 128, 128), (3, 1, 128, 8), (4, 1, 64, 104)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hk,d,dv", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("state", [False, True])
def test_ragged(sa, lengths, H, Hk, d, dv, dtype, state):
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=sum(lengths) + H + d, device="cuda", offset=2, behind=3)
    scale = d ** -0.5
    outs = {n: torch.full_like(s[n[1:]], 7.0) for n in ("dq", "dk", "dv")}
    got = sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], scale, offsets=s["offsets"],
                                         state_in=s["state_in"] if state else None, dstate_out=s["dstate_out"] if state else None, want_dstate=state, **outs)
    want = reference(s, scale, lengths, state=state, gradients=True)
    for name, g in zip(("dq", "dk", "dv", "dstate_in"), got):
        if g is not None:
            check(name, g, want[name], s, scale, dtype, lengths, state)
        if name != "dstate_in":
            assert bool((g[:2] == 7.0).all()) and bool((g[-3:] == 7.0).all())
    assert (got[3] is None) == (not state)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N,H,Hk,d,dv", [(2, 197, 3, 3, 64, 64), (40, 130, 8, 8, 32, 64), (1, 1500, 2, 1, 128, 72), (2, 600, 2, 2, 64, 128)])
def test_of_one_length(sa, B, N, H, Hk, d, dv, dtype):
    s = sequences([N] * B, H, Hk, d, dv, dtype, seed=N, device="cuda")
    q, k, v, do = (s[n].view(B, N, *s[n].shape[1:]) for n in ("q", "k", "v", "dout"))
    got = sa.sa_decay_attention_backward(do, q, k, v, s["log_decay"], 0.3)
    want = reference(s, 0.3, [N] * B, state=False, gradients=True)
    for name, g in zip(("dq", "dk", "dv"), got):
        check(name, g.reshape(want[name].shape), want[name], s, 0.3, dtype, [N] * B, False)


@pytest.mark.parametrize("decay", [0.0, -0.05, -2.0, -float("inf")])
def test_decays(sa, decay):
    lengths = [130, 64, 900]
    s = sequences(lengths, 2, 1, 64, 32, torch.float32, seed=3, device="cuda")
    s["log_decay"].fill_(decay)
    got = sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.2, offsets=s["offsets"], state_in=s["state_in"],
                                         dstate_out=s["dstate_out"], want_dstate=True)
    t = dict(s, log_decay=s["log_decay"].clamp(min=-800.0))
    want = reference(t, 0.2, lengths, gradients=True)
    for name, g in zip(("dq", "dk", "dv", "dstate_in"), got):
        check(name, g, want[name], t, 0.2, torch.float32, lengths)


@pytest.mark.parametrize("name", ["q", "k", "v", "state_in"])
def test_against_differences(sa, name):
    """The loss is linear in each of q, k, v and the state before: half the difference of its values at x + y and x - y is <gradient, y>, whatever y is."""
    lengths = [70, 300]
    s = sequences(lengths, 4, 2, 64, 40, torch.float32, seed=12, device="cuda")
    g = dict(zip(("q", "k", "v", "state_in"), sa.sa_decay_attention_backward(
        s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=s["state_in"], dstate_out=s["dstate_out"], want_dstate=True)))
    y = torch.randn(s[name].shape, generator=torch.Generator().manual_seed(1)).cuda()

    def loss(x):
        t = dict(s, **{name: x})
        o, last = sa.sa_decay_attention(t["q"], t["k"], t["v"], t["log_decay"], 0.1, offsets=s["offsets"], state_in=t["state_in"], want_state=True)
        terms = torch.cat([(o.double() * s["dout"].double()).flatten(), (last.double() * s["dstate_out"].double()).flatten()])
        return terms.sum(), terms.abs().sum()

    (up, size), (down, size2) = loss(s[name] + y), loss(s[name] - y)
    slope = (g[name].double() * y.double()).sum()
    # each value is a sum of fp32 results off by 2^-16 of the magnitudes that went into them (300 tokens and two widths of fp32 sums), which are
    # at most 40 times what is left of them; x + y is rounded once more
    assert abs((up - down).item() / 2 - slope.item()) <= 2.0 ** -16 * 40 * (size + size2).item() / (300 ** 0.5)


@pytest.mark.parametrize("dtype", TYPES)
def test_columns_of_a_wider_matrix(sa, dtype):
    B, N, H, Hk, d, dv = 2, 150, 4, 2, 64, 72
    s = sequences([N] * B, H, Hk, d, dv, dtype, seed=3, device="cuda")
    parts, heads, widths = [H * d, Hk * d, Hk * dv], (H, Hk, Hk), (d, d, dv)
    fused = torch.cat([s[n].reshape(B * N, -1) for n in ("q", "k", "v")], 1)
    q, k, v = (x.view(B, N, h, w) for x, h, w in zip(fused.split(parts, 1), heads, widths))
    do = s["dout"].view(B, N, H, dv)
    grad = torch.empty_like(fused)
    dq, dk, dv_ = (x.view(B, N, h, w) for x, h, w in zip(grad.split(parts, 1), heads, widths))
    sa.sa_decay_attention_backward(do, q, k, v, s["log_decay"], 0.3, dq=dq, dk=dk, dv=dv_)
    dense = sa.sa_decay_attention_backward(do, *(s[n].view(B, N, -1, s[n].shape[-1]) for n in ("q", "k", "v")), s["log_decay"], 0.3)
    for a, b in zip((dq, dk, dv_), dense):
        assert torch.equal(a, b)


def test_no_tokens(sa):
    e = torch.empty(0, 2, 64, device="cuda")
    g = torch.tensor([-0.5, 0.0], device="cuda")
    d = torch.randn(3, 2, 64, 64, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    got = sa.sa_decay_attention_backward(e, e, e, e, g, 1.0, offsets=off, dstate_out=d, want_dstate=True)
    assert torch.equal(got[3], d) and got[0].shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_training_step_in_a_graph(sa, dtype):
    """Forward and backward, captured once and replayed on new values with other work between: the same bits as without a graph, each time."""
    lengths, H, Hk, d, dv = [900, 40, 300], 4, 2, 64, 64
    steps = [sequences(lengths, H, Hk, d, dv, dtype, seed=i, device="cuda") for i in range(3)]
    s = {k: v.clone() for k, v in steps[0].items()}
    T = s["q"].shape[0]
    ws = [torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in (
        sa.sa_decay_attention_workspace_bytes(T, 3, H, Hk, d, dv, True), sa.sa_decay_attention_backward_workspace_bytes(T, 3, H, Hk, d, dv, True))]
    o, last = torch.empty_like(s["dout"]), torch.empty_like(s["state_in"])
    grads = dict(dq=torch.empty_like(s["q"]), dk=torch.empty_like(s["k"]), dv=torch.empty_like(s["v"]), dstate_in=torch.empty_like(last))

    def step(s):
        sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=s["state_in"], out=o, state_out=last, workspace=ws[0])
        sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=s["state_in"],
                                       dstate_out=s["dstate_out"], workspace=ws[1], **grads)
        return [o, last] + list(grads.values())

    eager = [[t.clone() for t in step(x)] for x in steps]
    again = [t.clone() for t in step(steps[1])]
    assert all(torch.equal(a, b) for a, b in zip(eager[1], again))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(s)
        with torch.cuda.graph(graph, stream=side):
            step(s)
    torch.cuda.current_stream().wait_stream(side)
    for i in (0, 1, 2, 1):
        for n, t in s.items():
            t.copy_(steps[i][n])
        for t in [o, last] + list(grads.values()):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([o, last] + list(grads.values()), eager[i])), i
        torch.randn(1000, 1000, device="cuda").sum()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [130, 1400])
def test_what_is_not_finite_stays_in_its_head(sa, N, dtype):
    """A NaN in dout reaches gradients of its own sequence and head, of k and v up to 63 tokens behind it, of q from 63 before it on."""
    s = sequences([N, N], 2, 2, 64, 64, dtype, seed=4, device="cuda")
    call = lambda s: sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"])      # noqa: E731
    clean = call(s)
    at = N // 2
    s["dout"][at, 0, 5] = float("nan")
    for name, a, b in zip("qkv", call(s), clean):
        assert torch.equal(a[N:], b[N:]) and torch.equal(a[:, 1], b[:, 1]), name
        if name == "q":
            assert torch.equal(a[:at - 63], b[:at - 63])
        else:
            assert torch.equal(a[at + 64:], b[at + 64:])
        assert not a[at, 0].isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hk", [(2, 2), (4, 2)])
def test_the_recurrence_token_by_token(sa, H, Hk, dtype):
    """R_t = scale q_t dout_t^T + e^g R_{t+1}, of the last token scale q_t dout_t^T + dstate_out: read literally, from the last token to the first, through
    one pass of a chunk and a half; an empty sequence hands dstate_out on."""
    lengths, d, dv, scale = [70, 0, 1], 32, 40, 0.3
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=21, device="cuda")
    s["log_decay"] = torch.tensor([-0.7, -0.05], device="cuda")
    got = sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], scale, offsets=s["offsets"], state_in=s["state_in"],
                                         dstate_out=s["dstate_out"], want_dstate=True)
    fade = s["log_decay"].double().exp()[:, None, None]
    q, do = (s[n].double().view(-1, Hk, H // Hk, s[n].shape[-1]) for n in ("q", "dout"))
    k, v = s["k"].double(), s["v"].double()
    dk, dv_rows, dstate = torch.empty_like(k), torch.empty_like(v), s["dstate_out"].double().clone()
    first = s["offsets"].tolist()
    for b, n in enumerate(lengths):
        for t in reversed(range(first[b], first[b] + n)):
            behind = dstate[b] if t == first[b] + n - 1 else fade * dstate[b]
            dstate[b] = behind + scale * (q[t].unsqueeze(-1) * do[t].unsqueeze(-2)).sum(1)
            dk[t] = (dstate[b] * v[t].unsqueeze(-2)).sum(-1)
            dv_rows[t] = (dstate[b] * k[t].unsqueeze(-1)).sum(-2)
        if n:
            dstate[b] *= fade
    for name, g, want in zip(("dk", "dv", "dstate_in"), got[1:], (dk, dv_rows, dstate)):
        check(name, g, want, s, scale, dtype, lengths)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hk,d,dv", [(3, 3, 64, 64), (6, 2, 96, 72), (2, 1, 40, 128)])
@pytest.mark.parametrize("state", [False, True])
def test_short_sequences_among_long_ones(sa, H, Hk, d, dv, dtype, state):
    """Most sequences of one segment (their mean is below 256), which take no state through the workspace."""
    lengths = [0, 3, 900, 0, 40, 70, 1, 300, 5, 9, 257, 256, 0]
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=H + d, device="cuda", offset=2, behind=3)
    ws = torch.full((sa.sa_decay_attention_backward_workspace_bytes(s["q"].shape[0], len(lengths), H, Hk, d, dv, True) // 4,), float("nan"), device="cuda")
    outs = {n: torch.full_like(s[n[1:]], 7.0) for n in ("dq", "dk", "dv")}
    got = sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.2, offsets=s["offsets"], workspace=ws, **outs,
                                         state_in=s["state_in"] if state else None, dstate_out=s["dstate_out"] if state else None, want_dstate=state)
    want = reference(s, 0.2, lengths, state=state, gradients=True)
    for name, g in zip(("dq", "dk", "dv", "dstate_in"), got):
        if g is not None:
            check(name, g, want[name], s, 0.2, dtype, lengths, state)
        if name != "dstate_in":
            assert bool((g[:2] == 7.0).all()) and bool((g[-3:] == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [197, 1400])
@pytest.mark.parametrize("H,Hk,d,dv", [(2, 2, 64, 64), (4, 2, 96, 72), (2, 2, 128, 128)])
def test_gradients_of_what_does_not_see_it_stay_as_they_are(sa, N, H, Hk, d, dv, dtype):
    """What is not finite in a token reaches dq of later tokens alone, dk and dv of earlier ones alone: all others have the same bits."""
    s = sequences([N, 30], H, Hk, d, dv, dtype, seed=4, device="cuda")
    call = lambda s: sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], want_dstate=True)      # noqa: E731
    clean = call(s)
    none = slice(0, 0)
    for at in (0, 70, N - 1):
        on, up, own = slice(at, N), slice(0, at + 1), slice(at, at + 1)
        #                 rows of dq, dk and dv that see the token (dq does not depend on q, dk not on k, dv not on v; the token's own dq on its dout)
        for name, sees in (("dout", (own, up, up)), ("q", (none, up, up)), ("k", (on, none, own)), ("v", (on, own, none))):
            bad = dict(s, **{name: s[name].clone()})
            bad[name][at, -1, 3] = float("nan")
            got = call(bad)
            for g, c, rows, label in zip(got, clean, sees, ("dq", "dk", "dv")):
                heads = slice(H - 1, H) if name in ("dout", "q") and label == "dq" else slice((Hk - 1) * (g.shape[1] // Hk), g.shape[1])
                rest = g.clone()
                rest[rows, heads] = c[rows, heads]
                assert torch.equal(rest, c), (name, at, label)
                assert rows == none or not g[rows, heads].isfinite().all(), (name, at, label)
            if name in ("k", "v"):
                assert torch.equal(got[3], clean[3])
            else:
                assert torch.equal(got[3][:, :Hk - 1], clean[3][:, :Hk - 1]) and torch.equal(got[3][1:], clean[3][1:]) and got[3][0, -1].isnan().any()
