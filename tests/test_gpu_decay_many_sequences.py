"""Linear attention with a decay for each head over ragged batches of more sequences than a wavefront has lanes: a workgroup finds the sequence of its segment in
several rounds, 64 sequences at a time."""
import pytest
import torch

from decay_forms import check, reference, sequences

pytestmark = pytest.mark.gpu


def lengths_of(B, T, seed):
    """B lengths with T tokens in all: runs of empty sequences at both ends and between, many of one token, a few long ones."""
    g = torch.Generator().manual_seed(seed)
    size = torch.rand(B, generator=g) ** 6
    size[torch.rand(B, generator=g) < 0.3] = 0.0
    size[:3] = size[-2:] = 0.0
    size[B // 2:B // 2 + min(70, B // 4)] = 0.0
    size[5] = 1.0
    n = (T * size / size.sum()).int().tolist()
    n[5] += T - sum(n)
    return n


# tokens: one pass, segments of 256 and longer ones; and, without states, 64 queries to a workgroup
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T", [(64, 200), (65, 200), (65, 3000), (128, 3000), (129, 500), (129, 9000), (700, 250), (700, 6000)])
@pytest.mark.parametrize("state", [False, True])
def test_prompts(sa, B, T, state, dtype):
    lengths, H, Hk, d, dv = lengths_of(B, T, B + T), 2, 1, 32, 40
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=B, device="cuda", offset=1, behind=2)
    o, last = sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.2, offsets=s["offsets"], state_in=s["state_in"] if state else None,
                                    want_state=state, out=torch.full_like(s["dout"], 7.0))
    want = reference(s, 0.2, lengths, state=state)
    check("out", o, want["out"], s, 0.2, dtype, lengths, state)
    assert bool((o[:1] == 7.0).all()) and bool((o[-2:] == 7.0).all())
    if state:
        check("state_out", last, want["state_out"], s, 0.2, dtype, lengths)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("B,T", [(64, 200), (65, 3000), (129, 500), (300, 9000)])
@pytest.mark.parametrize("state", [False, True])
def test_gradients(sa, B, T, state, dtype):
    lengths, H, Hk, d, dv = lengths_of(B, T, B + T), 2, 1, 32, 40
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=B, device="cuda", offset=1, behind=2)
    outs = {n: torch.full_like(s[n[1:]], 7.0) for n in ("dq", "dk", "dv")}
    got = sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.2, offsets=s["offsets"], **outs,
                                         state_in=s["state_in"] if state else None, dstate_out=s["dstate_out"] if state else None, want_dstate=state)
    want = reference(s, 0.2, lengths, state=state, gradients=True)
    for name, g in zip(("dq", "dk", "dv", "dstate_in"), got):
        if g is not None:
            check(name, g, want[name], s, 0.2, dtype, lengths, state)
        if name != "dstate_in":
            assert bool((g[:1] == 7.0).all()) and bool((g[-2:] == 7.0).all())


@pytest.mark.parametrize("B,T", [(4096, 4096), (4097, 30000), (9000, 2000)])
def test_thousands(sa, B, T):
    """The longest sequences, and some at the borders of rounds, against the definition; empty ones hand their states on."""
    lengths, H, d = lengths_of(B, T, B), 2, 16
    s = sequences(lengths, H, H, d, d, torch.bfloat16, seed=B, device="cuda")
    o, last = sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.3, offsets=s["offsets"], state_in=s["state_in"], want_state=True)
    at = s["offsets"].tolist()
    for b in sorted(range(B), key=lambda b: -lengths[b])[:40:3] + [0, 63, 64, 65, 127, 128, B // 2, B - 3, B - 1]:
        one = {n: t[at[b]:at[b + 1]] for n, t in s.items() if n in ("q", "k", "v", "dout")}
        one.update(log_decay=s["log_decay"], state_in=s["state_in"][b:b + 1], offsets=torch.tensor([0, lengths[b]], dtype=torch.int32))
        want = reference(one, 0.3, [lengths[b]])
        if lengths[b]:
            check("out", o[at[b]:at[b + 1]], want["out"], one, 0.3, torch.bfloat16, [lengths[b]])
        check("state_out", last[b:b + 1], want["state_out"], one, 0.3, torch.bfloat16, [lengths[b]])
    empty = [b for b in range(B) if not lengths[b]]
    assert torch.equal(last[empty], s["state_in"][empty])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_two_streams_and_a_graph(sa, dtype):
    """Short sequences among long ones: two calls at once on streams of their own, with a workspace each, and a captured step that is replayed on other values:
    the bits of calls by themselves."""
    B, T, H, d = 80, 4000, 2, 64
    lengths = lengths_of(B, T, 3)
    sets = [sequences(lengths, H, H, d, d, dtype, seed=i, device="cuda") for i in range(3)]

    def step(s, buffers):
        o, last, grads, ws = buffers
        sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=s["state_in"], out=o, state_out=last, workspace=ws[0])
        sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=s["state_in"],
                                       dstate_out=s["dstate_out"], workspace=ws[1], **grads)
        return [o, last] + list(grads.values())

    def buffers():
        s = sets[0]
        ws = [torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in (
            sa.sa_decay_attention_workspace_bytes(T, B, H, H, d, d, True), sa.sa_decay_attention_backward_workspace_bytes(T, B, H, H, d, d, True))]
        return (torch.zeros_like(s["dout"]), torch.empty_like(s["state_in"]),
                dict(dq=torch.zeros_like(s["q"]), dk=torch.zeros_like(s["k"]), dv=torch.zeros_like(s["v"]), dstate_in=torch.empty_like(s["state_in"])), ws)

    alone = [[t.clone() for t in step(s, buffers())] for s in sets]
    streams, own = [torch.cuda.Stream() for _ in range(2)], [buffers() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, s, b in zip(streams, sets, own):
            with torch.cuda.stream(stream):
                got = step(s, b)
    torch.cuda.synchronize()
    for want, (o, last, grads, _) in zip(alone, own):
        assert all(torch.equal(a, b) for a, b in zip(want, [o, last] + list(grads.values())))
    s, b, graph = {n: t.clone() for n, t in sets[0].items()}, own[0], torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=streams[0]):
        got = step(s, b)
    for i in (2, 0, 1, 2):
        for n, t in s.items():
            t.copy_(sets[i][n])
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, alone[i])), i
        torch.randn(1000, 1000, device="cuda").sum()
