"""Linear attention with a decay for each head, single tokens, and a decoder's run: prompts, then tokens, over one cache of states."""
import pytest
import torch

from decay_forms import HALF_STEP, check, forward, reference, sequences

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,H,Hk,d,dv", [(1, 3, 3, 64, 64), (5, 4, 2, 32, 24), (7, 12, 2, 128, 128), (3, 5, 1, 8, 8), (33, 2, 2, 128, 32), (2, 9, 3, 72, 104),
                                        (300, 1, 1, 64, 40)])
def test_step(sa, B, H, Hk, d, dv, dtype):
    s = sequences([1] * B, H, Hk, d, dv, dtype, seed=B + d, device="cuda")
    scale, places = d ** -0.5, B + 3
    slots = torch.randperm(places, generator=torch.Generator().manual_seed(B))[:B].to(torch.int32).cuda()
    cache = torch.randn(places, Hk, d, dv, device="cuda")
    s["state_in"] = cache[slots.long()].clone()
    want = reference(s, scale, [1] * B)
    # the states have one rounding after a product in fp32 and a decay off by 2^-22: what check allows is for prompts, and no less
    elsewhere = torch.full_like(cache, 9.0)
    o, last = sa.sa_decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], scale, cache, slots=slots, state_out=elsewhere)
    check("out", o, want["out"], s, scale, dtype, [1] * B)
    check("state_out", last[slots.long()], want["state_out"], s, scale, dtype, [1] * B)
    others = [p for p in range(places) if p not in slots.tolist()]
    assert bool((elsewhere[others] == 9.0).all())
    before = cache.clone()
    o2, same = sa.sa_decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], scale, cache, slots=slots)       # in place
    assert same is cache and torch.equal(o, o2) and torch.equal(cache[slots.long()], elsewhere[slots.long()])
    assert torch.equal(cache[others], before[others])


def test_slots_that_are_none(sa):
    """A padded batch: rows whose slot is none see their own token only and leave no state."""
    B, H, d = 4, 2, 64
    s = sequences([1] * B, H, H, d, d, torch.float32, seed=1, device="cuda")
    cache = torch.randn(2, H, d, d, device="cuda")
    slots = torch.tensor([1, -1, 2, -2 ** 31], dtype=torch.int32, device="cuda")
    before = cache.clone()
    o, _ = sa.sa_decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], 0.5, cache, slots=slots)
    assert torch.equal(cache[0], before[0]) and not torch.equal(cache[1], before[1])
    own = 0.5 * (s["q"] * s["k"]).double().sum(-1, keepdim=True) * s["v"].double()
    size = 0.5 * (s["q"] * s["k"]).abs().sum(-1, keepdim=True) * s["v"].abs()
    assert bool(((o.double() - own).abs() <= 70 * 2.0 ** -24 * size)[1:].all())


def test_no_memory(sa):
    s = sequences([1, 1], 1, 1, 64, 64, torch.float32, seed=1, device="cuda")
    g = torch.tensor([-float("inf")], device="cuda")
    state = torch.randn(2, 1, 64, 64, device="cuda")
    sa.sa_decay_attention_step(s["q"], s["k"], s["v"], g, 1.0, state)
    assert torch.equal(state, s["k"][..., None] * s["v"][..., None, :])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hk,d,dv", [(4, 4, 64, 64), (6, 2, 96, 72)])
def test_prompts_then_tokens(sa, H, Hk, d, dv, dtype):
    """As a server has it: ragged prompts into a cache, a second part of each prompt, then tokens one by one, through graphs that are replayed; the last
    rows and states are those of the whole sequences."""
    lengths, more, steps, places = [70, 300, 1, 129], [5, 200, 64, 0], 3, 6
    whole = [a + b + steps for a, b in zip(lengths, more)]
    s = sequences(whole, H, Hk, d, dv, dtype, seed=H, device="cuda")
    s["state_in"].zero_()
    scale = d ** -0.5
    want = reference(s, scale, whole)
    first = s["offsets"].tolist()
    slots = torch.tensor([4, 1, 5, 0], dtype=torch.int32, device="cuda")
    cache = torch.zeros(places, Hk, d, dv, device="cuda")
    got = torch.zeros_like(s["dout"])
    for part in (0, 1):
        ranges = [(f + (a if part else 0), b if part else a) for f, a, b in zip(first, lengths, more)]
        rows = torch.cat([torch.arange(x, x + n) for x, n in ranges]).cuda()
        off = torch.tensor([0] + [n for _, n in ranges]).cumsum(0).to(torch.int32).cuda()
        q, k, v = (s[n][rows] for n in ("q", "k", "v"))
        o, _ = sa.sa_decay_attention(q, k, v, s["log_decay"], scale, offsets=off, state_in=cache, state_out=cache, slots=slots)
        got[rows] = o
    at = torch.tensor([f + a + b for f, a, b in zip(first, lengths, more)], device="cuda")
    q, k, v = (s[n][at].clone() for n in ("q", "k", "v"))
    out = torch.empty(len(whole), H, dv, dtype=dtype, device="cuda")
    saved = cache.clone()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sa.sa_decay_attention_step(q, k, v, s["log_decay"], scale, cache, slots=slots, out=out)
        cache.copy_(saved)
        with torch.cuda.graph(graph, stream=side):
            sa.sa_decay_attention_step(q, k, v, s["log_decay"], scale, cache, slots=slots, out=out)
    torch.cuda.current_stream().wait_stream(side)
    cache.copy_(saved)
    for t in range(steps):
        for to, n in ((q, "q"), (k, "k"), (v, "v")):
            to.copy_(s[n][at + t])
        graph.replay()
        torch.cuda.synchronize()
        got[at + t] = out
    check("out", got, want["out"], s, scale, dtype, whole)
    check("state_out", cache[slots.long()], want["state_out"], s, scale, dtype, whole)
    assert bool((cache[[2, 3]] == 0).all())


def test_token_by_token_is_the_definition(sa):
    """A short sequence as steps against the definition read literally."""
    s = sequences([9], 2, 1, 16, 8, torch.float32, seed=6, device="cuda")
    out, last = forward(s["q"].double(), s["k"].double(), s["v"].double(), s["log_decay"].double(), 0.25, s["state_in"][0].double())
    state = s["state_in"].clone()
    for t in range(9):
        o, _ = sa.sa_decay_attention_step(s["q"][t:t + 1], s["k"][t:t + 1], s["v"][t:t + 1], s["log_decay"], 0.25, state)
        assert (o[0].double() - out[t]).abs().max().item() <= 64 * HALF_STEP[torch.float32] * 40      # sums of 16 products below 40
    assert (state[0].double() - last).abs().max().item() <= 32 * HALF_STEP[torch.float32] * 16


def test_decays_of_one_layer(sa):
    """A row of a table of decays, layer by layer, begins where it begins."""
    H, d, n = 3, 64, 150
    s = sequences([n, n], H, H, d, d, torch.bfloat16, seed=5, device="cuda")
    table = s["log_decay"].repeat(4, 1)
    q, k, v, do = (s[name].view(2, n, H, d) for name in ("q", "k", "v", "dout"))
    for row in (1, 2, 3):
        g, own = table[row], s["log_decay"]
        for call in (lambda g: sa.sa_decay_attention(q, k, v, g, 0.1, want_state=True),
                     lambda g: sa.sa_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], g, 0.1, s["state_in"], state_out=torch.zeros_like(s["state_in"])),
                     lambda g: sa.sa_decay_attention_backward(do, q, k, v, g, 0.1, want_dstate=True)):
            assert all(torch.equal(a, b) for a, b in zip(call(g), call(own)))
