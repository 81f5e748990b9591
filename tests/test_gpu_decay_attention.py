"""Linear attention with a decay for each head on the GPU: prompts against the definition in 64 bits, sequence by sequence."""
import pytest
import torch

from decay_forms import allowed, check, reference, sequences

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def run(sa, s, scale, state=True, **kw):
    out = torch.full_like(s["dout"], 7.0)
    o, last = sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], scale, offsets=s["offsets"], state_in=s["state_in"] if state else None,
                                    want_state=state, out=out, **kw)
    return o, last


# one token, borders of a chunk and of a tile, several segments, nothing at all; widths of every kernel and odd ones
LENGTHS = [[1], [16, 1, 17, 0, 15], [63, 64, 65], [127, 0, 129, 200], [700, 3, 90, 513]]
HEADS = [(3, 3, 64, 64), (4, 2, 32, 24), (2, 1, 8, 128), (6, 2, 96, 72), (2, 2, 128, 128), (5, 5, 72, 40), (3, 1, 128, 8)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hk,d,dv", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("state", [False, True])
def test_prompts_side_by_side(sa, lengths, H, Hk, d, dv, dtype, state):
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=sum(lengths) + H + d, device="cuda", offset=3, behind=2)
    scale = d ** -0.5
    o, last = run(sa, s, scale, state)
    want = reference(s, scale, lengths, state=state)
    check("out", o, want["out"], s, scale, dtype, lengths, state)
    if state:
        check("state_out", last, want["state_out"], s, scale, dtype, lengths)
    assert bool((o[:3] == 7.0).all()) and bool((o[-2:] == 7.0).all())        # rows that no sequence has


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N,H,Hk,d,dv", [
    (2, 197, 3, 3, 64, 64), (70, 130, 8, 8, 64, 64), (1, 1500, 2, 2, 128, 72), (3, 1030, 4, 2, 40, 64), (2, 64, 2, 1, 96, 96), (600, 1, 1, 1, 8, 8),
    (1, 2300, 1, 1, 64, 104)])
@pytest.mark.parametrize("state", [False, True])
def test_prompts_of_one_length(sa, B, N, H, Hk, d, dv, dtype, state):
    """[B, N, heads, width], through short sequences, one pass and segments."""
    s = sequences([N] * B, H, Hk, d, dv, dtype, seed=N, device="cuda")
    scale = -0.75 * d ** -0.5
    q, k, v = (s[n].view(B, N, *s[n].shape[1:]) for n in ("q", "k", "v"))
    o, last = sa.sa_decay_attention(q, k, v, s["log_decay"], scale, state_in=s["state_in"] if state else None, want_state=state)
    want = reference(s, scale, [N] * B, state=state)
    check("out", o.view(B * N, H, dv), want["out"], s, scale, dtype, [N] * B, state)
    if state:
        check("state_out", last, want["state_out"], s, scale, dtype, [N] * B)
    else:
        assert last is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths", [[200, 1, 70], [3000, 5]])
def test_decays_from_none_to_total(sa, lengths, dtype):
    """Heads that forget nothing, almost nothing, nearly all at once, all but their own token."""
    s = sequences(lengths, 6, 6, 32, 64, dtype, seed=5, device="cuda")
    s["log_decay"] = torch.tensor([0.0, -1e-6, -0.02, -3.0, -90.0, -float("inf")], device="cuda")
    # the definition needs no product of infinity and zero: a head without memory is one of exp(-800)
    t = dict(s, log_decay=s["log_decay"].clamp(min=-800.0))
    o, last = run(sa, s, 0.2)
    want = reference(t, 0.2, lengths)
    check("out", o, want["out"], t, 0.2, dtype, lengths)
    check("state_out", last, want["state_out"], t, 0.2, dtype, lengths)
    own = 0.2 * (s["q"][:, 5].double() * s["k"][:, 5].double()).sum(-1, keepdim=True) * s["v"][:, 5].double()
    assert bool(((o[:, 5].double() - own).abs() <= 0.02 * own.abs() + 1e-5).all())


@pytest.mark.parametrize("size", [2.0 ** -20, 2.0 ** -10, 1.0, 2.0 ** 8, 2.0 ** 14])
def test_products_outside_of_fp16(sa, size):
    """q k may be far outside of fp16 where out is not: v and scale bring it back."""
    lengths = [150, 700]
    s = sequences(lengths, 2, 2, 64, 64, torch.float16, seed=9, device="cuda")
    s["q"], s["k"] = (s["q"] * size).clamp(-6e4, 6e4), (s["k"] * size).clamp(-6e4, 6e4)
    s["state_in"] *= size
    scale = float(min(1.0, size ** -2))
    o, last = run(sa, s, scale)
    want = reference(s, scale, lengths)
    check("out", o, want["out"], s, scale, torch.float16, lengths)
    check("state_out", last, want["state_out"], s, scale, torch.float16, lengths)


@pytest.mark.parametrize("dtype", TYPES)
def test_columns_of_a_wider_matrix(sa, dtype):
    """q, k and v as column blocks of a fused projection's rows, out as one of a wider matrix: the same bits."""
    B, N, H, Hk, d, dv = 3, 300, 4, 2, 64, 72
    s = sequences([N] * B, H, Hk, d, dv, dtype, seed=3, device="cuda")
    parts = [H * d, Hk * d, Hk * dv]
    fused = torch.cat([s[n].reshape(B * N, -1) for n in ("q", "k", "v")] + [torch.full((B * N, 8), float("nan"), dtype=dtype, device="cuda")], 1)
    q, k, v = (x.view(B, N, h, w) for x, h, w in zip(fused.split(parts + [8], 1)[:3], (H, Hk, Hk), (d, d, dv)))
    wide = torch.full((B * N, H * dv + 16), 5.0, dtype=dtype, device="cuda")
    out = wide[:, 8:8 + H * dv].view(B, N, H, dv)
    sa.sa_decay_attention(q, k, v, s["log_decay"], 0.1, out=out)
    dense, _ = sa.sa_decay_attention(*(s[n].view(B, N, -1, s[n].shape[-1]) for n in ("q", "k", "v")), s["log_decay"], 0.1)
    assert torch.equal(out, dense)
    assert bool((wide[:, :8] == 5.0).all()) and bool((wide[:, -8:] == 5.0).all())


def test_a_tensor_of_more_than_2_31_elements(sa):
    """Tokens 2^16 bytes apart: the last ones begin behind 2^32 bytes."""
    T, H, d = 70001, 1, 64
    s = sequences([T], H, H, d, d, torch.bfloat16, seed=2, device="cuda")
    wide = torch.empty(T, 32768, dtype=torch.bfloat16, device="cuda")
    views = [wide[:, 64 * i:64 * i + 64].view(1, T, H, d) for i in (0, 200, 511)]
    for view, n in zip(views, ("q", "k", "v")):
        view.copy_(s[n].view(1, T, H, d))
    out = wide[:, 6400:6464].view(1, T, H, d)
    o, last = sa.sa_decay_attention(*views, s["log_decay"], 0.1, want_state=True, out=out)
    dense, same = sa.sa_decay_attention(*(s[n].view(1, T, H, d) for n in ("q", "k", "v")), s["log_decay"], 0.1, want_state=True)
    assert torch.equal(o, dense) and torch.equal(last, same)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hk", [(2, 2), (6, 2)])
def test_slots_of_a_cache(sa, H, Hk, dtype):
    """States in place in a cache; slots that are none begin with zeros and leave nothing; all other slots stay as they are."""
    lengths, d, dv = [70, 1, 0, 900, 64, 5], 64, 96
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=8, device="cuda")
    slots = torch.tensor([7, 2, 4, 0, -1, 9], dtype=torch.int32, device="cuda")          # of 9: -1 and 9 are none
    cache = torch.randn(9, Hk, d, dv, device="cuda")
    before = cache.clone()
    s["state_in"] = torch.stack([before[p] if 0 <= p < 9 else torch.zeros_like(before[0]) for p in slots.tolist()])
    o, last = sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=cache, state_out=cache, slots=slots)
    assert last is cache
    want = reference(s, 0.1, lengths)
    check("out", o, want["out"], s, 0.1, dtype, lengths)
    kept = [b for b, p in enumerate(slots.tolist()) if 0 <= p < 9]
    left = torch.stack([cache[p] if b in kept else want["state_out"][b].float() for b, p in enumerate(slots.tolist())])
    check("state_out", left, want["state_out"], s, 0.1, dtype, lengths)
    others = [p for p in range(9) if p not in slots.tolist()]
    assert torch.equal(cache[others], before[others])
    assert torch.equal(cache[4], before[4])                  # the empty sequence's


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [130, 1400])
def test_what_is_not_finite_stays_behind_its_chunk(sa, N, dtype):
    """A NaN or infinity reaches rows of its own sequence from 63 tokens before it on, and no others."""
    s = sequences([N, N], 2, 2, 64, 64, dtype, seed=4, device="cuda")
    clean, _ = run(sa, s, 0.1)
    at = N - 20
    for name, value in (("q", float("nan")), ("k", float("inf")), ("v", float("nan"))):
        bad = dict(s, **{name: s[name].clone()})
        bad[name][at, 0, 5] = value
        o, last = run(sa, bad, 0.1)
        assert torch.equal(o[:at - 63], clean[:at - 63]) and torch.equal(o[N:], clean[N:]) and torch.equal(o[:, 1], clean[:, 1])
        assert not o[at, 0].isfinite().all()
        assert last[1].isfinite().all() and last[0, 1].isfinite().all()


def test_offsets_that_are_none(sa):
    """Offsets outside of the tokens, or descending, read and write nothing outside."""
    s = sequences([100, 100], 2, 2, 64, 64, torch.float32, seed=1, device="cuda")
    for off in ([-50, 90, 1000], [150, 20, 120], [2 ** 31 - 1, -2 ** 31, 7]):
        s["offsets"] = torch.tensor(off, dtype=torch.int32, device="cuda")
        guard = torch.full((400, 2, 64), 3.0, device="cuda")
        sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=s["state_in"], want_state=True, out=guard[100:300])
        assert bool((guard[:100] == 3.0).all()) and bool((guard[300:] == 3.0).all())


def test_no_tokens(sa):
    e = torch.empty(0, 2, 64, device="cuda")
    g = torch.zeros(2, device="cuda")
    state = torch.randn(3, 2, 64, 64, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    o, last = sa.sa_decay_attention(e, e, e, g, 1.0, offsets=off, state_in=state, want_state=True)
    assert o.shape == (0, 2, 64) and torch.equal(last, state)
    _, last = sa.sa_decay_attention(e, e, e, g, 1.0, offsets=off, want_state=True)
    assert bool((last == 0).all())
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert sa.sa_decay_attention(e, e, e, g, 1.0, offsets=none)[0].shape == (0, 2, 64)
    four = torch.empty(2, 0, 2, 64, device="cuda")
    o, last = sa.sa_decay_attention(four, four, four, g, 1.0, state_in=state[:2].clone(), want_state=True)
    assert o.shape == four.shape and torch.equal(last, state[:2])


def test_more_heads_and_short_sequences_than_a_launch_has_threads_for(sa):
    """4096 heads of a single key/value head over 512 sequences of 512 tokens: 64 queries to a workgroup would be 2^24 workgroups of 256 threads."""
    B, N, H, d = 512, 512, 4096, 8
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("40 GB are needed")
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.empty(B, N, H, d, dtype=torch.float16, device="cuda").normal_(generator=g)
    k, v = (torch.randn(B, N, 1, d, generator=g, device="cuda").half() for _ in range(2))
    log_decay = torch.tensor([-0.1], device="cuda")
    out, _ = sa.sa_decay_attention(q, k, v, log_decay, 0.3)
    for b in (0, B - 1):
        for heads in (slice(0, 2), slice(H - 2, H)):
            s = dict(q=q[b, :, heads], k=k[b], v=v[b], dout=out[b, :, heads], log_decay=log_decay, state_in=torch.zeros(1, 1, d, d, device="cuda"),
                     offsets=torch.tensor([0, N], dtype=torch.int32))
            check("out", out[b, :, heads], reference(s, 0.3, [N], state=False)["out"], s, 0.3, torch.float16, [N], False)


def spread(lengths, H, Hk, d, dv, seed, names):
    """fp16 rows whose values span the type: every 7th token large, all others down to subnormals, and of each large token every other element of the
    left operand (names[0]) zero: what those elements meet are small values alone."""
    s = sequences(lengths, H, Hk, d, dv, torch.float16, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    left, right = (s[n] for n in names)
    T = right.shape[0]
    right *= (2.0 ** -torch.randint(0, 22, (T, 1, right.shape[-1]), generator=g)).half()
    large = torch.arange(T) % 7 == 3
    right[large] = (right[large].sign() * (2e4 + 4e4 * torch.rand(right[large].shape, generator=g))).half()
    left[large, :, ::2] = 0
    left[~large] *= (2.0 ** -torch.randint(0, 20, (T, 1, 1), generator=g)[~large]).half()
    s["log_decay"] = torch.tensor([-0.002, -0.9, -3.0, 0.0][:Hk])
    return {n: t.cuda() for n, t in s.items()}


def subnormal(s, left, right, scale, lengths, gradient=False):
    """What fp16's subnormal numbers add to what a state may be off by.  The matrix cores cut a sum of 32 products and what is there before 24 bits below the largest
    product's exponent, to which a subnormal operand counts as one of exponent -14: a product of such a left operand and x costs each of the 33 less
    than 2^-24 2^-14 |x|, and x's second term 2^-11 of that: in all less than 34 2^-38 |x| into the state, which that chunk's sum is added to in fp32."""
    t = dict(s, **{left: ((s[left] != 0) & (s[left].abs() < 2.0 ** -14)).double(), right: s[right].abs()})
    zero = torch.zeros_like(s["state_in"])
    r = reference(dict(t, state_in=zero, dstate_out=zero), scale, lengths, gradients=gradient)
    return 34 * 2.0 ** -38 * r["dstate_in" if gradient else "state_out"]


@pytest.mark.parametrize("H,Hk,d,dv", [(4, 4, 64, 64), (4, 2, 32, 40), (2, 2, 96, 72), (2, 2, 128, 128), (2, 1, 128, 64)])
@pytest.mark.parametrize("lengths", [[150, 1, 64], [900, 70]], ids=lambda l: "-".join(map(str, l)))
def test_states_hold_small_values_beside_large_ones(sa, lengths, H, Hk, d, dv):
    """fp16: an element of a state has fp32's precision of what it is made of, however large the values are whose keys are zero there."""
    def right(kind, got, want, s, more):
        slack, half = allowed(kind, s, 0.1, torch.float16, lengths)
        assert got.isfinite().all()
        assert bool(((got.double() - want).abs() <= slack + more + (want.abs() + slack) * half + 2.0 ** -133).all())

    s = spread(lengths, H, Hk, d, dv, sum(lengths) + d, ("k", "v"))
    s["state_in"].zero_()
    o, last = run(sa, s, 0.1)
    right("state_out", last, reference(s, 0.1, lengths)["state_out"], s, subnormal(s, "k", "v", 0.1, lengths))
    s = spread(lengths, H, Hk, d, dv, sum(lengths) + d + 5, ("q", "dout"))
    s["dstate_out"].zero_()
    got = sa.sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], dstate_out=s["dstate_out"],
                                         want_dstate=True)
    s["state_in"].zero_()
    want = reference(s, 0.1, lengths, gradients=True)["dstate_in"]
    right("dstate_in", got[3], want, s, subnormal(s, "q", "dout", 0.1, lengths, True))


# most sequences of one segment (their mean is below 256), some of several, empty ones at the ends and between
MIXED = [[0, 3, 900, 0, 40, 70, 1, 300, 5, 9, 257, 256, 0], [520, 5, 0, 9, 64, 100]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hk,d,dv", [(3, 3, 64, 64), (6, 2, 96, 72), (2, 2, 128, 128)])
@pytest.mark.parametrize("lengths", MIXED, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("first,last", [(False, False), (True, False), (False, True), (True, True)])
def test_short_sequences_among_long_ones(sa, lengths, H, Hk, d, dv, dtype, first, last):
    """Sequences of one segment go from their own state to their own, those of several through the workspace."""
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=H + d, device="cuda", offset=2, behind=3)
    if not first:
        s["state_in"].zero_()
    ws = torch.full((sa.sa_decay_attention_workspace_bytes(s["q"].shape[0], len(lengths), H, Hk, d, dv, True) // 4,), float("nan"), device="cuda")
    assert ws.numel() > 0
    o, left = sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.2, offsets=s["offsets"], state_in=s["state_in"] if first else None,
                                    want_state=last, out=torch.full_like(s["dout"], 7.0), workspace=ws)
    want = reference(s, 0.2, lengths)
    check("out", o, want["out"], s, 0.2, dtype, lengths)
    assert bool((o[:2] == 7.0).all()) and bool((o[-3:] == 7.0).all())
    if last:
        check("state_out", left, want["state_out"], s, 0.2, dtype, lengths)


def test_short_sequences_among_long_ones_in_place(sa):
    """A cache's states in place; slots that are none."""
    lengths, H, d = MIXED[0], 2, 64
    s = sequences(lengths, H, H, d, d, torch.bfloat16, seed=8, device="cuda")
    slots = torch.tensor([3, 14, 7, 0, -1, 9, 2, 15, 1, 4, 10, 99, 12], dtype=torch.int32, device="cuda")
    cache = torch.randn(15, H, d, d, device="cuda")
    before = cache.clone()
    s["state_in"] = torch.stack([before[p] if 0 <= p < 15 else torch.zeros_like(before[0]) for p in slots.tolist()])
    o, _ = sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=s["offsets"], state_in=cache, state_out=cache, slots=slots)
    want = reference(s, 0.1, lengths)
    check("out", o, want["out"], s, 0.1, torch.bfloat16, lengths)
    left = torch.stack([cache[p] if 0 <= p < 15 else want["state_out"][b].float() for b, p in enumerate(slots.tolist())])
    check("state_out", left, want["state_out"], s, 0.1, torch.bfloat16, lengths)
    others = [p for p in range(15) if p not in slots.tolist()]
    assert torch.equal(cache[others], before[others])


def test_offsets_that_are_none_among_short_sequences(sa):
    """Offsets that descend or leave the tokens, in a batch whose sequences are short on average: nothing outside is read or written."""
    T, H, d = 2000, 2, 64
    s = sequences([T], H, H, d, d, torch.float32, seed=1, device="cuda")
    bad = torch.randint(-3000, 5000, (8, 21), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    state = torch.randn(20, H, d, d, device="cuda")
    need = sa.sa_decay_attention_workspace_bytes(T, 20, H, H, d, d, True) // 4
    for off in bad:
        guard, ws = torch.full((T + 200, H, d), 3.0, device="cuda"), torch.full((need + 2048,), 5.0, device="cuda")
        sa.sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], 0.1, offsets=off.cuda(), state_in=state, want_state=True, out=guard[100:T + 100],
                              workspace=ws[1024:1024 + need])
        assert bool((guard[:100] == 3.0).all()) and bool((guard[T + 100:] == 3.0).all())
        assert bool((ws[:1024] == 5.0).all()) and bool((ws[1024 + need:] == 5.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths", [[130, 90], [1400, 70], [197]], ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("H,Hk,d,dv", [(2, 2, 64, 64), (4, 2, 96, 72), (2, 2, 128, 128), (2, 2, 64, 104), (3, 3, 32, 40)])
def test_rows_before_what_is_not_finite_stay_as_they_are(sa, lengths, H, Hk, d, dv, dtype, state):
    """Rows do not see later tokens, whatever is in them: the same bits; from the token on the columns of its values are NaN, all others the same bits."""
    s = sequences(lengths, H, Hk, d, dv, dtype, seed=4, device="cuda")
    clean, left = run(sa, s, 0.1, state)
    N, G = lengths[0], H // Hk
    for at in sorted({0, 37, N - 20, N - 1}):
        for name, value in (("q", float("nan")), ("k", float("nan")), ("k", -float("inf")), ("v", float("nan")), ("v", float("inf"))):
            bad = dict(s, **{name: s[name].clone()})
            bad[name][at, 1, 5] = value
            o, last = run(sa, bad, 0.1, state)
            heads = slice(1, 2) if name == "q" else slice(G, 2 * G)
            rest = o.clone()
            if name == "q":
                assert not o[at, 1].isfinite().any() and torch.equal(o[at + 1:N], clean[at + 1:N])
                rest[at, heads] = clean[at, heads]
            elif name == "k":
                assert not o[at, heads].isfinite().any()
                rest[at:N, heads] = clean[at:N, heads]
            else:
                assert o[at:N, heads, 5].isnan().all()
                rest[at:N, heads, 5] = clean[at:N, heads, 5]
            assert torch.equal(rest, clean), (name, at)
            if state:
                same = last.clone()
                if name == "k":
                    assert not last[0, 1, 5].isfinite().any()
                    same[0, 1, 5] = left[0, 1, 5]
                if name == "v":
                    assert last[0, 1, :, 5].isnan().all()
                    same[0, 1, :, 5] = left[0, 1, :, 5]
                assert torch.equal(same, left), (name, at)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N", [(3, 200), (2, 1500), (300, 100)])
def test_padding_of_any_bits(sa, B, N, dtype):
    """A padded batch of one length, whose rows behind each sequence's tokens are whatever was in memory."""
    H, d = 4, 64
    s = sequences([N] * B, H, H, d, d, dtype, seed=5, device="cuda")
    q, k, v = (s[n].view(B, N, H, d) for n in ("q", "k", "v"))
    clean, _ = sa.sa_decay_attention(q, k, v, s["log_decay"], 0.1)
    valid = torch.randint(0, N + 1, (B,), generator=torch.Generator().manual_seed(1)).cuda()
    behind = torch.arange(N, device="cuda")[None, :] >= valid[:, None]
    junk = torch.randint(-2 ** 31, 2 ** 31 - 1, (B, N, H, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(torch.int32)
    junk = junk.view(dtype)[..., :d]
    q, k, v = (torch.where(behind[..., None, None], junk.roll(i, 1), t) for i, t in enumerate((q, k, v)))
    assert not v.isfinite().all()
    o, _ = sa.sa_decay_attention(q, k, v, s["log_decay"], 0.1)
    assert torch.equal(o[~behind], clean[~behind])
