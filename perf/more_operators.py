"""Linear attention with a decay for each head, as cases that can be timed and checked one by one.

Three operators on one recurrence, S_t = exp(g) S_{t-1} + k_t v_t^T and o_t = scale q_t^T S_t, with S a [d, dv] state for each
sequence and key/value head: whole prompts (sequences side by side, a state in and out), single tokens over a cache of states, and
the gradient of the prompts.  `own` chooses between the calls that a user makes of `paper_2306_06446_amd.binding` and the same
mathematics in elementary torch operations.  Heads, widths and token counts are those of this repository's configurations (3 or
12 heads of 64 and 197 tokens an image, 4 heads of 64 over sequences of 16384 tokens) or generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_C = 64                    # tokens of a chunk of the plain form


def _case(name, kind, T, B, H, Hk, d, dv, type, ragged=False, states=False):
    """T tokens in B sequences, of the same length each unless `ragged`; H heads of q, Hk of k and v; states: sequences go on from
    a state and leave one (gradients: of both)."""
    return dict(name=name, kind=kind, T=T, B=B, H=H, Hk=Hk, d=d, dv=dv, type=type, ragged=ragged, states=states)


def listed():
    return [
        # one image in the heads of DeiT-Tiny, fp32 as the other attentions here take it: a call that is all latency
        _case("prompt, one image", "prompt", 197, 1, 3, 3, 64, 64, "f32"),
        # the DeiT-Base heads at batch 64: many short sequences
        _case("prompt, base batch", "prompt", 64 * 197, 64, 12, 12, 64, 64, "bf16"),
        # a single long prompt of a generic model, whose state a decoder goes on from: few heads, a long axis
        _case("prompt, one long", "prompt", 16384, 1, 16, 16, 128, 128, "bf16", states=True),
        # eight sequences of 16384 tokens, 4 heads of 64
        _case("prompt, long batch", "prompt", 8 * 16384, 8, 4, 4, 64, 64, "bf16"),
        # prompts of a serving batch as they come: ragged, each with its slot in the cache, heads that share keys and values, odd widths
        _case("prompt, ragged shared", "prompt", 50021, 37, 12, 4, 96, 72, "f16", ragged=True, states=True),
        # a single token of a single sequence
        _case("step, one sequence", "step", 1, 1, 3, 3, 64, 64, "bf16"),
        # decoding at batch 64, a generic model's heads: the states are all there is to read and write
        _case("step, batch", "step", 64, 64, 16, 16, 128, 128, "bf16"),
        # shared heads, an odd batch and odd widths, fp32
        _case("step, odd shared", "step", 333, 333, 12, 4, 80, 40, "f32"),
        # training on one image of DeiT-Tiny's heads
        _case("grad, one image", "grad", 197, 1, 3, 3, 64, 64, "f32"),
        # training at DeiT-Base's heads, batch 64
        _case("grad, base batch", "grad", 64 * 197, 64, 12, 12, 64, 64, "bf16"),
        # training on eight long sequences: the largest pass
        _case("grad, long batch", "grad", 8 * 16384, 8, 4, 4, 64, 64, "bf16"),
        # packed documents that go on from a state (truncated backpropagation), shared heads
        _case("grad, ragged shared", "grad", 30011, 37, 12, 4, 64, 104, "f16", ragged=True, states=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """A case of the same ranges: 1 to 131072 tokens in 1 to 512 sequences, up to 32 heads, widths 8 to 128 in steps of 8, every type."""
    top = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(("prompt", "prompt", "step", "grad", "grad"))
        B = _log_int(rng, 1, 512)
        N = 1 if kind == "step" else _log_int(rng, 1, 131072)
        H = rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 24, 32))
        Hk = rng.choice([h for h in range(1, H + 1) if H % h == 0] + [H, H, H])
        d, dv = (rng.choice((rng.choice((32, 64, 64, 128)), 8 * rng.randint(1, 16))) for _ in range(2))
        ragged = kind != "step" and rng.random() < 0.4
        T = B * N - (rng.randint(0, B * N // 4) if ragged else 0)
        case = _case("", kind, T, B, H, Hk, d, dv, rng.choice(("f32", "f16", "bf16")), ragged, kind != "step" and rng.random() < 0.5)
        case.pop("name")
        if T <= 131072 and work(case)["bytes"] <= top and (T // _C + B) * H <= 8192:
            return case


def work(case):
    T, B, H, Hk, d, dv = (case[k] for k in ("T", "B", "H", "Hk", "d", "dv"))
    size = torch.empty(0, dtype=_TYPES[case["type"]]).element_size()
    q, o, k, v, state = H * d, H * dv, Hk * d, Hk * dv, 4 * B * Hk * d * dv
    read, update = 2 * H * d * dv, 3 * Hk * d * dv           # a token's product with the state, its way into the state
    offsets = 4 * (B + 1) if case["ragged"] else 0
    if case["kind"] == "grad":
        return {"bytes": T * size * (2 * q + o + 2 * k + 2 * v) + offsets + (3 * state if case["states"] else 0) + 4 * Hk,
                "flops": T * (3 * read + 2 * update)}
    states = 2 * state if case["states"] or case["kind"] == "step" else 0
    return {"bytes": T * size * (q + o + k + v) + offsets + states + 4 * Hk, "flops": T * (read + update)}


# ------------------------------------------------------------------------------------------ inputs --

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _lengths(case, seed):
    """Tokens of each sequence: the same, or spread as documents are, a few long ones among many short; empty ones may be there."""
    T, B = case["T"], case["B"]
    if not case["ragged"]:
        return [T // B] * B
    rng = random.Random(seed)
    size = [math.exp(rng.gauss(0.0, 1.2)) for _ in range(B)]
    n = [int(T * s / sum(size)) for s in size]
    n[-1] += T - sum(n)
    return n


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, B, H, Hk, d, dv = (case[k] for k in ("T", "B", "H", "Hk", "d", "dv"))
    dtype = _TYPES[case["type"]]
    s = {"lengths": _lengths(case, seed)}
    s["q"], s["k"], s["v"] = _randn(g, T, H, d).to(dtype), _randn(g, T, Hk, d).to(dtype), _randn(g, T, Hk, dv).to(dtype)
    # heads that remember 2 to 1024 tokens, as models of this kind have them
    memory = 2.0 ** (1.0 + 9.0 * (torch.arange(Hk, device="cuda") + torch.rand(Hk, generator=g, device="cuda")) / Hk)
    s["log_decay"] = torch.log1p(-1.0 / memory)
    if case["states"] or case["kind"] == "step":
        # states behind a long text: sums of memory / 2 products
        s["state_in"] = _randn(g, B, Hk, d, dv) * torch.sqrt(0.5 * memory)[:, None, None]
    if case["kind"] != "grad" and (case["states"] or case["kind"] == "step"):
        s["slots"] = torch.randperm(B, generator=g, device="cuda").to(torch.int32)          # a cache in the order of arrival
    if case["kind"] == "grad":
        s["dout"] = (0.05 * _randn(g, T, H, dv)).to(dtype)
        if case["states"]:
            s["dstate_out"] = 0.05 * _randn(g, B, Hk, d, dv)
    s["scale"] = float(torch.tensor(d ** -0.5, dtype=torch.float32))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    T, B, H, Hk, d, dv = (case[k] for k in ("T", "B", "H", "Hk", "d", "dv"))
    if case["ragged"]:
        s["offsets"] = torch.tensor([0] + s["lengths"], device="cuda").cumsum(0).to(torch.int32)
    if own:
        # the output buffers and the workspace that a program keeps from call to call
        from paper_2306_06446_amd import binding as sa
        s["sa"] = sa
        dtype = _TYPES[case["type"]]
        if case["kind"] != "step" and not case["ragged"]:     # [B, N, heads, width], as the attentions here take them
            for name in ("q", "k", "v", "dout"):
                if name in s:
                    s[name] = s[name].view(B, T // B, *s[name].shape[1:])
        if case["kind"] == "grad":
            s["out"] = {n: torch.empty_like(s[n[1:]]) for n in ("dq", "dk", "dv")}
            if case["states"]:
                s["out"]["dstate_in"] = torch.empty_like(s["state_in"])
            size = sa.sa_decay_attention_backward_workspace_bytes(T, B, H, Hk, d, dv, case["ragged"])
        else:
            s["out"] = dict(out=torch.empty(*s["q"].shape[:-1], dv, dtype=dtype, device="cuda"))
            if "state_in" in s:
                s["out"]["state_out"] = torch.empty_like(s["state_in"])
            size = sa.sa_decay_attention_workspace_bytes(T, B, H, Hk, d, dv, case["ragged"])
        if case["kind"] != "step":
            s["out"]["workspace"] = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    elif case["kind"] != "step":
        # which tokens each chunk has (T: none), its sequence, its place in it and how many tokens it has: the sequences' plan
        rows, seq, start, count, first = [], [], [], [], 0
        for b, n in enumerate(s["lengths"]):
            at = torch.arange(-(-n // _C) * _C).view(-1, _C)
            rows.append(torch.where(at < n, first + at, T))
            seq += [b] * len(at)
            start += range(0, n, _C)
            count += [min(_C, n - c) for c in range(0, n, _C)]
            first += n
        s["rows"] = torch.cat(rows).cuda()
        s["seq"], s["start"], s["count"], s["length"] = (torch.tensor(x, device="cuda") for x in (seq, start, count, s["lengths"]))
    return s


# ---------------------------------------------------------------------------------------- the passes --

def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own[kind](s)
    return _plain[kind](s)


def _own_prompt(s):
    out, state = s["sa"].sa_decay_attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], offsets=s.get("offsets"),
                                            state_in=s.get("state_in"), slots=s.get("slots"), **s["out"])
    return [out.view(s["case"]["T"], *out.shape[-2:])] + ([state] if state is not None else [])


def _own_step(s):
    return list(s["sa"].sa_decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["state_in"],
                                                slots=s["slots"], **s["out"]))


def _own_grad(s):
    dq, dk, dv, dstate = s["sa"].sa_decay_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["log_decay"], s["scale"],
                                                             offsets=s.get("offsets"), state_in=s.get("state_in"),
                                                             dstate_out=s.get("dstate_out"), **s["out"])
    return [t.view(s["case"]["T"], *t.shape[-2:]) for t in (dq, dk, dv)] + ([dstate] if dstate is not None else [])


_own = dict(prompt=_own_prompt, step=_own_step, grad=_own_grad)


def _pow(g, n):
    """exp(n g), n a tensor of token counts: [heads, *n.shape]."""
    return torch.exp(g.view(-1, *[1] * n.dim()) * n.float())


def _chunked(s, x, heads):
    """[T, heads of x, w] to [chunks, heads, _C, w] fp32, zeros where a chunk has no token."""
    x = torch.cat([x.float(), x.new_zeros(1, *x.shape[1:], dtype=torch.float32)])[s["rows"]].transpose(1, 2)
    return x.repeat_interleave(heads // x.shape[1], 1) if heads != x.shape[1] else x


def _unchunked(s, x, dtype):
    """Back to [T, heads, w]."""
    T = s["case"]["T"]
    out = x.new_empty(T + 1, x.shape[1], x.shape[3])
    out[s["rows"].view(-1)] = x.transpose(1, 2).reshape(-1, x.shape[1], x.shape[3])
    return out[:T].to(dtype)


def _weights(s, Hk):
    """Decays within a chunk, to its tokens from the state before it, from them to the state behind it, and between chunks."""
    g = s["log_decay"]
    i = torch.arange(_C, device=g.device)
    far = i[:, None] - i[None, :]
    inside = torch.where(far >= 0, _pow(g, far.clamp(min=0)), torch.zeros((), device=g.device))
    into = _pow(g, i + 1)
    left = s["count"][:, None] - 1 - i
    out_of = torch.where(left >= 0, _pow(g, left.clamp(min=0)), torch.zeros((), device=g.device)).transpose(0, 1)
    end = s["start"] + s["count"]
    gap = s["start"][:, None] - end[None, :]
    same = (s["seq"][:, None] == s["seq"][None, :]) & (gap >= 0)
    between = torch.where(same, _pow(g, gap.clamp(min=0)), torch.zeros((), device=g.device))
    last = s["length"][:, None] - end[None, :]
    mine = torch.arange(len(s["length"]), device=g.device)[:, None] == s["seq"][None, :]
    to_end = torch.where(mine, _pow(g, last.clamp(min=0)), torch.zeros((), device=g.device))
    return inside, into, out_of, between, to_end


def _over(w, x):
    """w [Hk, m, n] on x [n, Hk, d, dv]: [m, Hk, d, dv]."""
    n, Hk, d, dv = x.shape
    y = torch.matmul(w, x.transpose(0, 1).reshape(Hk, n, d * dv))
    return y.view(Hk, -1, d, dv).transpose(0, 1)


def _plain_prompt(s):
    case = s["case"]
    H, Hk, g = case["H"], case["Hk"], s["log_decay"]
    inside, into, out_of, between, to_end = _weights(s, Hk)
    q, k, v = _chunked(s, s["q"], H), _chunked(s, s["k"], Hk), _chunked(s, s["v"], Hk)
    own_sum = torch.matmul((k * out_of[..., None]).transpose(2, 3).contiguous(), v)
    state = _over(between, own_sum)
    if "state_in" in s:
        first = s["state_in"]
        if "slots" in s:
            first = first[s["slots"].long()]
        state = state + _pow(g, s["start"]).t()[..., None, None] * first[s["seq"]]
    if H != Hk:
        k, v, state, inside, into = (x.repeat_interleave(H // Hk, a) for x, a in ((k, 1), (v, 1), (state, 1), (inside, 0), (into, 0)))
    o = torch.matmul(torch.matmul(q, k.transpose(2, 3).contiguous()) * inside, v) + torch.matmul(q * into[..., None], state)
    out = [_unchunked(s, o * s["scale"], s["q"].dtype)]
    if "state_in" in s:
        last = _over(to_end, own_sum) + _pow(g, s["length"]).t()[..., None, None] * first
        if "slots" in s:
            kept = torch.empty_like(last)
            kept[s["slots"].long()] = last
            last = kept
        out.append(last)
    return out


def _plain_step(s):
    case = s["case"]
    slots = s["slots"].long()
    k, v = s["k"].float(), s["v"].float()
    state = torch.exp(s["log_decay"])[:, None, None] * s["state_in"][slots] + k[..., None] * v[..., None, :]
    q = s["q"].float().view(case["B"], case["Hk"], -1, case["d"])
    out = torch.matmul(q, state).view(case["B"], case["H"], case["dv"]) * s["scale"]
    kept = torch.empty_like(state)
    kept[slots] = state
    return [out.to(s["q"].dtype), kept]


def _plain_grad(s):
    case = s["case"]
    H, Hk, g, dtype = case["H"], case["Hk"], s["log_decay"], s["q"].dtype
    G = H // Hk
    inside, into, out_of, between, to_end = _weights(s, Hk)
    q, do = _chunked(s, s["q"], H), _chunked(s, s["dout"], H) * s["scale"]
    k, v = _chunked(s, s["k"], Hk), _chunked(s, s["v"], Hk)
    state = _over(between, torch.matmul((k * out_of[..., None]).transpose(2, 3).contiguous(), v))
    if "state_in" in s:
        state = state + _pow(g, s["start"]).t()[..., None, None] * s["state_in"][s["seq"]]

    def shared(x):
        return x.repeat_interleave(G, 1) if G > 1 else x

    def summed(x):
        return x.view(x.shape[0], Hk, G, *x.shape[2:]).sum(2) if G > 1 else x

    wide_in, wide_into = (x.repeat_interleave(G, 0) if G > 1 else x for x in (inside, into))
    kh, vh = shared(k), shared(v)
    dp = torch.matmul(do, vh.transpose(2, 3).contiguous()) * wide_in
    dq = torch.matmul(dp, kh) + torch.matmul(do * wide_into[..., None], shared(state).transpose(2, 3).contiguous())
    own_sum = summed(torch.matmul((q * wide_into[..., None]).transpose(2, 3).contiguous(), do))
    dstate = _over(between.transpose(1, 2).contiguous(), own_sum)                   # of the state behind each chunk
    if "dstate_out" in s:
        rest = s["length"][s["seq"]] - s["start"] - s["count"]
        dstate = dstate + _pow(g, rest).t()[..., None, None] * s["dstate_out"][s["seq"]]
    dk = summed(torch.matmul(dp.transpose(2, 3).contiguous(), q)) + torch.matmul(v * out_of[..., None], dstate.transpose(2, 3).contiguous())
    p = torch.matmul(q, kh.transpose(2, 3).contiguous()) * wide_in
    dv = summed(torch.matmul(p.transpose(2, 3).contiguous(), do)) + torch.matmul(k * out_of[..., None], dstate)
    out = [_unchunked(s, x, dtype) for x in (dq, dk, dv)]
    if "dstate_out" in s:
        mine = torch.arange(case["B"], device=g.device)[:, None] == s["seq"][None, :]
        from_start = torch.where(mine, _pow(g, s["start"].expand(case["B"], -1)), torch.zeros((), device=g.device))
        out.append(_over(from_start, own_sum) + _pow(g, s["length"]).t()[..., None, None] * s["dstate_out"])
    return out


_plain = dict(prompt=_plain_prompt, step=_plain_step, grad=_plain_grad)


# ------------------------------------------------------------------------- the definitions in 64 bits --

def _decays(g, later, earlier):
    """exp((i - j) g) for j <= i, else 0."""
    n = later[:, None] - earlier[None, :]
    return torch.exp(g[:, None, None] * n.clamp(min=0)) * (n >= 0)


def exact(case, seed):
    """Every output as the sum over all pairs of tokens that its definition is, block by block of rows, sequence by sequence."""
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    H, Hk, g, scale, kind = case["H"], case["Hk"], s["log_decay"], s["scale"], case["kind"]
    G = H // Hk
    of = torch.arange(H, device=g.device) // G               # the key/value head of each head
    q, k, v = s["q"], s["k"], s["v"]
    if kind == "step":
        slots = s["slots"].long()
        new = torch.empty_like(s["state_in"])
        new[slots] = s["state_in"][slots] * g.exp().view(1, -1, 1, 1) + k.unsqueeze(-1) * v.unsqueeze(-2)
        return [(q.unsqueeze(-1) * new[slots][:, of]).sum(-2) * scale, new]
    states = [None] * case["B"]
    results = [torch.empty_like(t) for t in (q, k, v)] if kind == "grad" else [q.new_empty(case["T"], H, case["dv"])]
    first = 0
    for b, n in enumerate(s["lengths"]):
        at = slice(first, first + n)
        first += n
        sq, sk, sv = (x[at].transpose(0, 1).contiguous() for x in (q, k, v))       # [heads, n, w]
        place = int(s["slots"][b]) if "slots" in s else b
        initial = s["state_in"][place] if "state_in" in s else None
        pos = torch.arange(n, device=g.device, dtype=torch.float64)
        step = max(64, min(2048, 1 << 28 >> max(1, n * H).bit_length()))
        blocks = [slice(i, min(n, i + step)) for i in range(0, n, step)]
        if kind == "prompt":
            for r in blocks:
                c = slice(0, r.stop)
                a = torch.matmul(sq[:, r], sk[of, c].transpose(1, 2).contiguous()) * _decays(g, pos[r], pos[c])[of]
                o = torch.matmul(a, sv[of, c])
                if initial is not None:
                    o += torch.matmul(sq[:, r], initial[of]) * torch.exp(g[of, None, None] * (pos[r] + 1)[:, None])
                results[0][at][r] = o.transpose(0, 1) * scale
            if initial is not None:
                fade = torch.exp(g[:, None, None] * (n - 1 - pos)[:, None])
                states[place] = initial * torch.exp(g * n)[:, None, None] + torch.matmul((sk * fade).transpose(1, 2).contiguous(), sv)
            continue
        do = s["dout"][at].transpose(0, 1).contiguous() * scale
        behind = s["dstate_out"][b] if "dstate_out" in s else None
        for r in blocks:
            c = slice(0, r.stop)
            a = torch.matmul(do[:, r], sv[of, c].transpose(1, 2).contiguous()) * _decays(g, pos[r], pos[c])[of]
            dq = torch.matmul(a, sk[of, c])
            if initial is not None:
                dq += torch.matmul(do[:, r], initial[of].transpose(1, 2).contiguous()) * torch.exp(g[of, None, None] * (pos[r] + 1)[:, None])
            results[0][at][r] = dq.transpose(0, 1)
            # the same rows as keys: all later queries
            c = slice(r.start, n)
            fade = _decays(g, pos[c], pos[r]).transpose(1, 2).contiguous()[of]
            dk = torch.matmul(torch.matmul(sv[of, r], do[:, c].transpose(1, 2).contiguous()) * fade, sq[:, c])
            dv = torch.matmul(torch.matmul(sk[of, r], sq[:, c].transpose(1, 2).contiguous()) * fade, do[:, c])
            dk, dv = (x.view(Hk, G, *x.shape[1:]).sum(1) for x in (dk, dv))
            if behind is not None:
                rest = torch.exp(g[:, None, None] * (n - 1 - pos[r])[:, None])
                dk += rest * torch.matmul(sv[:, r], behind.transpose(1, 2).contiguous())
                dv += rest * torch.matmul(sk[:, r], behind)
            results[1][at][r] = dk.transpose(0, 1)
            results[2][at][r] = dv.transpose(0, 1)
        if behind is not None:
            fade = torch.exp(g[of, None, None] * (pos + 1)[:, None])
            from_rows = torch.matmul((sq * fade).transpose(1, 2).contiguous(), do)
            states[b] = behind * torch.exp(g * n)[:, None, None] + from_rows.view(Hk, G, *from_rows.shape[1:]).sum(1)
    return results + ([torch.stack(states)] if case["states"] else [])
