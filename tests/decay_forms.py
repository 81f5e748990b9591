"""Linear attention with a decay for each head in 64 bits, token by token as its definition reads, and sequences to try it on."""
import torch


def sequences(lengths, H, Hk, d, dv, dtype, seed=0, device="cpu", offset=0, behind=0):
    """Rows of sequences one behind the other, with `offset` rows before the first one and `behind` behind the last: NaN there."""
    g = torch.Generator().manual_seed(seed)
    T = offset + sum(lengths) + behind
    s = dict(q=torch.randn(T, H, d, generator=g), k=torch.randn(T, Hk, d, generator=g), v=torch.randn(T, Hk, dv, generator=g),
             dout=torch.randn(T, H, dv, generator=g))
    for t in s.values():
        t[:offset] = float("nan")
        t[T - behind:] = float("nan")
    s = {k: t.to(dtype).to(device) for k, t in s.items()}
    memory = 2.0 ** (torch.arange(Hk) % 8 + torch.rand(Hk, generator=g))
    s["log_decay"] = torch.log1p(-0.75 / memory).to(device)
    s["state_in"] = torch.randn(len(lengths), Hk, d, dv, generator=g).to(device)
    s["dstate_out"] = torch.randn(len(lengths), Hk, d, dv, generator=g).to(device)
    s["offsets"] = (offset + torch.tensor([0] + list(lengths)).cumsum(0)).to(torch.int32).to(device)
    return s


def forward(q, k, v, log_decay, scale, state):
    """One sequence: q [n, H, d], k [n, Hk, d], v [n, Hk, dv], state [Hk, d, dv], all fp64: (out [n, H, dv], state behind it)."""
    G = q.shape[1] // k.shape[1]
    lam = torch.exp(log_decay)[:, None, None]
    out = []
    for t in range(q.shape[0]):
        state = lam * state + k[t][:, :, None] * v[t][:, None, :]
        out.append(scale * torch.einsum("hd,hde->he", q[t], state.repeat_interleave(G, 0)))
    return torch.stack(out) if out else q.new_zeros(0, q.shape[1], v.shape[2]), state


def pairs(q, k, v, log_decay, scale, state):
    """The same as a sum over all pairs of tokens, for longer sequences."""
    n, G = q.shape[0], q.shape[1] // k.shape[1]
    i = torch.arange(n, device=q.device)
    far = i[:, None] - i[None, :]
    lam = torch.where(far >= 0, torch.exp(log_decay[:, None, None] * far.clamp(min=0)), torch.zeros((), dtype=q.dtype, device=q.device))
    lam = torch.where(far == 0, torch.ones_like(lam), lam).repeat_interleave(G, 0)
    kh, vh = (x.transpose(0, 1).repeat_interleave(G, 0) for x in (k, v))
    fade = torch.exp(log_decay[:, None] * (i + 1)).repeat_interleave(G, 0)
    o = torch.matmul(torch.matmul(q.transpose(0, 1), kh.transpose(1, 2).contiguous()) * lam, vh)
    o = o + fade[..., None] * torch.matmul(q.transpose(0, 1), state.repeat_interleave(G, 0))
    left = n - 1 - i
    keep = torch.where(left == 0, torch.ones((), dtype=q.dtype, device=q.device), torch.exp(log_decay[:, None] * left))
    last = torch.exp(log_decay * n)[:, None, None] * state if n else state
    last = last + torch.matmul((k.transpose(0, 1) * keep[..., None]).transpose(1, 2).contiguous(), v.transpose(0, 1))
    return scale * o.transpose(0, 1), last


def reference(s, scale, lengths, one=pairs, state=True, gradients=False):
    """All sequences in 64 bits: dict of out and state_out, with gradients also dq, dk, dv, dstate_in of <out, dout> + <state_out, dstate_out>."""
    first = s["offsets"].tolist()
    leaves = {n: s[n].double() for n in ("q", "k", "v")}
    leaves["state_in"] = s["state_in"].double() if state else torch.zeros_like(s["state_in"], dtype=torch.float64)
    out = torch.full(s["dout"].shape, float("nan"), dtype=torch.float64, device=s["q"].device)
    states, grads = [], {n: torch.full(t.shape, float("nan"), dtype=torch.float64, device=t.device) for n, t in leaves.items()}
    for b, n in enumerate(lengths):
        at = slice(first[b], first[b] + n)
        x = {name: (t[at] if name != "state_in" else t[b]).clone().requires_grad_(gradients) for name, t in leaves.items()}
        o, last = one(x["q"], x["k"], x["v"], s["log_decay"].double(), scale, x["state_in"])
        out[at] = o.detach()
        states.append(last.detach())
        if gradients:
            loss = (o * s["dout"][at].double()).sum() + (last * (s["dstate_out"][b].double() if state else 0.0)).sum()
            for (name, t), got in zip(x.items(), torch.autograd.grad(loss, list(x.values()), allow_unused=True)):
                got = torch.zeros_like(t) if got is None else got
                if name == "state_in":
                    grads[name][b] = got
                else:
                    grads[name][at] = got
    r = dict(out=out, state_out=torch.stack(states))
    if gradients:
        r.update(dq=grads["q"], dk=grads["k"], dv=grads["v"], dstate_in=grads["state_in"])
    return r


HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def allowed(kind, s, scale, dtype, lengths, state=True):
    """What a result may be off by, element by element: half a step of the type it is rounded to, and what sums in fp32 over operands off by
    `terms` may be, relative to the same sum of magnitudes.  Of that sum every product of three operands passes at most two made operands (2^-18 each in
    16 bits, 2^-22 in fp32 and in the states), a decay (an exponent of up to 30 halves of 2^-24, and it is a factor of two or three), and fp32 additions, one for each
    token and element behind each other at most: (n + d + dv) 2^-24."""
    big = {n: t.abs() if torch.is_tensor(t) and t.is_floating_point() and n != "log_decay" else t for n, t in s.items()}
    r = reference(big, abs(scale), lengths, state=state, gradients=kind != "out" and kind != "state_out")
    n = max(lengths) if lengths else 0
    fp32 = kind in ("state_out", "dstate_in")
    terms = (2.0 ** -22 if fp32 or dtype is torch.float32 else 2.0 ** -17) + (n + s["q"].shape[-1] + s["v"].shape[-1] + 90) * 2.0 ** -24
    return r[kind] * terms, 2.0 ** -24 if fp32 else HALF_STEP[dtype]


def check(kind, got, want, s, scale, dtype, lengths, state=True):
    slack, half = allowed(kind, s, scale, dtype, lengths, state)
    there = ~want.isnan()
    tiny = 2.0 ** -25 if dtype is torch.float16 and kind not in ("state_out", "dstate_in") else 2.0 ** -133     # half of the smallest subnormal's step
    off = (got.double() - want).abs()[there]
    lim = (slack + (want.abs() + slack) * half)[there] + tiny
    assert got[there].isfinite().all(), kind
    worst = (off / lim).max().item() if off.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g times what it may be off by" % (kind, worst)
    return worst
