"""The operators that train the mixture half of a block, as cases that can be timed and checked one by one.

Four operators: LayerNorm that keeps its statistics (with the router's logits), its gradient (with the residual's and the
router's), the latency-aware balance loss with its gradient and the tokens of each expert, and the gradient of the gated
combine behind a top-1 dispatch.  `own` chooses between the calls that a user makes of `paper_2306_06446_amd.binding` and the
same mathematics in elementary torch operations.  Widths and token counts are those of this repository's configurations
(DeiT-Tiny and -Base blocks, 197 tokens an image; sequences of 16384 tokens) or generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-6
_PAIRS = (("f32", "f32"), ("f32", "f16"), ("f32", "bf16"), ("f16", "f16"), ("bf16", "bf16"))


def _norm(name, T, E, x, y, experts=0):
    """sa_layernorm: rows of type x to rows of type y; experts > 0: the router's logits as well."""
    return dict(name=name, kind="norm", T=T, E=E, x=x, y=y, experts=experts)


def _norm_grad(name, T, E, x, y, experts=0, residual=True, weights=True):
    """sa_layernorm_backward: weights = False is a frozen norm, of which only the rows' gradient is wanted."""
    return dict(name=name, kind="norm_grad", T=T, E=E, x=x, y=y, experts=experts, residual=residual, weights=weights)


def _balance(name, T, experts, noise_std, padded):
    """sa_moe_balance_loss_grad: `padded` of the tokens are padding and count for nothing."""
    return dict(name=name, kind="balance", T=T, experts=experts, noise_std=noise_std, padded=padded)


def _combine_grad(name, T, E, y, src, experts):
    """sa_combine_rows_backward: all experts' rows, in the order of the dispatch."""
    return dict(name=name, kind="combine_grad", T=T, E=E, y=y, src=src, experts=experts)


def listed():
    return [
        # a single row: the latency of a norm in a loop over tokens
        _norm("norm, one token", 1, 768, "f32", "f16"),
        # the second norm of a DeiT-Base block, batch 64: fp32 residual stream, fp16 rows for the experts, router of two
        _norm("norm, base batch", 64 * 197, 768, "f32", "f16", 2),
        # a width that no vector load divides, in 16 bits throughout
        _norm("norm, odd width", 5003, 4099, "bf16", "bf16"),
        # one image of a DeiT-Tiny block in training: few rows, all the gradients
        _norm_grad("norm grad, one image", 197, 192, "f32", "f32", 2),
        # the second norm of the DeiT-Base block at batch 64, mixed precision, router and residual
        _norm_grad("norm grad, base batch", 64 * 197, 768, "f32", "f16", 2),
        # an odd width and an odd number of rows, no residual
        _norm_grad("norm grad, odd width", 3001, 1001, "f16", "f16", 0, False),
        # eight long sequences at a generic model's width: the largest pass
        _norm_grad("norm grad, long batch", 8 * 16384, 1024, "bf16", "bf16"),
        # the loss of one image: a pass that is all latency
        _balance("balance, one image", 197, 2, 0.1, 0.0),
        # eight long sequences over eight experts, a tenth of the tokens padding
        _balance("balance, long batch", 8 * 16384, 8, 0.25, 0.1),
        # many short documents in one step, two experts
        _balance("balance, a million tokens", 1000003, 2, 0.1, 0.0),
        # both experts of the DeiT-Base block, fp16 rows under an fp32 residual stream
        _combine_grad("combine grad, base batch", 64 * 197, 768, "f32", "f16", 2),
        # eight experts, a ragged number of tokens, bf16
        _combine_grad("combine grad, eight experts", 50021, 500, "bf16", "bf16", 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """A case of the same ranges: 1 to 131072 rows of 8 to 8192 columns, 1 to a million tokens of 2 to 8 experts, every type."""
    top = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(("norm", "norm_grad", "norm_grad", "balance", "combine_grad"))
        x, y = rng.choice(_PAIRS)
        T, E = _log_int(rng, 1, 131072), _log_int(rng, 8, 8192)
        if rng.random() < 0.5:
            E = max(8, E // 8 * 8)
        experts = rng.choice((0, 0, 2, 2, rng.randint(3, 8)))
        if kind == "norm":
            case = _norm("", T, E, x, y, experts)
        elif kind == "norm_grad":
            case = _norm_grad("", T, E, x, y, experts, rng.random() < 0.6, rng.random() < 0.8)
        elif kind == "balance":
            case = _balance("", _log_int(rng, 1, 1000000), rng.choice((2, 2, 3, 4, 6, 8)), rng.uniform(0.05, 1.0),
                            rng.choice((0.0, 0.0, rng.uniform(0.0, 0.6))))
        else:
            case = _combine_grad("", T, E, x, y, max(2, experts))
        case.pop("name")
        if work(case)["bytes"] <= top:
            return case


def work(case):
    T, n = case["T"], case.get("experts", 0)
    size = {k: torch.empty(0, dtype=v).element_size() for k, v in _TYPES.items()}
    if case["kind"] == "balance":
        # logits in, their gradient out, a byte of the padding mask; a softmax, a normal distribution and its density per logit
        return {"bytes": T * (8 * n + (1 if case["padded"] else 0)) + 16 * n, "flops": T * n * 60}
    E = case["E"]
    if case["kind"] == "norm":
        return {"bytes": T * E * (size[case["x"]] + size[case["y"]]) + T * (8 + 4 * n) + E * (8 + 4 * n),
                "flops": T * E * (8 + 2 * n)}
    if case["kind"] == "norm_grad":
        rows = T * E * (size[case["x"]] * (3 if case["residual"] else 2) + size[case["y"]])
        columns = E * (4 + (4 + 4 * n if n else 0) + (8 + 4 * n if case["weights"] else 0))
        return {"bytes": rows + T * (8 + 4 * n) + columns, "flops": T * E * (14 + 4 * n)}
    return {"bytes": T * E * (size[case["y"]] + 2 * size[case["src"]]) + T * (4 + 4 + 4 + 8 * n), "flops": T * E * 3}


# ------------------------------------------------------------------------------------------ inputs --

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _rows(g, T, E, dtype):
    """A residual stream: every token has its own size and offset, a few columns are much larger than the rest."""
    x = _randn(g, T, E)
    x *= torch.exp(0.5 * _randn(g, T, 1))
    x += 0.5 * _randn(g, T, 1)
    big = torch.randperm(E, generator=g, device="cuda")[:max(1, E // 256)]
    x[:, big] *= 8.0
    return x.to(dtype)


def _logits(g, T, n):
    """Router logits with preferred experts; an eighth of the tokens has logits on a coarse grid, as from 8-bit activations, with ties."""
    l = _randn(g, T, n) * 1.5 + 0.5 * _randn(g, 1, n)
    l[::8] = torch.round(2.0 * l[::8]) / 2.0
    return l.contiguous()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, n = case["T"], case.get("experts", 0)
    s = {}
    if case["kind"] == "balance":
        s["logits"] = _logits(g, T, n)
        a = 0.5 + _rand(g, n)
        s["alpha"] = a / a.sum()
        s["dlosses"] = 0.01 * (0.5 + _rand(g, 2))            # the weights of the two losses in the sum that is trained on
        if case["padded"]:
            s["valid"] = (_rand(g, T) >= case["padded"]).to(torch.uint8)
            s["logits"][s["valid"] == 0] = float("nan")      # padding holds whatever was there
        return s
    E = case["E"]
    if case["kind"] == "combine_grad":
        s["logits"] = _logits(g, T, n)
        top = s["logits"][:, 0].clone()
        expert = torch.zeros(T, dtype=torch.int64, device="cuda")
        for e in range(1, n):                                # the largest, ties to the lowest index
            better = s["logits"][:, e] > top
            top = torch.where(better, s["logits"][:, e], top)
            expert = torch.where(better, torch.full_like(expert, e), expert)
        s["perm"] = torch.sort(expert, stable=True).indices.to(torch.int32)
        s["gate"] = torch.softmax(s["logits"].double(), 1).gather(1, expert[:, None])[:, 0].float()
        s["dy"] = (0.05 * _randn(g, T, E)).to(_TYPES[case["y"]])
        s["src"] = _randn(g, T, E).to(_TYPES[case["src"]])
        return s
    s["x"] = _rows(g, T, E, _TYPES[case["x"]])
    s["gamma"] = 1.0 + 0.1 * _randn(g, E)
    s["beta"] = 0.1 * _randn(g, E)
    if n:
        s["wg"] = _randn(g, E, n) / math.sqrt(E)
        s["bg"] = 0.1 * _randn(g, n)
    if case["kind"] == "norm_grad":
        s["dy"] = (0.05 * _randn(g, T, E)).to(_TYPES[case["y"]])
        if case["residual"]:
            s["dres"] = (0.05 * _randn(g, T, E)).to(_TYPES[case["x"]])
        if n:
            s["dlogits"] = 0.05 * _randn(g, T, n)
        x = s["x"].double()
        mean = x.mean(1)
        s["mean"] = mean.float()                             # what the forward pass left
        s["rstd"] = (1.0 / torch.sqrt((x - mean[:, None]).square_().mean(1) + _EPS)).float()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        # the output buffers and the workspace that a training program keeps from step to step
        from paper_2306_06446_amd import binding as sa
        T, n = case["T"], case.get("experts", 0)
        f32 = dict(dtype=torch.float32, device="cuda")
        s["sa"] = sa
        if case["kind"] == "norm":
            s["out"] = dict(y=torch.empty(T, case["E"], dtype=_TYPES[case["y"]], device="cuda"), mean=torch.empty(T, **f32),
                            rstd=torch.empty(T, **f32))
            if n:
                s["out"]["logits"] = torch.empty(T, n, **f32)
        elif case["kind"] == "norm_grad":
            E = case["E"]
            s["out"] = dict(dx=torch.empty_like(s["x"]))
            if case["weights"]:
                s["out"].update(dgamma=torch.empty(E, **f32), dbeta=torch.empty(E, **f32))
                if n:
                    s["out"].update(dwg=torch.empty(E, n, **f32), dbg=torch.empty(n, **f32))
                s["out"]["workspace"] = torch.empty(sa.sa_layernorm_backward_workspace_bytes(T, E, n), dtype=torch.uint8, device="cuda")
        elif case["kind"] == "balance":
            s["out"] = dict(losses=torch.empty(2, **f32), sums=torch.empty(2, n, **f32),
                            counts=torch.empty(n, dtype=torch.int32, device="cuda"), dlogits=torch.empty(T, n, **f32),
                            workspace=torch.empty(sa.sa_moe_balance_loss_grad_workspace_bytes(T, n), dtype=torch.uint8, device="cuda"))
        else:
            s["out"] = dict(dsrc=torch.empty_like(s["src"]), dgate=torch.empty(T, **f32), dlogits=torch.empty(T, n, **f32))
    return s


# ---------------------------------------------------------------------------------------- the passes --

def run(s):
    case = s["case"]
    if own:
        return _own[case["kind"]](s)
    return _plain[case["kind"]](s)


def _own_norm(s):
    y, mean, rstd, logits = s["sa"].sa_layernorm(s["x"], s["gamma"], s["beta"], _EPS, wg=s.get("wg"), bg=s.get("bg"), **s["out"])
    return [y, mean, rstd] + ([logits] if logits is not None else [])


def _own_norm_grad(s):
    case = s["case"]
    out = s["sa"].sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], _EPS, mean=s["mean"], rstd=s["rstd"],
                                        dres=s.get("dres"), dlogits=s.get("dlogits"), wg=s.get("wg"),
                                        want_params=case["weights"], **s["out"])
    return [t for t in out if t is not None]


def _own_balance(s):
    return list(s["sa"].sa_moe_balance_loss_grad(s["logits"], s["alpha"], s["case"]["noise_std"], s["dlosses"],
                                                 valid=s.get("valid"), **s["out"]))


def _own_combine_grad(s):
    return list(s["sa"].sa_combine_rows_backward(s["dy"], s["src"], rows=s["perm"], gate=s["gate"], logits=s["logits"], **s["out"]))


_own = dict(norm=_own_norm, norm_grad=_own_norm_grad, balance=_own_balance, combine_grad=_own_combine_grad)


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + _EPS)
    y = c * rstd[:, None] * s["gamma"] + s["beta"]
    out = [y.to(_TYPES[s["case"]["y"]]), mean, rstd]
    if "wg" in s:
        out.append(y @ s["wg"] + s["bg"])
    return out


def _plain_norm_grad(s):
    h = s["dy"].float()
    if "dlogits" in s:
        h = h + s["dlogits"] @ s["wg"].t()
    rstd = s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * rstd
    g = h * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if "dres" in s:
        dx = dx + s["dres"].float()
    out = [dx.to(s["x"].dtype)]
    if s["case"]["weights"]:
        out += [(h * xh).sum(0, dtype=torch.float64).float(), h.sum(0, dtype=torch.float64).float()]      # sums over all tokens
        if "dlogits" in s:
            y = xh * s["gamma"] + s["beta"]
            dl = s["dlogits"]
            out += [torch.stack([(y * dl[:, e:e + 1]).sum(0, dtype=torch.float64) for e in range(dl.shape[1])], 1).float(),
                    dl.sum(0, dtype=torch.float64).float()]
    return out


def _plain_balance(s):
    l, n, std = s["logits"], s["case"]["experts"], s["case"]["noise_std"]
    if "valid" in s:
        valid = s["valid"][:, None] != 0
        l = torch.where(valid, l, torch.zeros_like(l))
    e = torch.exp(l - l.max(1, keepdim=True).values)
    p = e / e.sum(1, keepdim=True)
    d, other, first = [], [], torch.zeros_like(l)
    for i in range(n):                                       # each expert's best competitor: by logits, ties to the lowest index
        best = None
        for j in range(n):
            if j == i:
                continue
            if best is None:
                best, at = l[:, j], torch.full_like(l[:, j], j, dtype=torch.int64)
            else:
                more = l[:, j] > best
                best, at = torch.where(more, l[:, j], best), torch.where(more, torch.full_like(at, j), at)
        d.append(p[:, i] - p.gather(1, at[:, None])[:, 0])
        other.append(at)
        first[:, i] = ((l[:, i] > best) | ((l[:, i] == best) & (at > i))).float()
    z = torch.stack(d, 1) / std
    q = 0.5 * torch.erfc(z * -math.sqrt(0.5))
    f = torch.exp(-0.5 * z * z) / (std * math.sqrt(2.0 * math.pi))
    if "valid" in s:
        p, q, f, first = [torch.where(valid, t, torch.zeros_like(t)) for t in (p, q, f, first)]
    losses, sums, a = [], [], []
    for kind, t in enumerate((p, q)):
        u = t.sum(0, dtype=torch.float64) * s["alpha"].double()      # long sums, and differences of nearly equal ones
        m = u.mean()
        losses.append(((u - m) ** 2).mean() / (m * m))
        sums.append(u)
        a.append((2.0 / (n * m * m) * (u - (u * u).sum() / u.sum()) * s["alpha"].double() * s["dlosses"][kind].double()).float())
    up = a[0].expand_as(p).clone()
    for i in range(n):
        t = a[1][i] * f[:, i]
        up[:, i] += t
        up.scatter_add_(1, other[i][:, None], -t[:, None])
    dl = p * (up - (p * up).sum(1, keepdim=True))
    counts = first.sum(0, dtype=torch.float64).to(torch.int32)
    return [torch.stack(losses).float(), torch.stack(sums).float(), counts, dl]


def _plain_combine_grad(s):
    perm = s["perm"].long()
    dy = s["dy"].float()[perm]
    dsrc = (dy * s["gate"][perm][:, None]).to(s["src"].dtype)
    dg = (dy * s["src"].float()).sum(1)
    dgate = torch.empty_like(s["gate"])
    dgate[perm] = dg
    l = s["logits"]
    e = torch.exp(l - l.max(1, keepdim=True).values)
    p = e / e.sum(1, keepdim=True)
    chosen = torch.zeros_like(l)
    best, at = l[:, 0], torch.zeros_like(perm)
    for j in range(1, l.shape[1]):
        more = l[:, j] > best
        best, at = torch.where(more, l[:, j], best), torch.where(more, torch.full_like(at, j), at)
    chosen.scatter_(1, at[:, None], 1.0)
    top = (p * chosen).sum(1, keepdim=True)
    return [dsrc, dgate, dgate[:, None] * top * (chosen - p)]


_plain = dict(norm=_plain_norm, norm_grad=_plain_norm_grad, balance=_plain_balance, combine_grad=_plain_combine_grad)


# ------------------------------------------------------------------------- the definitions in 64 bits --

def exact(case, seed):
    s = {k: v.double() if v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    kind = case["kind"]
    if kind == "norm":
        mean = s["x"].sum(1) / case["E"]
        dev = s["x"] - mean.unsqueeze(1)
        sd = ((dev ** 2).sum(1) / case["E"] + _EPS).sqrt()
        y = dev.div_(sd.unsqueeze(1)).mul_(s["gamma"]).add_(s["beta"])
        return [y, mean, 1.0 / sd] + ([y.matmul(s["wg"]) + s["bg"]] if "wg" in s else [])
    if kind == "norm_grad":
        xh = (s["x"] - s["mean"].unsqueeze(1)) * s["rstd"].unsqueeze(1)
        h = s["dy"]
        if "dlogits" in s:
            h = h + s["dlogits"].matmul(s["wg"].t().contiguous())
        out = [(h * xh).sum(0), h.sum(0)]
        if "dlogits" in s:
            out += [(xh * s["gamma"] + s["beta"]).t().contiguous().matmul(s["dlogits"]), s["dlogits"].sum(0)]
        if not case["weights"]:
            out = []
        h = h * s["gamma"]
        slope = (h * xh).sum(1, keepdim=True) / case["E"]
        dx = (h - h.sum(1, keepdim=True) / case["E"] - xh * slope) * s["rstd"].unsqueeze(1)
        return [dx + s["dres"] if "dres" in s else dx] + out
    if kind == "combine_grad":
        perm = s["perm"].long()
        expert_dy = s["dy"].index_select(0, perm)
        dgate = torch.zeros_like(s["gate"]).index_copy_(0, perm, (expert_dy * s["src"]).sum(1))
        l = s["logits"]
        p = torch.softmax(l, 1)
        index = torch.arange(l.shape[1], device=l.device)
        e = torch.where(l == l.amax(1, keepdim=True), index, l.shape[1]).amin(1)      # lowest index of the largest
        top = p.gather(1, e.unsqueeze(1))
        onehot = (index.unsqueeze(0) == e.unsqueeze(1)).double()
        return [expert_dy * s["gate"].index_select(0, perm).unsqueeze(1), dgate, dgate.unsqueeze(1) * top * (onehot - p)]
    # the loss, over the tokens that count, and its gradient term by term
    l, n, std = s["logits"], case["experts"], float(torch.tensor(case["noise_std"], dtype=torch.float32))
    keep = s["valid"] != 0 if "valid" in s else torch.ones(l.shape[0], dtype=torch.bool, device=l.device)
    l = l[keep]
    p = torch.softmax(l, 1)
    rank = torch.sort(l, dim=1, descending=True, stable=True).indices        # ties: the lowest index first
    first, second = rank[:, :1], rank[:, 1:2]
    index = torch.arange(n, device=l.device).unsqueeze(0)
    other = torch.where(index == first, second, first)
    z = (p - p.gather(1, other)) / std
    load = torch.special.ndtr(z)
    density = torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi) / std
    imp_u, load_u = s["alpha"] * p.sum(0), s["alpha"] * load.sum(0)
    losses, grads = [], []
    for w, u in zip(s["dlosses"], (imp_u, load_u)):
        mean = u.mean()
        var = ((u - mean) ** 2).mean()
        losses.append(var / mean ** 2)
        grads.append(w * s["alpha"] * (2 * (u - mean) / n / mean ** 2 - 2 * var / mean ** 3 / n))
    dp = grads[0] + grads[1] * density
    dp.scatter_add_(1, other, -(grads[1] * density))
    dl = torch.zeros_like(s["logits"])
    dl[keep] = p * (dp - (dp * p).sum(1, keepdim=True))
    counts = torch.bincount(first[:, 0], minlength=n).to(torch.int32)
    return [torch.stack(losses), torch.stack((imp_u, load_u)), counts, dl]
