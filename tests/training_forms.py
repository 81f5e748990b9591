"""The training operators in 64 bits, from their formulas (plain torch on the CPU), and how far a kernel in 32 bits may be off.

U is half a step of fp32.  A sum that the kernels take in D additions in a row (the rest in a tree) is off by at most
D * U * (sum of magnitudes); D = 512 covers every sum of these tests: a row of 8192 elements is 128 elements to a lane or fewer, and
columns are summed over ranges of rows that are summed again, at most 256 ranges of at most 64 + T / 256 rows each.
"""
import math

import torch

U = 2.0 ** -24
D = 512
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}      # half a subnormal step


def f64(t):
    return None if t is None else t.detach().double().cpu()


def rounding(t, dtype):
    """One rounding of t to dtype (fp32 results of the last operation included)."""
    return HALF_STEP[dtype] * t.abs() + SMALLEST[dtype]


# ------------------------------------------------------------------------------------------- LayerNorm --

def norm(x, gamma, beta, eps, wg=None, bg=None):
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None] * gamma + beta
    return y, mean, rstd, (None if wg is None else y @ wg + bg)


def stats_off(x, mean, rstd):
    """Errors of mean, of rstd and of xh where a kernel computes both from x in 32 bits."""
    d_mean = D * U * x.abs().mean(1)
    c = (x - mean[:, None]).abs()
    # the centred squares have their own roundings and the error of the mean in first order: 2 c d_mean, whose sum over a row is 0
    # but for roundings; d_mean^2 is what is left of it
    d_rstd = rstd * ((D / 2 + 4) * U + 0.5 * rstd ** 2 * d_mean ** 2)
    d_xh = rstd[:, None] * (d_mean[:, None] + 2 * U * c) + c * d_rstd[:, None]
    return d_mean + U * mean.abs(), d_rstd, d_xh


def norm_off(x, gamma, beta, eps, wg=None):
    y, mean, rstd, _ = norm(x, gamma, beta, eps)
    d_mean, d_rstd, d_xh = stats_off(x, mean, rstd)
    d_y = gamma.abs() * d_xh + 2 * U * ((y - beta).abs() + y.abs() + beta.abs())
    d_logits = None
    if wg is not None:
        d_logits = d_y @ wg.abs() + (D + 2) * U * (y.abs() @ wg.abs() + 1.0)
    return d_y, d_mean, d_rstd, d_logits


def norm_grad(dy, x, gamma, beta, mean, rstd, dres=None, dlogits=None, wg=None):
    h = dy if dlogits is None else dy + dlogits @ wg.T
    xh = (x - mean[:, None]) * rstd[:, None]
    g = h * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if dres is not None:
        dx = dx + dres
    out = [dx, (h * xh).sum(0), h.sum(0)]
    if dlogits is not None:
        out += [(xh * gamma + beta).T @ dlogits, dlogits.sum(0)]
    return out


def norm_grad_off(dy, x, gamma, beta, mean, rstd, dres=None, dlogits=None, wg=None, stats_given=True):
    """Errors of what norm_grad returns, before an output's own rounding."""
    size = dy.abs() if dlogits is None else dy.abs() + dlogits.abs() @ wg.abs().T
    h = dy if dlogits is None else dy + dlogits @ wg.T
    e_h = 9 * U * size if dlogits is not None else torch.zeros_like(dy)
    xh = (x - mean[:, None]) * rstd[:, None]
    e_xh, e_rstd = 3 * U * xh.abs(), torch.zeros_like(rstd)
    if not stats_given:
        _, e_rstd, e = stats_off(x, mean, rstd)
        e_xh = e_xh + e
    g = h * gamma
    e_g = e_h * gamma.abs() + U * g.abs()
    c0, c1 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    e_c0 = e_g.mean(1, keepdim=True) + D * U * g.abs().mean(1, keepdim=True)
    e_gx = e_g * xh.abs() + e_xh * g.abs()
    e_c1 = e_gx.mean(1, keepdim=True) + D * U * (g * xh).abs().mean(1, keepdim=True)
    inner = g.abs() + c0.abs() + (xh * c1).abs()
    r = rstd[:, None]
    e_dx = r * (e_g + e_c0 + xh.abs() * e_c1 + e_xh * c1.abs() + 4 * U * inner) + inner * (e_rstd[:, None] + U * r)
    if dres is not None:
        e_dx = e_dx + U * dres.abs()
    out = [e_dx, (e_h * xh.abs() + e_xh * h.abs()).sum(0) + D * U * (h * xh).abs().sum(0), e_h.sum(0) + D * U * h.abs().sum(0)]
    if dlogits is not None:
        y = (xh * gamma).abs() + beta.abs()
        out += [(e_xh * gamma.abs() + 2 * U * y).T @ dlogits.abs() + D * U * (y.T @ dlogits.abs()), D * U * dlogits.abs().sum(0)]
    return out


# --------------------------------------------------------------------------- balance loss and combine --

def ranks(logits):
    """First and second choice of each token, ties to the lowest index."""
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices
    return order[:, 0], order[:, 1]


def others(logits):
    first, second = ranks(logits)
    index = torch.arange(logits.shape[1])
    return torch.where(index[None, :] == first[:, None], second[:, None], first[:, None])


def balance_losses(logits, alpha, std):
    """Differentiable form on the tokens that count: losses, sums, and what the gradient is made of."""
    p = torch.softmax(logits, 1)
    z = (p - p.gather(1, others(logits))) / std
    q = 0.5 * torch.erfc(-z / math.sqrt(2.0))
    sums = torch.stack((alpha * p.sum(0), alpha * q.sum(0)))
    mean = sums.mean(1, keepdim=True)
    losses = ((sums - mean) ** 2).mean(1) / mean[:, 0] ** 2
    return losses, sums, p, z


def balance(logits, alpha, std, dlosses, valid=None):
    T, n = logits.shape
    keep = torch.ones(T, dtype=torch.bool) if valid is None else valid.bool()
    l = logits[keep]
    dl = torch.zeros_like(logits)
    if l.shape[0] == 0:
        return torch.zeros(2, dtype=l.dtype), torch.zeros(2, n, dtype=l.dtype), torch.zeros(n, dtype=torch.int64), dl
    losses, sums, p, z = balance_losses(l, alpha, std)
    mean = sums.mean(1, keepdim=True)
    c = 2.0 / (n * mean ** 2) * (sums - (sums ** 2).sum(1, keepdim=True) / sums.sum(1, keepdim=True)) * alpha * dlosses[:, None]
    f = c[1] * torch.exp(-0.5 * z * z) / (std * math.sqrt(2 * math.pi))
    a = (c[0] + f).scatter_add(1, others(l), -f)
    dl[keep] = p * (a - (p * a).sum(1, keepdim=True))
    return losses, sums, torch.bincount(ranks(l)[0], minlength=n), dl


def balance_off(logits, alpha, std, dlosses, valid=None):
    """Errors of losses, sums and dlogits.  A probability is off by its exponent's rounding, exp's own 2 units and a few more."""
    T, n = logits.shape
    keep = torch.ones(T, dtype=torch.bool) if valid is None else valid.bool()
    l = logits[keep]
    out = torch.zeros_like(logits)
    if l.shape[0] == 0:
        return torch.zeros(2), torch.zeros(2, n), out
    losses, sums, p, z = balance_losses(l, alpha, std)
    gap = (l - l.max(1, keepdim=True).values).abs()
    gap = torch.where(gap.isfinite(), gap, torch.zeros_like(gap))
    e_p = p * U * (gap + (p * gap).sum(1, keepdim=True) + n + 10)
    e_z = (e_p + e_p.gather(1, others(l))) / std + 3 * U * z.abs()
    e_q = 0.4 * e_z + 4 * U
    e_sums = torch.stack((alpha * e_p.sum(0), alpha * e_q.sum(0)))
    mean = sums.mean(1, keepdim=True)
    slope = 2.0 / (n * mean ** 2) * (sums - (sums ** 2).sum(1, keepdim=True) / sums.sum(1, keepdim=True))
    e_losses = (slope.abs() * e_sums).sum(1) + 4 * (e_sums / mean).max(1).values ** 2 + 4 * U * losses
    e_c = alpha * dlosses.abs()[:, None] * (2.0 / (n * mean ** 2)) * (1.0 + n * losses[:, None].sqrt()) * 4 * e_sums.max(1, keepdim=True).values
    c = slope.abs() * alpha * dlosses.abs()[:, None]
    e_c = e_c + 4 * U * c
    peak = torch.exp(-0.5 * z * z) / (std * math.sqrt(2 * math.pi))
    e_f = e_c[1] * peak + c[1] * (0.61 * e_z + 8 * U) / (std * math.sqrt(2 * math.pi))
    f = c[1] * peak
    a = c[0] + f + f.sum(1, keepdim=True)
    e_a = e_c[0] + e_f + e_f.sum(1, keepdim=True) + (n + 2) * U * a
    both = a + (p * a).sum(1, keepdim=True)
    e_mean = (p * e_a + e_p * a).sum(1, keepdim=True) + n * U * (p * a).sum(1, keepdim=True)
    out[keep] = p * (e_a + e_mean) + e_p * both + 4 * U * p * both
    return e_losses, e_sums + 2 * U * sums, out


def combine_grad(dy, src, rows, gate, logits):
    """Of selected rows `rows`: dsrc, dgate and dlogits of those rows."""
    d = dy[rows]
    dgate = (d * src).sum(1)
    l = logits[rows]
    p = torch.softmax(l, 1)
    e = ranks(l)[0]
    chosen = torch.nn.functional.one_hot(e, l.shape[1]).to(p.dtype)
    top = (p * chosen).sum(1, keepdim=True)
    return d * gate[rows][:, None], dgate, dgate[:, None] * top * (chosen - p)


def combine_grad_off(dy, src, rows, gate, logits):
    d = dy[rows]
    dsrc, dgate, dl = combine_grad(dy, src, rows, gate, logits)
    e_gate = D * U * (d * src).abs().sum(1)
    l = logits[rows]
    p = torch.softmax(l, 1)
    gap = (l - l.max(1, keepdim=True).values).abs()
    gap = torch.where(gap.isfinite(), gap, torch.zeros_like(gap))
    rel = U * (gap.max(1, keepdim=True).values + l.shape[1] + 10)
    top = p.max(1, keepdim=True).values
    # (k == e) - p_k of a sure token: p itself is known to `rel` only
    return U * dsrc.abs(), e_gate, e_gate[:, None] * top * 1.0 + dgate.abs()[:, None] * top * (rel + 3 * rel * p) + 4 * U * dl.abs()
