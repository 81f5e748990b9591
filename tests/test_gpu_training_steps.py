"""LayerNorm of training and its gradient over many rows, on the GPU against their formulas in 64 bits (there as well): rows whose
statistics and logits stay in lanes for several steps before they leave, sums over parts of several rows.

How far sums over rows may be off: a part's rows are added up one by one in fp32, at most 65 of them here (33001 rows in 508 parts), a
workgroup's sums of up to 64 groups of lanes one by one as well, the up to 512 parts in fp64.  That is less than training_forms.D additions."""
import pytest
import torch

import training_forms as tf
from test_gpu_layernorm_train import BF16, EPS, F16, F32, inputs

pytestmark = pytest.mark.gpu


def check(got, want, off, dtype, what):
    lim = off + tf.rounding(want.abs() + off, dtype)
    err = (got.double() - want).abs()
    assert got.shape == want.shape and bool((err <= lim).all()), \
        "%s: off by %g where %g is allowed" % (what, float(err.max()), float(lim.flatten()[(err - lim).argmax()]))


def doubles(s, *names):
    return [None if s.get(k) is None else s[k].double() for k in names]


def forward(sa, s, yt):
    y, mean, rstd, logits = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, y_dtype=yt, wg=s.get("wg"), bg=s.get("bg"))
    for t0 in range(0, y.shape[0], 16384):                   # the 64-bit forms of some rows at a time
        rows = slice(t0, t0 + 16384)
        x, gamma, beta, wg, bg = [t[rows] if k == 0 else t for k, t in enumerate(doubles(s, "x", "gamma", "beta", "wg", "bg"))]
        want, off = tf.norm(x, gamma, beta, EPS, wg, bg), tf.norm_off(x, gamma, beta, EPS, wg)
        for got, w, o, dtype, what in zip((y, mean, rstd, logits), want, off, (yt, F32, F32, F32), ("y", "mean", "rstd", "logits")):
            if got is not None:
                check(got[rows], w, o, dtype, what)
    return mean, rstd


def backward(sa, s, mean, rstd, n, stats, **kw):
    got = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, mean=mean if stats else None, rstd=rstd if stats else None,
                                   dres=s["dres"], dlogits=s.get("dlogits"), wg=s.get("wg"), **kw)
    dy, x, gamma, beta, dres, dlogits, wg = doubles(s, "dy", "x", "gamma", "beta", "dres", "dlogits", "wg")
    mean, rstd = (mean.double(), rstd.double()) if stats else tf.norm(x, gamma, beta, EPS)[1:3]
    args = (dy, x, gamma, beta, mean, rstd, dres, dlogits, wg)
    for name, g, w, e in zip(("dx", "dgamma", "dbeta", "dwg", "dbg"), got, tf.norm_grad(*args), tf.norm_grad_off(*args, stats_given=stats)):
        check(g, w, e, g.dtype, name)


# A step of the launch is 16384 rows of up to 64 elements, 8192 of up to 128, 4096 of up to 256, 1024 of 4100; behind many experts 8192 of
# 33 elements, 2048 of 300 and 768, 512 of 2049 and 256 of 5000.  Of 16, 32 or 64 steps (8 of many experts and whole wavefronts) the statistics
# leave together: whole periods, one row more, and a last step that is not full.
@pytest.mark.parametrize("E,T", [(8, 300001), (8, 262144), (8, 262145), (3, 262143), (60, 278528), (100, 262221), (200, 262144), (200, 270337)])
@pytest.mark.parametrize("n", [0, 2])
def test_rows_of_many_steps(sa, E, T, n):
    forward(sa, inputs(T, E, F32, F32, n, T), F32)


@pytest.mark.parametrize("xt,yt", [(F32, F16), (BF16, BF16)], ids=str)
@pytest.mark.parametrize("n", [3, 5, 8])
@pytest.mark.parametrize("E,T", [(33, 140001), (300, 36865), (768, 20000), (768, 32768), (2049, 9001), (2049, 4096), (5000, 4099), (5000, 2047)])
def test_rows_of_many_steps_with_many_experts(sa, xt, yt, E, T, n):
    forward(sa, inputs(T, E, xt, yt, n, T + n), yt)


def test_wide_rows_of_more_steps_than_a_wavefront_has_lanes(sa):
    forward(sa, inputs(65545, 4100, BF16, BF16, 2, 1), BF16)


@pytest.mark.parametrize("stats", [True, False])
@pytest.mark.parametrize("xt,yt", [(F32, F32), (F32, BF16), (F16, F16)], ids=str)
@pytest.mark.parametrize("n,E,T", [(5, 33, 40001), (5, 250, 5003), (8, 250, 9000), (5, 768, 4099), (8, 768, 12608), (3, 1500, 3001), (8, 1500, 6007)])
def test_sums_over_rows_behind_many_experts(sa, xt, yt, n, E, T, stats):
    s = inputs(T, E, xt, yt, n, E + n)
    mean, rstd = forward(sa, s, yt)
    backward(sa, s, mean, rstd, n, stats)


@pytest.mark.parametrize("stats", [True, False])
@pytest.mark.parametrize("xt,yt", [(F32, F16), (BF16, BF16)], ids=str)
@pytest.mark.parametrize("n,E,T", [(3, 2049, 1500), (8, 2049, 1501), (3, 4100, 1499), (8, 4100, 1500), (3, 8191, 700), (3, 2049, 33001)])
def test_sums_over_rows_of_wide_rows_behind_many_experts(sa, xt, yt, n, E, T, stats):
    s = inputs(T, E, xt, yt, n, E + n)
    mean, rstd = forward(sa, s, yt)
    backward(sa, s, mean, rstd, n, stats)


def test_statistics_beyond_32_bits_of_elements(sa):
    forward(sa, inputs(270001, 8192, BF16, BF16, 2, 2), BF16)        # 2.2e9 of them


@pytest.mark.parametrize("T", [(1 << 28) + 5, (1 << 23) + 77, 40000])
def test_sums_over_very_many_rows_of_one_sign(sa, T):
    """As a loss that is a plain sum has them: what a row adds is small against what there is, and rounded the same way again and again.  A lane
    adds up 512 rows in fp32 at most, a workgroup's 64 groups of lanes follow, the parts are fp64."""
    f = lambda *v: torch.tensor(v, device="cuda")      # noqa: E731
    x, dy, dl = f(1.0, -1.0).repeat(T, 1), torch.full((T, 2), 0.1, device="cuda"), torch.full((T, 2), 0.3, device="cuda")
    gamma, beta = f(1.0, 2.0), f(0.5, -3.0)
    _, dgamma, dbeta, dwg, dbg = sa.sa_layernorm_backward(dy, x, gamma, beta, EPS, dlogits=dl, wg=torch.zeros(2, 2, device="cuda"))
    c, d = float(dy[0, 0]), float(dl[0, 0])
    xh = f(1.0, -1.0).double() / (1.0 + EPS) ** 0.5
    y = gamma.double() * xh + beta.double()
    size = (gamma.double() * xh).abs() + beta.double().abs()             # both parts of y by themselves
    bound = (512 + 64 + 8) * tf.U * T                       # and what makes a row's summands: xh, two products, the output
    for got, want, of in ((dgamma, T * c * xh, c * xh.abs()), (dbeta, T * c * torch.ones_like(xh), c * torch.ones_like(xh)),
                          (dwg, (T * d * y)[:, None].repeat(1, 2), (d * size)[:, None].repeat(1, 2)),
                          (dbg, T * d * torch.ones_like(xh), d * torch.ones_like(xh))):
        err = (got.double() - want).abs()
        assert bool((err <= bound * of).all()), (err / want.abs() / tf.U)


@pytest.mark.parametrize("xt,yt,E,n,T", [(BF16, BF16, 2049, 3, 300000), (F16, F16, 2051, 0, 300000), (F32, BF16, 1026, 2, 530000)], ids=str)
def test_sums_over_more_rows_than_parts_of_512(sa, xt, yt, E, n, T):
    s = inputs(T, E, xt, yt, n, 3)
    need = sa.sa_layernorm_backward_workspace_bytes(T, E, n)
    ws = torch.full((need + 1024,), 7, dtype=torch.uint8, device="cuda")
    backward(sa, s, *sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS)[1:3], n, True, workspace=ws[:need])
    assert bool((ws[need:] == 7).all())
