"""LayerNorm of training and its gradient on the GPU against their formulas in 64 bits."""
import pytest
import torch

import training_forms as tf

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
PAIRS = [(F32, F32), (F32, F16), (F32, BF16), (F16, F16), (BF16, BF16)]
EPS = 1e-6


def check(got, want, off, dtype=None, what=""):
    """|got - want| <= off, with one rounding to dtype more."""
    lim = off if dtype is None else off + tf.rounding(want.abs() + off, dtype)
    err = (tf.f64(got) - want).abs()
    assert got.shape == want.shape and bool((err <= lim).all()), \
        "%s: off by %g where %g is allowed" % (what, float(err.max()), float(lim.flatten()[(err - lim).argmax()]))


def inputs(T, E, xt, yt, n, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
    s = dict(x=(r(T, E) * torch.exp(0.5 * r(T, 1)) + r(T, 1)).to(xt), gamma=1 + 0.2 * r(E), beta=0.3 * r(E), dy=r(T, E).to(yt),
             dres=r(T, E).to(xt))
    if n:
        s.update(wg=r(E, n) / E ** 0.5, bg=r(n), dlogits=r(T, n))
    return s


def run_forward(sa, s, yt, n):
    y, mean, rstd, logits = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, y_dtype=yt, wg=s.get("wg"), bg=s.get("bg"))
    x, gamma, beta, wg, bg = [tf.f64(s.get(k)) for k in ("x", "gamma", "beta", "wg", "bg")]
    want = tf.norm(x, gamma, beta, EPS, wg, bg)
    off = tf.norm_off(x, gamma, beta, EPS, wg)
    assert y.dtype == yt
    check(y, want[0], off[0], yt, "y")
    check(mean, want[1], off[1], None, "mean")
    check(rstd, want[2], off[2], F32, "rstd")
    if n:
        check(logits, want[3], off[3], None, "logits")
    return mean, rstd


def run_backward(sa, s, mean, rstd, n, residual, stats=True, **kw):
    dl = s["dlogits"] if n else None
    got = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, mean=mean if stats else None, rstd=rstd if stats else None,
                                   dres=s["dres"] if residual else None, dlogits=dl, wg=s["wg"] if n else None, **kw)
    check_backward(got, s, mean, rstd, n, residual, stats)
    return got


def check_backward(got, s, mean, rstd, n, residual, stats=True, xt=None):
    args = [tf.f64(s[k]) for k in ("dy", "x", "gamma", "beta")] + [tf.f64(mean), tf.f64(rstd)]
    if not stats:
        args[4:] = tf.norm(args[1], args[2], args[3], EPS)[1:3]
    args += [tf.f64(s["dres"]) if residual else None] + ([tf.f64(s["dlogits"]), tf.f64(s["wg"])] if n else [None, None])
    want, off = tf.norm_grad(*args), tf.norm_grad_off(*args, stats_given=stats)
    for name, g, w, e in zip(("dx", "dgamma", "dbeta", "dwg", "dbg"), got, want, off):
        if g is not None:
            check(g, w, e, got[0].dtype if name == "dx" else F32, name)
    assert got[0].dtype == s["x"].dtype


# every width at which another kernel, a partial vector or a partial wavefront begins
WIDTHS = [1, 2, 3, 7, 8, 9, 60, 64, 65, 127, 128, 129, 192, 250, 256, 257, 500, 511, 512, 513, 768, 1000, 1001, 1024, 1025, 1536, 1537,
          2000, 2047, 2048, 2049, 2560, 4095, 4096, 4097, 5000, 8189, 8191, 8192]


@pytest.mark.parametrize("n", [0, 2, 5])
@pytest.mark.parametrize("xt,yt", PAIRS, ids=str)
def test_every_width(sa, xt, yt, n):
    for i, E in enumerate(WIDTHS):
        T = (1, 2, 5, 67)[i % 4] if E > 2 else 67
        s = inputs(T, E, xt, yt, n, E)
        mean, rstd = run_forward(sa, s, yt, n)
        run_backward(sa, s, mean, rstd, n, residual=i % 3 != 0, stats=i % 2 == 0)


@pytest.mark.parametrize("T", [1, 2, 3, 15, 16, 17, 63, 64, 65, 197, 1023, 1025, 4099, 12608])
@pytest.mark.parametrize("xt,yt,E,n", [(F32, F16, 96, 2), (BF16, BF16, 200, 0), (F16, F16, 33, 8), (F32, F32, 1028, 2)], ids=str)
def test_numbers_of_rows(sa, T, xt, yt, E, n):
    s = inputs(T, E, xt, yt, n, T)
    mean, rstd = run_forward(sa, s, yt, n)
    run_backward(sa, s, mean, rstd, n, residual=True, stats=T % 2 == 0)


def test_wide_rows_many(sa):
    s = inputs(1500, 5000, BF16, BF16, 2, 3)
    mean, rstd = run_forward(sa, s, BF16, 2)
    run_backward(sa, s, mean, rstd, 2, True)


@pytest.mark.parametrize("offset,scale", [(1000.0, 1.0), (0.0, 1e-4), (-3.0, 1e4), (5.0, 0.0)])
@pytest.mark.parametrize("E", [96, 2048])
def test_rows_far_from_zero_tiny_large_and_constant(sa, offset, scale, E):
    s = inputs(33, E, F32, F32, 0, 5)
    s["x"] = torch.randn(33, E, device="cuda") * scale + offset
    mean, rstd = run_forward(sa, s, F32, 0)
    run_backward(sa, s, mean, rstd, 0, True)


@pytest.mark.parametrize("E", [64, 700, 4100])
def test_a_row_that_is_not_finite_stays_alone(sa, E):
    s = inputs(20, E, F32, BF16, 2, 9)
    clean = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, y_dtype=BF16, wg=s["wg"], bg=s["bg"])
    grad = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, mean=clean[1], rstd=clean[2], dlogits=s["dlogits"], wg=s["wg"])
    s["x"][7, 3], s["x"][11, E - 1] = float("nan"), float("inf")
    got = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, y_dtype=BF16, wg=s["wg"], bg=s["bg"])
    dx = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, dlogits=s["dlogits"], wg=s["wg"], want_params=False)[0]
    rest = [t for t in range(20) if t not in (7, 11)]
    for g, c in zip(got, clean):
        assert torch.equal(g[rest], c[rest]) and bool(g[7].isnan().all()) and not bool(g[11].isfinite().all())      # the mean of an infinite row is infinite
    assert torch.equal(dx[rest], grad[0][rest]) and bool(dx[[7, 11]].isnan().all())


@pytest.mark.parametrize("E,n", [(60, 2), (1001, 2), (4096, 2), (100, 5), (1500, 8), (2500, 3), (8190, 8)])
def test_outputs_on_request_and_the_same_bits_again(sa, E, n):
    s = inputs(70, E, F32, F16, n, 4)
    y, mean, rstd, logits = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, y_dtype=F16, wg=s["wg"], bg=s["bg"])
    again = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, y_dtype=F16, want_stats=False)
    assert torch.equal(again[0], y) and again[1:] == (None, None, None)
    again = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, want_y=False, wg=s["wg"], bg=s["bg"])
    assert again[0] is None and torch.equal(again[1], mean) and torch.equal(again[2], rstd) and torch.equal(again[3], logits)
    kw = dict(mean=mean, rstd=rstd, dres=s["dres"], dlogits=s["dlogits"], wg=s["wg"])
    first = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, **kw)
    for g, f in zip(sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, **kw), first):
        assert torch.equal(g, f)
    frozen = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, want_params=False, **kw)
    assert torch.equal(frozen[0], first[0]) and frozen[1:] == (None,) * 4


@pytest.mark.parametrize("E,n", [(192, 2), (1003, 4), (5000, 0)])
def test_parameter_gradients_accumulate(sa, E, n):
    s = inputs(300, E, F32, F32, n, 6)
    mean, rstd = run_forward(sa, s, F32, n)
    once = run_backward(sa, s, mean, rstd, n, False)
    names = ("dgamma", "dbeta", "dwg", "dbg")[:4 if n else 2]
    held = {k: torch.randn_like(g) for k, g in zip(names, once[1:])}
    want = {k: held[k] + g for k, g in zip(names, once[1:])}
    kw = dict(mean=mean, rstd=rstd, dlogits=s.get("dlogits"), wg=s.get("wg"), accumulate=True, **held)
    got = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, **kw)
    for k, g in zip(names, got[1:]):
        assert g is held[k] and torch.equal(g, want[k])
    none = {k: torch.full_like(v, 7.0) for k, v in held.items()}
    empty = {k: s[k][:0] for k in ("dy", "x")}
    kw = dict(mean=mean[:0], rstd=rstd[:0], dlogits=s["dlogits"][:0] if n else None, wg=s.get("wg"), **none)
    sa.sa_layernorm_backward(empty["dy"], empty["x"], s["gamma"], s["beta"], EPS, accumulate=True, **kw)
    assert all(bool((v == 7.0).all()) for v in none.values())
    sa.sa_layernorm_backward(empty["dy"], empty["x"], s["gamma"], s["beta"], EPS, **kw)
    assert all(bool((v == 0.0).all()) for v in none.values())
    assert sa.sa_layernorm(empty["x"], s["gamma"], s["beta"], EPS)[0].shape == (0, E)


@pytest.mark.parametrize("E", [100, 1001, 4100, 8192])
@pytest.mark.parametrize("place", ["dres", "dy", "x"])
def test_dx_takes_the_place_of_what_it_is_made_of(sa, E, place):
    s = inputs(50, E, F32, F32, 2, 8)
    mean, rstd = run_forward(sa, s, F32, 2)
    kept = {k: v.clone() for k, v in s.items()}
    got = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, mean=mean, rstd=rstd, dres=s["dres"], dlogits=s["dlogits"],
                                   wg=s["wg"], dx=s[place])
    check_backward(got, kept, mean, rstd, 2, True)
    y = sa.sa_layernorm(kept["x"], s["gamma"], s["beta"], EPS, y=kept["x"].clone())[0]
    x = kept["x"].clone()
    assert torch.equal(sa.sa_layernorm(x, s["gamma"], s["beta"], EPS, y=x)[0], y)


@pytest.mark.parametrize("xt,T,E", [(F32, 1500, 5001), (BF16, 2000, 2061), (F16, 3000, 1030), (BF16, 700, 8189), (F32, 4000, 333), (F16, 900, 4100)], ids=str)
@pytest.mark.parametrize("n", [0, 2, 3])
def test_in_place_gives_the_same_bits(sa, xt, T, E, n):
    """Elements at a row's end are computed by two lanes, of wide rows in two wavefronts: both from what was there before."""
    s = inputs(T, E, xt, xt, n, 21)
    y, mean, rstd, _ = sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS)
    x = s["x"].clone()
    assert torch.equal(sa.sa_layernorm(x, s["gamma"], s["beta"], EPS, y=x)[0], y)
    for stats in (True, False):
        kw = dict(mean=mean if stats else None, rstd=rstd if stats else None, dlogits=s.get("dlogits"), wg=s.get("wg"))
        want = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, dres=s["dres"], **kw)
        for place in ("dres", "dy", "x"):
            t = {k: s[k].clone() for k in ("dres", "dy", "x")}
            got = sa.sa_layernorm_backward(t["dy"], t["x"], s["gamma"], s["beta"], EPS, dres=t["dres"], dx=t[place], **kw)
            assert got[0] is t[place]
            for g, w in zip(got, want):
                assert (g is None and w is None) or torch.equal(g, w), place


@pytest.mark.parametrize("T,E,xt,yt", [(3, 5, BF16, BF16), (33, 1001, F16, F16), (70, 4099, F32, BF16), (9, 130, F32, F32)], ids=str)
def test_nothing_is_written_behind_the_outputs(sa, T, E, xt, yt):
    n, s = 3, inputs(T, E, xt, yt, 3, 2)

    def room(*shape, dtype=F32):
        count = 1
        for k in shape:
            count *= k
        whole = torch.full((count + 64,), 7.0, dtype=dtype, device="cuda")
        return whole, whole[:count].view(shape)

    rooms = dict(y=room(T, E, dtype=yt), mean=room(T), rstd=room(T), logits=room(T, n))
    out = {k: v[1] for k, v in rooms.items()}
    sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, wg=s["wg"], bg=s["bg"], **out)
    back = dict(dx=room(T, E, dtype=xt), dgamma=room(E), dbeta=room(E), dwg=room(E, n), dbg=room(n))
    need = sa.sa_layernorm_backward_workspace_bytes(T, E, n)
    ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    got = sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, mean=out["mean"], rstd=out["rstd"], dres=s["dres"],
                                   dlogits=s["dlogits"], wg=s["wg"], workspace=ws[:need], **{k: v[1] for k, v in back.items()})
    check_backward(got, s, out["mean"], out["rstd"], n, True)
    for whole, part in list(rooms.values()) + list(back.values()):
        assert bool((whole[part.numel():] == 7.0).all())
    assert bool((ws[need:] == 7).all())


def test_offsets_beyond_32_bits(sa):
    T, E = 270001, 8192                     # 2.2e9 elements
    x = torch.empty(T, E, dtype=BF16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    dy = torch.empty_like(x).normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    gamma, beta = torch.ones(E, device="cuda"), torch.zeros(E, device="cuda")
    y, mean, rstd, _ = sa.sa_layernorm(x, gamma, beta, EPS)
    dx, dgamma, dbeta, _, _ = sa.sa_layernorm_backward(dy, x, gamma, beta, EPS, mean=mean, rstd=rstd)
    for rows in (slice(0, 3), slice(131071, 131074), slice(262143, 262146), slice(T - 3, T)):
        a = [tf.f64(t) for t in (x[rows], gamma, beta)]
        check(y[rows], tf.norm(*a, EPS)[0], tf.norm_off(*a, EPS)[0], BF16, "y")
        b = [tf.f64(t) for t in (dy[rows], x[rows], gamma, beta, mean[rows], rstd[rows])]
        check(dx[rows], tf.norm_grad(*b)[0], tf.norm_grad_off(*b)[0], BF16, "dx")
    total = sum(dy[i:i + 30000].double().sum(0) for i in range(0, T, 30000))
    size = sum(dy[i:i + 30000].double().abs().sum(0) for i in range(0, T, 30000))
    # ranges of 64 + T / 256 rows, and 256 of them: 1400 additions in a row at most
    assert bool(((dbeta.double() - total).abs() <= 1400 * tf.U * size).all())


@pytest.mark.parametrize("E,n", [(192, 2), (2500, 0)])
def test_another_stream_and_replays_of_a_graph(sa, E, n):
    s = inputs(197, E, F32, F16, n, 12)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        mean, rstd = run_forward(sa, s, F16, n)
        eager = run_backward(sa, s, mean, rstd, n, True)
    torch.cuda.current_stream().wait_stream(stream)
    out = {k: torch.empty_like(v) for k, v in zip(("dx", "dgamma", "dbeta", "dwg", "dbg"), eager) if v is not None}
    ws = torch.empty(sa.sa_layernorm_backward_workspace_bytes(197, E, n), dtype=torch.uint8, device="cuda")
    y, fm, fr = torch.empty(197, E, dtype=F16, device="cuda"), torch.empty_like(mean), torch.empty_like(rstd)
    logits = torch.empty(197, n, device="cuda") if n else None

    def step():
        sa.sa_layernorm(s["x"], s["gamma"], s["beta"], EPS, y=y, mean=fm, rstd=fr, wg=s.get("wg"), bg=s.get("bg"), logits=logits)
        sa.sa_layernorm_backward(s["dy"], s["x"], s["gamma"], s["beta"], EPS, mean=fm, rstd=fr, dres=s["dres"], dlogits=s.get("dlogits"),
                                 wg=s.get("wg"), workspace=ws, **out)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        s["x"].copy_(inputs(197, E, F32, F16, n, 30 + k)["x"])
        for t in out.values():
            t.fill_(-1.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in out.values()] + [y.clone()]
        step()
        assert all(torch.equal(a, b) for a, b in zip(replayed, list(out.values()) + [y]))
        check_backward([out.get(k) for k in ("dx", "dgamma", "dbeta", "dwg", "dbg")], s, fm, fr, n, True)


def test_binding_refuses_wrong_shapes_types_and_orders(sa):
    s = inputs(8, 32, F32, F16, 2, 1)
    mean, rstd = torch.zeros(8, device="cuda"), torch.ones(8, device="cuda")
    back = lambda **kw: sa.sa_layernorm_backward(**{**dict(dy=s["dy"], x=s["x"], gamma=s["gamma"], beta=s["beta"], eps=EPS, mean=mean,      # noqa: E731
                                                           rstd=rstd, dres=s["dres"], dlogits=s["dlogits"], wg=s["wg"]), **kw})
    back()
    for bad in (dict(dy=s["dy"][:7]), dict(dy=s["dy"].double()), dict(gamma=s["gamma"][:31]), dict(mean=mean[:7]), dict(dres=s["dres"].half()),
                dict(dres=s["dres"].t()), dict(dlogits=s["dlogits"][:, :1]), dict(wg=s["wg"].t().contiguous()), dict(x=s["x"].cpu()),
                dict(dx=torch.empty(8, 33, device="cuda")), dict(accumulate=True), dict(want_params=False, dgamma=s["gamma"]),
                dict(gamma=s["gamma"].cpu()), dict(x=s["x"].double())):
        with pytest.raises((ValueError, sa.SAError)):
            back(**bad)
    for bad in (dict(y=torch.empty(8, 33, device="cuda")), dict(mean=mean.half()), dict(wg=s["wg"][:31], bg=s["bg"]), dict(wg=s["wg"]),
                dict(beta=s["beta"].half())):
        with pytest.raises((ValueError, sa.SAError)):
            sa.sa_layernorm(**{**dict(x=s["x"], gamma=s["gamma"], beta=s["beta"], eps=EPS), **bad})
