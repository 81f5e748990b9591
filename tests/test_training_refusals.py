"""What the training operators refuse, each with its own code and before anything is launched (on a host without a GPU a launch comes
back as SA_ERR_HIP), and what the binding refuses before it calls the library."""
import ctypes

import pytest
import torch

from paper_2306_06446_amd import binding

FAKE, ODD = 0x1000, 0x1004
OK, INVALID, SHAPE, ALIGN, WORKSPACE, HIP, UNSUPPORTED = 0, -1, -2, -3, -4, -5, -6


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.device_count() > 0:
        pytest.skip("the pointers of these calls are made up: for hosts without a GPU")
    return binding.load_library()


def caller(function, defaults):
    def call(**kw):
        assert set(kw) <= set(defaults), set(kw) - set(defaults)
        rc = function(*{**defaults, **kw}.values())
        if rc not in (OK, HIP):
            assert binding.load_library().sa_last_error() != b""
        return rc
    return call


def test_layernorm(lib):
    call = caller(lib.sa_layernorm, dict(x=FAKE, x_type=0, T=10, E=65, gamma=FAKE, beta=FAKE, eps=1e-6, y=FAKE, y_type=1, mean=FAKE,
                                         rstd=FAKE, wg=FAKE, bg=FAKE, n=2, logits=FAKE, stream=None))
    assert call() == HIP and call(y=None) == HIP and call(logits=None, n=0, wg=None, bg=None) == HIP
    for types in ((3, 0), (0, -1), (0, 7)):
        assert call(x_type=types[0], y_type=types[1]) == INVALID
    for types in ((1, 0), (2, 1), (1, 2), (2, 0)):
        assert call(x_type=types[0], y_type=types[1]) == UNSUPPORTED
    assert call(T=-1) == INVALID and call(E=0) == INVALID and call(E=8193) == UNSUPPORTED and call(T=1 << 31) == SHAPE
    assert call(n=1) == SHAPE and call(n=9) == SHAPE and call(wg=None) == INVALID and call(bg=None) == INVALID
    assert call(y=None, mean=None, rstd=None, logits=None) == INVALID
    for name in ("x", "gamma", "beta"):
        assert call(**{name: None}) == INVALID, name
    for name in ("x", "gamma", "beta", "y", "mean", "rstd", "wg", "bg", "logits"):
        assert call(**{name: ODD}) == ALIGN, name
    assert call(T=0, x=None, gamma=None, beta=None, y=None, mean=None, rstd=None, logits=None) == OK


def test_layernorm_backward(lib):
    call = caller(lib.sa_layernorm_backward, dict(
        dy=FAKE, y_type=2, x=FAKE, x_type=2, T=10, E=65, gamma=FAKE, beta=FAKE, eps=1e-6, mean=FAKE, rstd=FAKE, dres=FAKE, dlogits=FAKE,
        wg=FAKE, n=3, dx=FAKE, dgamma=FAKE, dbeta=FAKE, dwg=FAKE, dbg=FAKE, accumulate=0, workspace=FAKE, bytes=1 << 40, stream=None))
    frozen = dict(dgamma=None, dbeta=None, dwg=None, dbg=None, workspace=None, bytes=0)
    assert call() == HIP and call(mean=None, rstd=None) == HIP and call(dres=None) == HIP and call(**frozen) == HIP
    assert call(dlogits=None, wg=None, n=0, dwg=None, dbg=None, beta=None) == HIP and call(dwg=None, dbg=None, beta=None) == HIP
    assert call(x_type=1) == UNSUPPORTED and call(y_type=5) == INVALID
    assert call(T=-1) == INVALID and call(E=-3) == INVALID and call(E=10000) == UNSUPPORTED and call(T=1 << 31) == SHAPE
    assert call(n=1) == SHAPE and call(n=9) == SHAPE and call(n=0) == SHAPE
    assert call(mean=None) == INVALID and call(rstd=None) == INVALID
    assert call(dgamma=None) == INVALID and call(dbeta=None) == INVALID and call(dwg=None) == INVALID and call(dbg=None) == INVALID
    assert call(dlogits=None) == INVALID and call(dgamma=None, dbeta=None) == INVALID
    assert call(wg=None) == INVALID and call(beta=None) == INVALID
    for name in ("dy", "x", "gamma", "dx"):
        assert call(**{name: None}) == INVALID, name
    for name in ("dy", "x", "gamma", "beta", "mean", "rstd", "dres", "dlogits", "wg", "dx", "dgamma", "dbeta", "dwg", "dbg", "workspace"):
        assert call(**{name: ODD}) == ALIGN, name
    need = lib.sa_layernorm_backward_workspace_bytes(10, 65, 3)
    assert need > 0 and call(bytes=need - 1) == WORKSPACE and call(workspace=None) == WORKSPACE and call(bytes=need) == HIP
    assert lib.sa_last_error() != b""
    # a frozen norm of wide rows behind a router of many experts has its weights in another order in the workspace
    assert call(**{**frozen, "E": 2049}) == WORKSPACE and call(**{**frozen, "E": 2048}) == HIP and call(**{**frozen, "E": 2049, "n": 2}) == HIP
    assert call(**{**frozen, "E": 2049, "workspace": FAKE, "bytes": 4 * 2052 * 3 + 256}) == HIP
    for sizes in ((0, 64, 0), (-1, 64, 0), (10, 0, 0), (10, 8193, 0), (10, 64, 1), (10, 64, 9), (1 << 31, 64, 0)):
        assert lib.sa_layernorm_backward_workspace_bytes(*sizes) == 0, sizes
    assert call(T=0, accumulate=1) == OK and call(T=0) == HIP        # sums over no rows are zeros, which a launch has to write


def test_balance_loss_grad(lib):
    call = caller(lib.sa_moe_balance_loss_grad, dict(
        logits=FAKE, T=1000, E=3, valid=FAKE, alpha=FAKE, noise_std=0.5, dlosses=FAKE, losses=FAKE, sums=FAKE, counts=FAKE, dlogits=FAKE,
        accumulate=0, workspace=FAKE, bytes=1 << 40, stream=None))
    assert call() == HIP and call(valid=None, sums=None, counts=None) == HIP and call(T=0, logits=None, dlogits=None, valid=None) == HIP
    assert call(T=-1) == INVALID and call(T=1 << 31) == SHAPE and call(E=1) == SHAPE and call(E=9) == SHAPE
    for std in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        assert call(noise_std=std) == INVALID, std
    for name in ("logits", "alpha", "dlosses", "losses", "dlogits"):
        assert call(**{name: None}) == INVALID, name
    for name in ("logits", "valid", "alpha", "dlosses", "losses", "sums", "counts", "dlogits", "workspace"):
        assert call(**{name: ODD}) == ALIGN, name
    need = lib.sa_moe_balance_loss_grad_workspace_bytes(1000, 3)
    assert need > 0 and call(bytes=need - 1) == WORKSPACE and call(workspace=None) == WORKSPACE and call(bytes=need) == HIP
    for sizes in ((-1, 2), (10, 1), (10, 9), (1 << 31, 2)):
        assert lib.sa_moe_balance_loss_grad_workspace_bytes(*sizes) == 0, sizes


def test_combine_rows_backward(lib):
    rows = lambda r=FAKE, c=None, e=0, m=10: ctypes.byref(binding.SaRows(r, c, e, m))      # noqa: E731
    call = caller(lib.sa_combine_rows_backward, dict(
        dy=FAKE, y_type=0, src=FAKE, src_type=1, rows=rows(), gate=FAKE, logits=FAKE, n=2, E=65, dsrc=FAKE, dgate=FAKE, dlogits=FAKE,
        stream=None))
    assert call() == HIP and call(gate=None, logits=None, dlogits=None) == HIP and call(src=None, dgate=None, dlogits=None) == HIP
    assert call(rows=rows(None)) == HIP and call(rows=rows(FAKE, FAKE, 7)) == HIP and call(rows=rows(m=0), dy=None) == OK
    assert call(y_type=1, src_type=0) == UNSUPPORTED and call(y_type=9) == INVALID
    assert call(E=0) == SHAPE and call(E=(1 << 30) + 1) == SHAPE and call(n=1) == SHAPE and call(n=9) == SHAPE
    assert call(rows=None) == INVALID and call(rows=rows(m=-1)) == INVALID and call(rows=rows(m=1 << 31)) == SHAPE
    assert call(rows=rows(None, FAKE)) == INVALID and call(rows=rows(FAKE, FAKE, 8)) == INVALID
    assert call(dy=None) == INVALID and call(src=None) == INVALID and call(logits=None) == INVALID and call(gate=None) == INVALID
    assert call(dsrc=None, dgate=None, dlogits=None) == INVALID
    for name in ("dy", "src", "gate", "logits", "dsrc", "dgate", "dlogits"):
        assert call(**{name: ODD}) == ALIGN, name
    assert call(rows=rows(0x1002)) == ALIGN


def test_binding_refuses_what_is_not_on_the_current_gpu():
    x, v = torch.zeros(4, 8), torch.zeros(8)
    for f in (lambda: binding.sa_layernorm(x, v, v, 1e-6), lambda: binding.sa_layernorm_backward(x, x, v, v, 1e-6),
              lambda: binding.sa_moe_balance_loss_grad(x, v, 0.1, torch.zeros(2)),
              lambda: binding.sa_combine_rows_backward(x, x, gate=torch.zeros(4))):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            f()
