"""What the binding of the training operators refuses before it calls the library.  Nothing here needs a GPU: the device of the arguments is the
host, and in the library's place stands what notes the call."""
import pytest
import torch

from paper_2306_06446_amd import binding


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    stub = Library()
    monkeypatch.setattr(binding, "load_library", lambda: stub)
    monkeypatch.setattr(binding, "_current_device", lambda t, name, dtypes, dims=2: (-1, None))
    return stub


def test_combine_backward_refuses_counts_that_do_not_reach_the_expert(lib):
    """The kernel reads counts[0 .. expert], and finds the expert's rows by their sum."""
    T, E = 12, 8
    out = lambda: dict(dsrc=torch.zeros(T, E), dgate=torch.zeros(T), dlogits=torch.zeros(T, 3))      # noqa: E731
    call = lambda counts, expert: binding.sa_combine_rows_backward(      # noqa: E731
        torch.zeros(T, E), torch.zeros(T, E), rows=torch.arange(T, dtype=torch.int32), counts=counts, expert=expert, gate=torch.ones(T),
        logits=torch.zeros(T, 3), **out())
    counts = torch.tensor([5, 4, 3], dtype=torch.int32)
    for expert in (0, 1, 2):
        call(counts, expert)
    assert lib.calls == ["sa_combine_rows_backward"] * 3
    for short, expert in ((counts, 3), (counts[:1], 1), (counts[:0], 0), (counts, 7), (counts, -1)):
        with pytest.raises(ValueError):
            call(short, expert)
    assert len(lib.calls) == 3


def test_layernorm_refuses_what_is_no_type_or_shape_of_its_arguments(lib):
    """As other wrong arguments are refused: by a ValueError that names the argument."""
    x, v = torch.zeros(4, 8), torch.zeros(8)
    stats = dict(mean=torch.zeros(4), rstd=torch.zeros(4), dx=torch.zeros(4, 8), want_params=False)
    binding.sa_layernorm(x, v, v, 1e-6, y=torch.zeros(4, 8), want_stats=False)
    binding.sa_layernorm_backward(x, x, v, v, 1e-6, **stats)
    binding.sa_layernorm(x, v, v, 1e-6, want_y=False, y_dtype=torch.float64, **{k: stats[k] for k in ("mean", "rstd")})      # of no rows
    assert len(lib.calls) == 3
    for f, name in ((lambda: binding.sa_layernorm(x, v, v, 1e-6, y=torch.zeros(4, 8).double(), want_stats=False), "y"),
                    (lambda: binding.sa_layernorm(x, v, v, 1e-6, y=torch.zeros(4, 8, dtype=torch.int32), want_stats=False), "y"),
                    (lambda: binding.sa_layernorm(x, v, v, 1e-6, y_dtype=torch.float64, want_stats=False), "y"),
                    (lambda: binding.sa_layernorm(x, v, v, 1e-6, y=x.clone(), want_stats=False, wg=v, bg=v), "wg"),
                    (lambda: binding.sa_layernorm_backward(x.double(), x, v, v, 1e-6, **stats), "dy"),
                    (lambda: binding.sa_layernorm_backward(x, x, v, v, 1e-6, dlogits=torch.zeros(4), wg=torch.zeros(8, 4), **stats), "dlogits")):
        with pytest.raises(ValueError, match="^%s:" % name):
            f()
    assert len(lib.calls) == 3


def test_combine_backward_refuses_logits_of_one_dimension(lib):
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="^logits:"):
        binding.sa_combine_rows_backward(x, x, gate=torch.ones(4), logits=torch.zeros(4), dsrc=x.clone(), dgate=torch.zeros(4))
    assert not lib.calls
