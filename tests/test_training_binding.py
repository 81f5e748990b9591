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
