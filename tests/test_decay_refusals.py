"""What linear attention with a decay for each head refuses, each with its own code and before anything is launched (on a host without a GPU a launch
comes back as SA_ERR_HIP), what the binding refuses before it calls the library, and what the compiler made of the kernels."""
import re

import pytest
import torch

from paper_2306_06446_amd import binding
from test_kernel_resources import kernels      # noqa: F401
from test_training_refusals import ALIGN, FAKE, HIP, INVALID, ODD, OK, SHAPE, UNSUPPORTED, WORKSPACE, caller, lib      # noqa: F401

A, B_, C, D, E, F, G = (0x10000 * i for i in range(1, 8))


def refuses_heads(call, T="T", hip=HIP):
    assert call(type=3) == INVALID and call(type=-1) == INVALID
    assert call(**{T: -8}) == INVALID and call(**{T: 1 << 31}) == SHAPE
    assert call(H=0) == SHAPE and call(Hk=0) == SHAPE and call(H=4, Hk=3) == SHAPE and call(H=-4) == SHAPE
    assert call(H=4096, Hk=1, qs=1 << 19, os=1 << 19) == hip and call(H=8192, Hk=1, qs=1 << 20, os=1 << 20) == UNSUPPORTED
    for name in ("d", "dv"):
        assert call(**{name: 60}) == SHAPE and call(**{name: 0}) == SHAPE and call(**{name: -8}) == SHAPE and call(**{name: 136}) == UNSUPPORTED, name


def refuses_rows(call, names):
    for name in names:
        stride = {"dout": "os", "out": "os", "q": "qs", "k": "ks", "v": "vs", "dq": "dqs", "dk": "dks", "dv_rows": "dvs"}[name]
        assert call(**{name: None}) == INVALID, name
        assert call(**{name: ODD}) == ALIGN, name
        assert call(**{stride: 8}) == SHAPE and call(**{stride: -512}) == SHAPE and call(**{stride: 1004}) == ALIGN, name
        assert call(**{stride: 1 << 22}) == UNSUPPORTED, name


def test_prompts(lib):      # noqa: F811
    call = caller(lib.sa_decay_attention, dict(
        q=A, qs=1024, k=B_, ks=1024, v=C, vs=1024, type=1, g=FAKE, T=96, B=2, off=None, H=4, Hk=2, d=64, dv=72, scale=0.1, first=D, last=E, slots=None,
        places=0, out=F, os=1024, ws=G, bytes=1 << 40, stream=None))
    assert call() == HIP and call(first=None) == HIP and call(last=None) == HIP and call(off=FAKE) == HIP and call(slots=FAKE, places=5) == HIP
    assert call(first=D, last=D) == HIP and call(type=0) == HIP and call(type=2) == HIP
    refuses_heads(call)
    refuses_rows(call, ("q", "k", "v", "out"))
    assert call(B=-1) == INVALID and call(T=97) == SHAPE and call(T=97, off=FAKE) == HIP and call(B=0) == SHAPE and call(B=0, off=FAKE) == OK
    assert call(T=1 << 30, B=1, off=FAKE) == UNSUPPORTED and call(T=65536 * 2, B=65536, Hk=2) == UNSUPPORTED
    assert call(places=-1) == HIP and call(places=-1, slots=FAKE) == INVALID
    for name in ("q", "k", "v"):
        assert call(out={"q": A, "k": B_, "v": C}[name]) == INVALID
    assert call(g=None) == INVALID
    for name in ("first", "last", "ws"):
        assert call(**{name: ODD}) == ALIGN, name
    assert call(g=ODD) == HIP and call(g=0x1002) == ALIGN
    assert call(off=0x1002) == ALIGN and call(slots=0x1002, places=3) == ALIGN and call(off=ODD) == HIP
    need = lib.sa_decay_attention_workspace_bytes(4000, 1, 4, 2, 64, 72, 0)
    assert need > 0 and call(T=4000, B=1, bytes=need) == HIP and call(T=4000, B=1, bytes=need - 1) == WORKSPACE and call(T=4000, B=1, ws=None) == WORKSPACE
    assert lib.sa_decay_attention_workspace_bytes(96, 2, 4, 2, 64, 72, 0) == 0 and call(ws=None, bytes=0) == HIP
    for sizes in ((97, 2, 4, 2, 64, 72, 0), (-1, 1, 4, 2, 64, 72, 0), (96, 2, 4, 3, 64, 72, 0), (96, 2, 4, 2, 60, 72, 0), (96, 2, 4, 2, 64, 136, 0)):
        assert lib.sa_decay_attention_workspace_bytes(*sizes) == 0, sizes
    # no tokens: nothing to do, unless states are to be left
    none = dict(T=0, q=None, k=None, v=None, out=None)
    assert call(**none, last=None) == OK and call(**none) == HIP and call(**none, off=FAKE) == HIP


def test_steps(lib):      # noqa: F811
    call = caller(lib.sa_decay_attention_step, dict(
        q=A, qs=1024, k=B_, ks=1024, v=C, vs=1024, type=1, g=FAKE, B=6, H=4, Hk=2, d=64, dv=72, scale=0.1, first=D, last=E, slots=None, places=0, out=F, os=1024,
        stream=None))
    assert call() == HIP and call(last=D) == HIP and call(slots=FAKE, places=5) == HIP and call(B=0, q=None, first=None) == OK
    refuses_heads(call, "B")
    refuses_rows(call, ("q", "k", "v", "out"))
    assert call(slots=FAKE, places=-1) == INVALID and call(out=A) == INVALID and call(out=B_) == INVALID and call(out=C) == INVALID
    for name in ("first", "last"):
        assert call(**{name: None}) == INVALID and call(**{name: ODD}) == ALIGN, name
    assert call(g=None) == INVALID and call(g=ODD) == HIP and call(g=0x1002) == ALIGN
    assert call(slots=0x1002, places=3) == ALIGN and call(B=(1 << 31) - 1, Hk=4, H=4) == UNSUPPORTED


@pytest.mark.parametrize("dv,states", [(64, 1 << 24), (72, 1 << 23)])
def test_steps_of_more_threads_than_a_launch_has(lib, dv, states):      # noqa: F811
    """256 threads to 64 columns of a state, and less than 2^32 of them: more states are refused before the launch."""
    call = caller(lib.sa_decay_attention_step, dict(
        q=A, qs=1024, k=B_, ks=1024, v=C, vs=1024, type=1, g=FAKE, B=6, H=4, Hk=4, d=8, dv=dv, scale=0.1, first=D, last=E, slots=None, places=0, out=F, os=1024,
        stream=None))
    assert call(B=states // 4 - 1) == HIP and call(B=states // 4) == UNSUPPORTED


def test_backward(lib):      # noqa: F811
    call = caller(lib.sa_decay_attention_backward, dict(
        dout=A, os=1024, q=B_, qs=1024, k=C, ks=1024, v=D, vs=1024, type=1, g=FAKE, T=96, B=2, off=None, H=4, Hk=2, d=64, dv=72, scale=0.1, first=0x100000,
        dlast=0x200000, dq=E, dqs=1024, dk=F, dks=1024, dv_rows=G, dvs=1024, dfirst=0x300000, ws=0x400000, bytes=1 << 40, stream=None))
    assert call() == HIP and call(first=None) == HIP and call(dlast=None) == HIP and call(dfirst=None) == HIP and call(off=FAKE) == HIP
    refuses_heads(lambda **kw: call(**kw, **({"dqs": kw["qs"]} if "qs" in kw and "H" in kw else {})))
    refuses_rows(call, ("dout", "q", "k", "v", "dq", "dk", "dv_rows"))
    for name in ("dq", "dk", "dv_rows"):
        for other in (A, B_, C, D):
            assert call(**{name: other}) == INVALID, name
    assert call(dq=F) == INVALID and call(dk=G) == INVALID and call(dv_rows=E) == INVALID
    assert call(dfirst=0x100000) == INVALID and call(dfirst=0x200000) == INVALID and call(g=None) == INVALID
    for name in ("first", "dlast", "dfirst", "ws"):
        assert call(**{name: ODD}) == ALIGN, name
    assert call(g=ODD) == HIP and call(g=0x1002) == ALIGN
    need = lib.sa_decay_attention_backward_workspace_bytes(4000, 1, 4, 2, 64, 72, 0)
    assert need > 0 and call(T=4000, B=1, bytes=need) == HIP and call(T=4000, B=1, bytes=need - 1) == WORKSPACE and call(T=4000, B=1, ws=None) == WORKSPACE
    none = dict(T=0, dout=None, q=None, k=None, v=None, dq=None, dk=None, dv_rows=None)
    assert call(**none, dfirst=None) == OK and call(**none) == HIP and call(B=0, off=FAKE) == OK


@pytest.mark.parametrize("T,B,ragged", [(1, 1, 0), (5, 5, 1), (50021, 37, 1), (8 * 16384, 8, 0), (1 << 29, 1, 0), (100000, 1, 1), (300, 150, 0)])
def test_workspaces_hold_what_is_asked_for(lib, T, B, ragged):      # noqa: F811
    """A call takes its query's size, whatever states it has."""
    for H, Hk, d, dv in ((4, 4, 64, 64), (12, 4, 96, 72), (8, 1, 128, 128)):
        need = lib.sa_decay_attention_workspace_bytes(T, B, H, Hk, d, dv, ragged)
        back = lib.sa_decay_attention_backward_workspace_bytes(T, B, H, Hk, d, dv, ragged)
        assert need % (4 * Hk * d * dv) == 0 and back % (8 * Hk * d * dv) == 0
        s, off, ws = H * 128, FAKE if ragged else None, 0x400000
        for first, last in ((None, None), (D, None), (None, E), (D, E)):
            assert lib.sa_decay_attention(A, s, B_, s, C, s, 1, FAKE, T, B, off, H, Hk, d, dv, 1.0, first, last, None, 0, F, s, ws, need, None) == HIP
            assert lib.sa_decay_attention_backward(A, s, B_, s, C, s, D, s, 1, FAKE, T, B, off, H, Hk, d, dv, 1.0, first, last, E, s, F, s, G, s, None, ws,
                                                   back, None) == HIP


@pytest.mark.parametrize("T,B,H,Hk,d,dv", [(51200, 512, 32, 32, 128, 128), (51200, 512, 32, 32, 64, 64), (20000, 20000, 2, 2, 64, 64), (3000, 3000, 16, 16, 128, 128),
                                             (5000, 40, 12, 4, 96, 72)])
def test_short_ragged_sequences_take_no_places_of_their_own(lib, T, B, H, Hk, d, dv):      # noqa: F811
    """A sequence of one segment (256 tokens at least) needs no state in the workspace, and there are T / 256 sequences of more at most, with T / 256 ends of
    full segments: however many sequences there are, 2 T / 256 places."""
    most = 2 * (T // 256) * 4 * Hk * d * dv
    assert 0 < lib.sa_decay_attention_workspace_bytes(T, B, H, Hk, d, dv, 1) <= most
    assert 0 < lib.sa_decay_attention_backward_workspace_bytes(T, B, H, Hk, d, dv, 1) <= 2 * most


class Library:
    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0

    def __init__(self):
        self.calls = []


@pytest.fixture
def stub(monkeypatch):
    stub = Library()
    monkeypatch.setattr(binding, "load_library", lambda: stub)
    monkeypatch.setattr(binding, "_current_device", lambda t, name, dtypes, dims=2: (-1, None))
    return stub


def test_binding_takes_rows_at_one_distance(stub):
    """Heads are dense, tokens are at one distance: of a block of columns that of the wide rows; all else is a ValueError that names the argument."""
    B, N, H, d = 2, 6, 4, 16
    x, g, ws = torch.zeros(B, N, H, d), torch.zeros(H), torch.zeros(64, dtype=torch.uint8)
    call = lambda q=x, k=x, v=x, **kw: binding.sa_decay_attention(q, k, v, g, 1.0, out=kw.pop("out", x.clone()), workspace=ws, **kw)      # noqa: E731
    wide = torch.zeros(B, N, 3 * H * d)
    call(q=wide[..., 64:128].view(B, N, H, d))
    assert stub.calls[-1][1][1] == 3 * H * d and stub.calls[-1][1][3] == H * d
    call(q=torch.zeros(2 * B, N, H, d)[::2][:1].expand(1, N, H, d), k=x[:1], v=x[:1], out=x[:1].clone())
    assert stub.calls[-1][1][1] == H * d
    one = torch.zeros(B, 3, H, d)[:, :1]                     # one token of each sequence, 3 apart
    call(q=one, k=x[:, :1], v=x[:, :1], out=torch.zeros(B, 1, H, d))
    assert [stub.calls[-1][1][i] for i in (1, 3)] == [3 * H * d, 6 * H * d]
    n = len(stub.calls)
    for bad, name in ((dict(q=torch.zeros(B, H, N, d).transpose(1, 2)), "q"), (dict(k=torch.zeros(B, N, H, 2 * d)[..., ::2]), "k"),
                      (dict(v=torch.zeros(B, N + 1, H, d)[:, :N]), "v"), (dict(q=torch.zeros(B, N, H, 2 * d)[..., :d]), "q"),
                      (dict(k=torch.zeros(1, 1, H, d).expand(B, N, H, d)), "k"), (dict(q=x.half()), "k"), (dict(out=torch.zeros(B, N, H, 8)), "out"),
                      (dict(v=torch.zeros(B, N + 1, H, d)), "v"), (dict(k=torch.zeros(B * N, H, d)), "k, v"),
                      (dict(state_in=torch.zeros(B, H, d, 8)), "state_in"), (dict(state_out=torch.zeros(B + 1, H, d, d)), "state_out"),
                      (dict(state_in=torch.zeros(B, H, d, d).half()), "state_in"), (dict(state_in=torch.zeros(9, H, d, d), slots=torch.zeros(B)), "slots"),
                      (dict(state_in=torch.zeros(9, H, d, d), slots=torch.zeros(3, dtype=torch.int32)), "slots"),
                      (dict(want_state=True, slots=torch.zeros(B, dtype=torch.int32)), "want_state"),
                      (dict(state_in=torch.zeros(9, H, d, d), state_out=torch.zeros(8, H, d, d), slots=torch.zeros(B, dtype=torch.int32)), "state_in, state_out")):
        with pytest.raises(ValueError, match="^%s:" % name):
            call(**bad)
    t = torch.zeros(B * N, H, d)
    for off in (torch.zeros(3), torch.zeros(0, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="^offsets:"):
            binding.sa_decay_attention(t, t, t, g, 1.0, offsets=off, out=t.clone(), workspace=ws)
    with pytest.raises(ValueError, match="^log_decay:"):
        binding.sa_decay_attention(x, x, x, torch.zeros(H + 1), 1.0, out=x.clone(), workspace=ws)
    s = torch.zeros(5, H, d, d)
    with pytest.raises(ValueError, match="^state_in:"):
        binding.sa_decay_attention_step(t, t, t, g, 1.0, s, out=t.clone())              # 5 states of 12 sequences, and no slots
    with pytest.raises(ValueError, match="^dq:"):
        binding.sa_decay_attention_backward(x, x, x, x, g, 1.0, dq=x.half(), dk=x.clone(), dv=x.clone(), workspace=ws)
    with pytest.raises(ValueError, match="^dout:"):
        binding.sa_decay_attention_backward(x[:, :5], x, x, x, g, 1.0, dq=x.clone(), dk=x.clone(), dv=x.clone(), workspace=ws)
    assert len(stub.calls) == n


def test_no_scratch(kernels):      # noqa: F811
    """A register in scratch memory makes a wavefront wait for the rows that are under way."""
    found = {n: k for n, k in kernels.items() if re.search(r"decay_(rows|short|states|scan|step)_kernel", n)}
    assert len(found) > 40
    for n, k in found.items():
        assert k[".private_segment_fixed_size"] == 0, n
        assert k[".group_segment_fixed_size"] <= 160 * 1024, n
