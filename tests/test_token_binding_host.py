"""What tokens.py does around the calls of the library, without a GPU: tensors of the host that say they are on a device, and a boundary that
records what it is given."""
import weakref
from contextlib import contextmanager

import pytest
import torch

A = pytest.importorskip("paper_2404_09679_amd", reason="build the library first (python paper_2404_09679_amd/build.py)")
T = A.tokens


class Boundary:
    """In the library's place: every call is recorded, and `during` runs inside it.  `device` is the current one, `on` the tensors'."""

    def __init__(self):
        self.calls, self.during, self.device, self.on = [], lambda: None, 0, 0

    def __getattr__(self, name):
        def call(*args):
            self.during()
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def boundary(monkeypatch):
    b = Boundary()
    monkeypatch.setattr(T, "lib", b)
    monkeypatch.setattr(T, "_bytes", lambda call, *sizes: 4096)
    monkeypatch.setattr(T, "_stream", lambda device: 0)
    monkeypatch.setattr(T, "_current_device", lambda: b.device, raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: b.on)

    @contextmanager
    def device(index):
        before, b.device = b.device, index
        yield
        b.device = before

    monkeypatch.setattr(torch.cuda, "device", device)
    return b


def calls(dtype=torch.float32):
    """Every operator once, by name: a function that calls it."""
    x, w, h = torch.zeros(4, 8, dtype=dtype), torch.zeros(8, 16, dtype=dtype), torch.zeros(4, 16, dtype=dtype)
    t, f, saved = torch.zeros(4, dtype=torch.int32), torch.zeros(4), torch.zeros(4096, dtype=torch.uint8)
    drop = A.Dropout(0.5, 1)
    return {"antdt_dropout": lambda: A.dropout(x, drop, residual=x),
            "antdt_token_lookup": lambda: A.token_lookup(x, t, dropout=drop),
            "antdt_token_gradient": lambda: A.token_gradient(x, t, 5, dropout=drop),
            "antdt_gated_forward": lambda: A.gated_forward(x, w, w, saved=saved),
            "antdt_gated_backward": lambda: A.gated_backward(h, x, w, w, saved),
            "antdt_token_logprobs": lambda: A.token_logprobs(x, t, 2),
            "antdt_token_logprobs_gradient": lambda: A.token_logprobs_gradient(x, t, torch.zeros(4, 4), f, f)}


@pytest.mark.parametrize("name", list(calls()))
def test_buffers_live_until_the_call_returns(boundary, monkeypatch, name):
    """Results and workspaces that a call makes: one that goes back to torch's allocator before the kernels are enqueued may be another
    thread's by then."""
    made, new = [], T._new

    def noted(*args):
        out = new(*args)
        made.append(weakref.ref(out))
        return out

    seen = []
    monkeypatch.setattr(T, "_new", noted)
    boundary.during = lambda: seen.append([r() is not None for r in made])
    calls()[name]()
    assert [n for n, _ in boundary.calls] == [name]
    assert made and seen == [[True] * len(made)]


@pytest.mark.parametrize("name", list(calls()))
def test_kernels_go_to_the_operands_device(boundary, name):
    """torch's default stream has the same handle on every device: which one is meant is the current device's."""
    seen = []
    boundary.during = lambda: seen.append(boundary.device)
    for current, on in ((0, 0), (0, 1), (2, 0)):
        boundary.device, boundary.on = current, on
        calls()[name]()
        assert seen.pop() == on and boundary.device == current


def test_the_step_of_a_dropout_is_on_the_operands_device(boundary, monkeypatch):
    """Its address goes into the kernel."""
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    step = torch.zeros(1, dtype=torch.int64)
    drop = A.Dropout(0.5, 1, step=step)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1 if t.dtype == torch.int64 else 0)
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: A.dropout(x, drop), lambda: A.token_lookup(x, t, dropout=drop), lambda: A.token_gradient(x, t, 5, dropout=drop)):
        with pytest.raises(ValueError, match="step"):
            call()
    assert not boundary.calls
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    A.dropout(x, drop)
    assert len(boundary.calls) == 1


def test_the_stride_of_a_single_row_is_no_leading_dimension(boundary):
    """The last token of a long sequence, [1, T, K] sliced to [1, K]: its stride T K means nothing."""
    x = torch.zeros(1, 2100, 1024, dtype=torch.bfloat16)[:, -1]
    w = torch.zeros(1024, 16, dtype=torch.bfloat16)
    assert x.stride(0) > 1 << 21
    odd = torch.zeros(1, 16 + 3, dtype=torch.bfloat16)[:, :16]
    out = A.gated_forward(x, w, w, out=odd)
    name, args = boundary.calls.pop()
    assert out is odd and name == "antdt_gated_forward" and args[1] == 1024 and args[11] == 16
    A.token_lookup(torch.zeros(1, 9)[:, :5], torch.zeros(1, dtype=torch.int32))
    name, args = boundary.calls.pop()
    assert args[1] == 5 and args[10] == 5
    A.token_logprobs_gradient(torch.zeros(1, 7), None, torch.zeros(1, 8)[:, :4], None, torch.zeros(1))
    two = torch.zeros(2, 9)[:, :5]
    A.dropout(two, A.Dropout(0.5, 1))
    assert boundary.calls.pop()[1][1] == 9


def test_refusals_of_the_gated_blocks_tensors(boundary):
    x, w = torch.zeros(4, 8), torch.zeros(8, 16)
    saved = torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: A.gated_saved(x.half(), w), lambda: A.gated_saved(x[0], w), lambda: A.gated_saved(x, w[0]), lambda: A.gated_saved(x, w[0, 0]),
                 lambda: A.gated_forward(x, w[0, 0], w), lambda: A.gated_forward(x, w[0], w[0]), lambda: A.gated_forward(x, w, w[0, 0]),
                 lambda: A.gated_backward(torch.zeros(4, 16), x, w[0, 0], w, saved)):
        with pytest.raises(ValueError):
            call()
    assert not boundary.calls
