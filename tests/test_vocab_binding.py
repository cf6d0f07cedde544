"""What HFVocab, and HFNet of its streams, hand to the C calls and to torch,
with both faked.  No GPU."""

from types import SimpleNamespace

import pytest

from paper_1606_00511_amd import hf as H


def bare(cls):
    """An object without a C context; nothing is freed when it goes."""
    kind = type(cls.__name__, (cls,), {"close": lambda self: None})
    return kind.__new__(kind)


class Fakes:
    """A library that answers `codes` in turn and then HF_OK, and torch's
    current stream."""

    def __init__(self, monkeypatch):
        self.calls, self.codes, self.recorded = [], [], []
        self.stream = 0
        self.torch = SimpleNamespace(cuda=SimpleNamespace(
            current_device=lambda: 0,
            current_stream=lambda i=None: SimpleNamespace(cuda_stream=self.stream)))
        monkeypatch.setattr(H, "lib", lambda: self)
        self.hf_vocab_last_error = lambda h: b"an error"
        self.hf_strerror = lambda c: b"a code"

    def __getattr__(self, name):
        def call(h, *args):
            self.calls.append((name, *args))
            return self.codes.pop(0) if self.codes else H.HF_OK
        return call

    def vocab(self):
        net = bare(H.HFVocab)
        net._torch, net._h, net._stream = self.torch, 1, None
        net.device = SimpleNamespace(index=0)
        net.workspace = SimpleNamespace(
            record_stream=lambda s: self.recorded.append(s.cuda_stream))
        return net


@pytest.fixture
def fakes(monkeypatch):
    return Fakes(monkeypatch)


def test_every_stream_is_recorded_for_the_workspace(fakes):
    """The allocator knows of each stream that the workspace is used on, the
    first one included: the context may have been made on another."""
    net = fakes.vocab()
    for s in (0, 0, 5, 5, 0, 7):
        fakes.stream = s
        net._call("hf_vocab_check")
    assert [c[1] for c in fakes.calls if c[0] == "hf_vocab_set_stream"] == [0, 5, 0, 7]
    assert set(fakes.recorded) == {0, 5, 7}


def test_a_switch_that_failed_is_made_again(fakes):
    """A switch of streams fails, and the caller goes back to the stream of
    before: the C context is told, as it may be on the other one."""
    net = fakes.vocab()
    net._call("hf_vocab_check")
    fakes.stream, fakes.codes = 5, [H.HF_EHIP]
    with pytest.raises(H.HFError):
        net._call("hf_vocab_check")
    fakes.stream = 0
    del fakes.calls[:]
    net._call("hf_vocab_check")
    assert fakes.calls == [("hf_vocab_set_stream", 0), ("hf_vocab_check",)]


def test_every_stream_is_recorded_for_a_nets_workspace(fakes, monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda d=None: SimpleNamespace(cuda_stream=fakes.stream))
    net = bare(H.HFNet)
    net._h, net._last, net.device = 1, None, None
    net.workspace = fakes.vocab().workspace
    for s in (0, 0, 5, 0, 7):
        fakes.stream = s
        net._stream()
    assert [c[1] for c in fakes.calls if c[0] == "hf_set_stream"] == [0, 0, 5, 0, 7]
    assert set(fakes.recorded) == {0, 5, 7}


def test_a_gradient_given_but_not_needed(fakes):
    """A buffer for a gradient that the call is told not to compute: refused,
    for the caller expects one or the other.  Without the buffer it is None."""
    import torch
    net = fakes.vocab()
    net._torch, net.device, net.dtype = torch, torch.device("cpu"), torch.float32
    net.vocab, net.width = 5, 3
    net._call = lambda fn, *args: fakes.calls.append((fn, *args))
    X, W = torch.zeros(2, 3), torch.zeros(5, 3)
    y = torch.zeros(2, dtype=torch.int32)
    ids, t = y[:, None].repeat(1, 4), torch.zeros(2, 4)
    for call, targets in ((net.hf_vocab_loss_grad, (y,)), (net.hf_vocab_distill_grad, (ids, t))):
        for kw in (dict(dX=torch.empty(2, 3), need_dX=False),
                   dict(dW=torch.empty(5, 3), need_dW=False),
                   dict(dW=torch.empty(5, 3), need_dW=False, accumulate=True)):
            with pytest.raises(ValueError):
                call(X, W, *targets, **kw)
        assert not fakes.calls
        got = call(X, W, *targets, need_dX=False)
        assert got[2] is None and got[3].shape == (5, 3)
        got = call(X, W, *targets, need_dW=False)
        assert got[3] is None and got[2].shape == (2, 3)
        assert [c[0] for c in fakes.calls] == [call.__name__] * 2
        del fakes.calls[:]
