"""The vocabulary calls on changing streams: one context's workspace is used by
one call at a time, whatever stream each call is on."""

import pytest

from paper_1606_00511_amd import hf as H
from tests.test_gpu_vocab import head_inputs

pytestmark = pytest.mark.gpu


def inputs(k, rows=3000, V=20000, D=512):
    return head_inputs("bf16", rows, V, D, seed=k)


def test_switches_with_a_refused_call_between():
    """A long call on one stream, a refused one on a second, a call with other
    inputs on a third, again and again: the bits of each alone."""
    import torch
    jobs = [inputs(k) for k in range(2)]
    net = H.HFVocab(20000, 512, 3000, "bf16")
    want = [[o.clone() for o in net.hf_vocab_loss_grad(*j)] for j in jobs]
    s = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        with torch.cuda.stream(s[0]):
            got.append((0, net.hf_vocab_loss_grad(*jobs[0])))
        with torch.cuda.stream(s[1]), pytest.raises(H.HFError):
            net.hf_vocab_loss_grad(*jobs[0], denom=-1.0)
        with torch.cuda.stream(s[2]):
            got.append((1, net.hf_vocab_loss_grad(*jobs[1])))
    torch.cuda.synchronize()
    for k, outs in got:
        for a, b in zip(want[k], outs):
            assert torch.equal(a, b)


def test_capture_between_eager_calls():
    """A long eager call on one stream, a captured call on a second, an eager
    one with other inputs on a third, and replays: the bits of each alone."""
    import torch
    jobs = [inputs(k) for k in range(2)]
    net = H.HFVocab(20000, 512, 3000, "bf16")
    want = [[o.clone() for o in net.hf_vocab_loss_grad(*j)] for j in jobs]
    first, side, third = (torch.cuda.Stream() for _ in range(3))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    # (begun and ended by hand: torch.cuda.graph waits for the device first)
    with torch.cuda.stream(side):
        net.hf_vocab_loss_grad(*jobs[0])
        torch.cuda.synchronize()
        with torch.cuda.stream(first):
            eager = [net.hf_vocab_loss_grad(*jobs[0])]
        g.capture_begin()
        caught = net.hf_vocab_loss_grad(*jobs[0])
        g.capture_end()
    with torch.cuda.stream(third):
        eager.append(net.hf_vocab_loss_grad(*jobs[1]))
    torch.cuda.synchronize()
    for w, got in zip(want, eager):
        for a, b in zip(w, got):
            assert torch.equal(a, b)
    for _ in range(3):
        for o in caught:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want[0], caught):
            assert torch.equal(a, b)
        for a, b in zip(want[1], net.hf_vocab_loss_grad(*jobs[1])):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_workspace_of_a_dropped_context():
    """A context dropped while a side stream still works in its workspace: the
    allocator does not hand the memory to another stream meanwhile."""
    import torch
    X, W, y = inputs(0)
    want = [o.clone() for o in H.HFVocab(20000, 512, 3000, "bf16").hf_vocab_loss_grad(X, W, y)]
    net = H.HFVocab(20000, 512, 3000, "bf16")      # on the default stream
    at, size = net.workspace.data_ptr(), net.workspace.numel()
    s, done = torch.cuda.Stream(), torch.cuda.Event()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(50):
            got = net.hf_vocab_loss_grad(X, W, y)
        done.record()
    del net
    new = torch.empty(size, dtype=torch.uint8, device="cuda")
    apart = new.data_ptr() >= at + size or at >= new.data_ptr() + size
    assert done.query() or apart
    new.fill_(0xff)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
