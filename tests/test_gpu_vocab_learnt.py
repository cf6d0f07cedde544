"""Rows that the model has learnt: the target has nearly all the probability, so
its loss and its delta are what is left of 1, which is next to nothing.

The words but the target have rows of W of zeros, so z_v = 0 exactly.  The
target's z = 40 is what is left of products that first add up to thousands and
then take them away again: its sum in fp32 is off by some E, of the order of
0.01, that depends on the order of the sum, and by at most D e times the
products' magnitudes.  A target's logit that is not the one which the softmax
had would be off against it by as much.
  s        the sum over the words of exp(z_v - z): 1 for the target, and
           (V - 1) exp(-z) < 1e-12 of all others whatever E; its sum has at most
           64 + 8 + tiles / 64 + 64 additions to what holds the 1, e each
  loss     log s
  delta    1 / s - 1 for a label; the quotient and the exp are good to 8 e
  lists    the target's q by the teacher's logits of 40, 0, 0, ...: as small
The tests read delta from dX = delta W_y / rows.
"""

import math

import pytest

from paper_1606_00511_amd import hf as H
from tests.test_gpu_vocab import E32, dt, gen, within

pytestmark = pytest.mark.gpu


def learnt(name, rows, V, D, sign=1):
    """X, W and the one word that the rows have learnt; the sums' errors of
    sign -1 are those of 1 turned around."""
    import torch
    half, g = D // 2, gen(D)
    a = (torch.rand(half, generator=g, device="cuda") * 64 + 8).bfloat16()
    b = (torch.rand(half, generator=g, device="cuda") + 0.1).bfloat16()
    one = torch.ones(1, device="cuda").bfloat16()
    x = torch.cat([a, a, one])
    w = torch.cat([sign * b, -sign * b, 40 * one])
    assert D * E32 * float((x.double() * w.double()).abs().sum()) < 10
    word = V * 5 // 7
    W = torch.zeros(V, w.numel(), device="cuda", dtype=dt(name))
    W[word] = w.to(W.dtype)
    return x[None].repeat(rows, 1).to(dt(name)), W, word


def check(V, rows, rl, dX=None):
    import torch
    bound = (136 + V // 32 // 64 + 8) * E32 + 1e-12
    zero = torch.zeros(rows, dtype=torch.float64, device="cuda")
    within(rl, zero, zero + bound, "row losses")
    if dX is not None:
        within(dX[:, -1].float() * (rows / 40), zero, zero + bound * 1.01, "delta")


SHAPES = [(1, 700, 512), (5, 20000, 512), (40, 3000, 1024), (128, 20000, 512), (129, 700, 320),
          (300, 9000, 1000), (1500, 5000, 512), (3000, 20000, 1024), (4096, 4100, 770)]


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D", SHAPES)
def test_labels(name, rows, V, D):
    import torch
    for sign in (1, -1):
        X, W, word = learnt(name, rows, V, D, sign)
        y = torch.full((rows,), word, dtype=torch.int32, device="cuda")
        net = H.HFVocab(V, W.shape[1], rows, name)
        check(V, rows, net.hf_vocab_loss(X, W, y)[1])
        _, rl, dX, _ = net.hf_vocab_loss_grad(X, W, y)
        check(V, rows, rl, dX)


@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_labels_in_pieces(name):
    """Logits computed again in pieces, the word in the first and in the last."""
    import torch
    rows, V, D = 8200, 131100, 64
    for sign in (1, -1):
        X, W, word = learnt(name, rows, V, D, sign)
        net = H.HFVocab(V, W.shape[1], rows, name)
        for v in (word, 3, V - 1):
            W = torch.zeros_like(W).index_copy_(0, torch.tensor([v], device="cuda"), W[[word]])
            y = torch.full((rows,), v, dtype=torch.int32, device="cuda")
            word = v
            _, rl, dX, _ = net.hf_vocab_loss_grad(X, W, y)
            check(V, rows, rl, dX)


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D,K", [
    (1, 700, 512, 1), (5, 20000, 512, 16), (40, 3000, 1024, 5), (128, 20000, 512, 128),
    (129, 700, 320, 33), (300, 9000, 1000, 64), (1500, 5000, 512, 7), (3000, 20000, 1024, 32),
    (4096, 4100, 770, 65), (8200, 131100, 64, 3), (300, 60000, 256, 1), (1000, 50000, 384, 2),
    (1500, 50000, 320, 2)])
def test_lists(name, rows, V, D, K):
    """The word in each place of the list in turn, some lists ending early; tau
    squared of the label's bound, and of q's."""
    import torch
    for sign in (1, -1):
        X, W, word = learnt(name, rows, V, D, sign)
        at = torch.arange(rows, device="cuda") % K
        k = torch.arange(K, device="cuda")[None]
        ids = (word + 1 + k).repeat(rows, 1) % V
        ids[torch.arange(rows), at] = word
        ids = torch.where(k > torch.maximum(at, torch.randint(0, K, (rows,), device="cuda",
                                                              generator=gen(K)))[:, None],
                          H.HF_IGNORE, ids).int()
        t = torch.where(ids == word, 40.0, 0.0)
        net = H.HFVocab(V, W.shape[1], rows, name)
        for tau in (1.0, 0.5):
            bound = tau ** 2 * ((136 + V // 32 // 64 + 24) * E32 + 1e-12)
            zero = torch.zeros(rows, dtype=torch.float64, device="cuda")
            within(net.hf_vocab_distill(X, W, ids, t, tau)[1], zero, zero + bound, "losses alone")
            _, rl, dX, _ = net.hf_vocab_distill_grad(X, W, ids, t, tau)
            within(rl, zero, zero + bound, "losses")
            within(dX[:, -1].float() * (rows / 40 / tau), zero, zero + 1.01 * bound / tau ** 2,
                   "delta")
