"""The vocabulary calls at sizes that meet several of their limits, and on
values and arguments between the cases of the other tests."""

import math

import pytest

from paper_1606_00511_amd import hf as H
from tests.test_gpu_vocab import (E32, IGN, check_head, dt, gen, head_inputs, label_targets,
                                  list_targets, mask_rows, reference, teacher, unit, within)

pytestmark = pytest.mark.gpu


def T():
    import torch
    return torch


def test_embedding_past_a_million_workgroups():
    """Rows times strips of 1 KiB that take a second dimension of the grid;
    every element of the first and last rows and of every 997th."""
    torch = T()
    torch.cuda.empty_cache()
    rows, V, D = 65793, 5, 16500
    E = torch.randn(V, D, generator=gen(0), device="cuda")
    tok = mask_rows(torch.randint(0, V, (rows,), generator=gen(1), device="cuda").int(), "some")
    net = H.HFVocab(V, D, rows, "fp32")
    out = torch.full((rows, D), 7.0, device="cuda")
    net.hf_vocab_embed(E, tok, 2.0, out=out)
    assert -(-rows * -(-D // 256) // 4) > 1 << 20
    at = torch.cat([torch.arange(64), torch.arange(0, rows, 997), torch.arange(rows - 64, rows)])
    keep = (tok >= 0)[at, None]
    assert torch.equal(out[at], torch.where(keep, E[tok[at].long().clamp(min=0)] * 2, 0.0))
    assert int((out == 7).sum()) == 0
    net.hf_vocab_check()
    del net, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_row_gradients_past_a_million_workgroups(name):
    """Row gradients of several pieces of the vocabulary, with more groups of
    columns than the kernel that finishes them has threads.  The vocabulary's
    words are 5 different rows of W, so the reference needs 5 columns of them;
    checked on the first and last rows and every 997th."""
    torch = T()
    torch.cuda.empty_cache()
    rows, V, D, R = 65793, 13000 if name == "bf16" else 7000, 16390, 5
    X, W, y = head_inputs(name, rows, R, D)
    net = H.HFVocab(V, D, rows, name)
    word = torch.arange(V, device="cuda") % R
    _, rl, dX, _ = net.hf_vocab_loss_grad(X, W[word].contiguous(), y, need_dW=False)
    assert rows * -(-D // 4) > 256 << 20
    at = torch.cat([torch.arange(64), torch.arange(0, rows, 997),
                    torch.arange(rows - 64, rows)]).cuda()
    # p of a row of W is that of all its words together
    n = torch.bincount(word, minlength=R).double()
    x, w = X[at].double(), W.double()
    z = x @ w.t()
    lp = torch.log_softmax(z + n.log(), 1)
    q = torch.zeros_like(z).scatter_(1, y[at].long()[:, None], 1.0)
    ez = (D * E32 * (x.abs() @ w.abs().t()) + E32 * z.abs()).amax(1, keepdim=True)
    elp = 2 * ez + (512 + V // 128) * E32
    p1 = lp.exp() / n                  # of a word
    # each word's delta is rounded: p by its error, by u, and by the fp16
    # exponentials of bf16; the label's own word has p - 1
    u = unit(name)
    each = p1 * (elp + 64 * E32 + u) + (2.0 ** -12 * p1 + 2.0 ** -25 * p1.amax(1, keepdim=True)
                                        if name == "bf16" else 0.0)
    ed = n * each + q * (u + 256 * E32)
    d = lp.exp() - q
    terms = (lp.exp() + q) @ w.abs()
    want = (d @ w) / rows
    bound = ((ed @ w.abs()) * (1 + u) + terms * (V + 64) * E32) / rows + (u + 4 * E32) * want.abs()
    within(dX[at], want, bound, "dX")
    label = lp.gather(1, y[at].long()[:, None])[:, 0] - n[y[at].long()].log()
    within(rl[at], -label, (elp[:, 0] + 256 * E32) * (1 + label.abs()) + E32, "row losses")
    assert torch.isfinite(dX).all()
    del net, dX
    torch.cuda.empty_cache()


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D", [(1, 1000, 64), (1, 70000, 72), (31, 5000, 200),
                                      (64, 30000, 128), (65, 700, 64), (128, 20000, 320)])
def test_few_rows_in_their_own_workspace(name, rows, V, D):
    """A workspace of just the bytes asked for, full of NaN, with more of them
    on both sides, which stay as they are."""
    torch = T()
    X, W, y = head_inputs(name, rows, V, D)
    ids, t = teacher(rows, V, 40)
    net = H.HFVocab(V, D, rows, name)
    n, side = net.workspace.numel(), 1 << 20
    room = torch.full((n + 2 * side,), 0xff, dtype=torch.uint8, device="cuda")
    net._check(H.lib().hf_vocab_set_workspace(net._h, room.data_ptr() + side, n))
    q_of, used = label_targets(y, V)
    check_head(name, reference(X, W, q_of, 1.0, used, rows), V,
               net.hf_vocab_loss_grad(X, W, y), two=name == "bf16")
    q_of, used = list_targets(ids, t, 2.0, V)
    check_head(name, reference(X, W, q_of, 2.0, used, rows), V,
               net.hf_vocab_distill_grad(X, W, ids, t, 2.0), two=name == "bf16")
    net.hf_vocab_embed_grad(y, X)
    assert (room[:side] == 0xff).all() and (room[n + side:] == 0xff).all()


@pytest.mark.parametrize("rows", [200, 1500])
def test_words_far_below_their_neighbours(rows):
    """bf16 keeps exponentials in fp16, below the largest of 64 or 128 words: a
    word whose logit is 10 to 20 less than a neighbour's has its gradient to the
    bits of the type all the same.  p is off by its exponential's rounding,
    2^-12, and the error of z - lse; delta by u besides, its sum over the rows
    by 2 rows e, the result by u."""
    torch = T()
    V, D, u = 700, 64, unit("bf16")
    # x = 1 in one column, and small whole numbers over 8 in another
    X = torch.zeros(rows, D, device="cuda", dtype=torch.bfloat16)
    X[:, 0] = 1
    X[:, 1] = torch.randint(1, 9, (rows,), generator=gen(0), device="cuda") / 8.0
    y = torch.zeros(rows, dtype=torch.int32, device="cuda")
    W = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    W[0, 0] = W[640, 0] = 20                # the largest of their entries
    gaps = (10, 12, 14, 16, 17, 18, 19, 20)
    for i, g in enumerate(gaps):
        W[1 + 5 * i, 0] = W[641 + 5 * i, 0] = 20 - g
    net = H.HFVocab(V, D, rows, "bf16")
    dW = net.hf_vocab_loss_grad(X, W, y)[3]
    x = X.double()
    z = x @ W.double().t()
    p = torch.log_softmax(z, 1).exp()
    want = (p.t() @ x) / rows
    elp = 2 * (D * E32 * 20 + E32 * 20) + (512 + V // 128) * E32 + 64 * E32
    rel = (2.0 ** -12 + elp + u) * (1 + u) + 2 * rows * E32 + u + 4 * E32
    at = [v + 5 * i for i in range(len(gaps)) for v in (1, 641)]
    within(dW[at], want[at], rel * want[at].abs() + 1e-38, "dW")
