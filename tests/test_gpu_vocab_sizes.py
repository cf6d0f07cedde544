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


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [100, 300, 3000])
def test_last_words(name, rows):
    """Labels among the last words of an odd vocabulary: what these words give
    is most of each row's gradient, far above the bound of its sum."""
    torch = T()
    V, D = 50257, 200
    X, W, _ = head_inputs(name, rows, V, D)
    y = (V - 1 - torch.arange(rows, device="cuda") % 130).int()
    net = H.HFVocab(V, D, rows, name)
    q_of, used = label_targets(y, V)
    ref = reference(X, W, q_of, 1.0, used, rows)
    assert (ref["adX"] * V * E32).mean() < 0.02 * ref["dX"].abs().mean()
    check_head(name, ref, V, net.hf_vocab_loss_grad(X, W, y), two=name == "bf16" and rows <= 128)


# (fp32 and bf16 in pieces, W in place or packed; the last: a piece of W's
# packing ends within a piece of the logits, in the kept one and those computed
# again)
PIECES = [("fp32", 8000, 131075, 72), ("bf16", 8000, 131075, 72), ("bf16", 8000, 131075, 64),
          ("fp32", 12000, 70000, 2050), ("bf16", 12000, 131500, 2050)]


@pytest.mark.parametrize("name,rows,V,D", PIECES)
def test_pieces_with_all_the_options(name, rows, V, D):
    """Logits computed again in pieces: with NaN and infinities in masked rows,
    one gradient only, a strided dW, and dW added to, for labels and lists."""
    torch = T()
    torch.cuda.empty_cache()
    X, W, y = head_inputs(name, rows, V, D)
    y = mask_rows(y, "some")
    X[y < 0] = math.nan
    X[(y < 0).nonzero()[::2, 0]] = math.inf
    ids, t = teacher(rows, V, 20)
    ids[y < 0] = IGN
    net = H.HFVocab(V, D, rows, name)
    u = unit(name)
    for call, targets, (q_of, used), tau in (
            (net.hf_vocab_loss_grad, (y,), label_targets(y, V), 1.0),
            (net.hf_vocab_distill_grad, (ids, t, 2.0), list_targets(ids, t, 2.0, V), 2.0)):
        n = int(used.sum())
        ref = reference(X, W, q_of, tau, used, n, chunk=512)
        want = [o.clone() for o in call(X, W, *targets)]
        check_head(name, ref, V, want)
        assert torch.equal(call(X, W, *targets, need_dW=False)[2], want[2])
        assert torch.equal(call(X, W, *targets, need_dX=False)[3], want[3])
        wide = torch.full((V, D + 5), 7.0, device="cuda", dtype=dt(name))
        call(X, W, *targets, dW=wide[:, 3:3 + D], need_dX=False)
        assert torch.equal(wide[:, 3:3 + D], want[3])
        assert (wide[:, :3] == 7).all() and (wide[:, 3 + D:] == 7).all()
        # dW += : one rounding of the sum
        old = torch.randn(V, D, generator=gen(9), device="cuda").to(dt(name)) * 1e-3
        got = call(X, W, *targets, dW=old.clone(), accumulate=True)[3]
        total = ref["dW"] + old.double()
        within(got, total, ref["edW"] * (1 + u) + ref["adW"] * (u + (2 * rows + 64) * E32) *
               (1 + 2 * u) + (u + 4 * E32) * total.abs() + E32 * old.double().abs(), "dW +=")
        del ref, want, wide, old, got, total
    net.hf_vocab_check()
    del net
    torch.cuda.empty_cache()


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [40, 300])
def test_rows_that_count_with_no_numbers(name, rows):
    """NaN and infinities in rows that count: NaN or infinity where the
    definition has one, and nowhere else."""
    torch = T()
    V, D = 300, 64
    X, W, y = head_inputs(name, rows, V, D)
    y %= 100
    net = H.HFVocab(V, D, rows, name)
    want = [o.clone() for o in net.hf_vocab_loss_grad(X, W, y)]
    for bad in (math.nan, math.inf, -math.inf):
        Z = X.clone()
        Z[7, 3] = bad                       # logits of both infinities, or NaN
        loss, rl, dX, dW = net.hf_vocab_loss_grad(Z, W, y)
        others = torch.arange(rows, device="cuda") != 7
        assert rl[7].isnan() and loss[0].isnan() and dX[7].isnan().all() and dW.isnan().all()
        assert torch.equal(rl[others], want[1][others])
        assert torch.equal(dX[others], want[2][others])
        assert net.hf_vocab_loss(Z, W, y)[0].isnan()
        # a list of two on every row, with the label's place first
        ids = torch.stack([y, y + 100], 1).int()
        t = torch.zeros(rows, 2, device="cuda")
        good = [o.clone() for o in net.hf_vocab_distill_grad(X, W, ids, t)]
        for got in (net.hf_vocab_distill_grad(Z, W, ids, t),):
            assert got[1][7].isnan() and got[2][7].isnan().all() and got[3].isnan().all()
            assert torch.equal(got[2][others], good[2][others])
        if bad != -math.inf:                # (which is a masked place)
            t[7, 1] = bad
            got = net.hf_vocab_distill_grad(X, W, ids, t)
            assert got[1][7].isnan() and got[2][7].isnan().any()
            assert torch.equal(got[2][others], good[2][others])


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [40, 300])
def test_words_without_probability(name, rows):
    """Words whose logits are -inf (a column of X at 1, -inf there in their
    rows of W): the others' losses are those of the vocabulary without them;
    a label there has a loss of infinity; every word there, the loss is NaN."""
    torch = T()
    V, D = 700, 64
    X, W, y = head_inputs(name, rows, V, D)
    X[:, 0], W[:, 0] = 1, 0
    y %= 100
    net = H.HFVocab(V, D, rows, name)
    q_of, used = label_targets(y, 300)
    ref = reference(X, W[:300].contiguous(), q_of, 1.0, used, rows)
    W[300:, 0] = -math.inf                  # whole entries of the statistics
    loss, rl = net.hf_vocab_loss(X, W, y)
    check_head(name, ref, V, (loss, rl, None, None))
    loss, rl, dX, dW = net.hf_vocab_loss_grad(X, W, y)
    check_head(name, ref, V, (loss, rl, None, dW[:300]), two=name == "bf16" and rows <= 128)
    assert (dW[300:] == 0).all()
    # 0 times -inf in the column, as the definition has it; the others as ever
    assert dX[:, 0].isnan().all() and torch.isfinite(dX[:, 1:]).all()
    y[5] = 650
    rl = net.hf_vocab_loss(X, W, y)[1]
    assert rl[5].item() == math.inf and torch.isfinite(rl[:5]).all()
    W[:, 0] = -math.inf
    assert net.hf_vocab_loss(X, W, y)[1].isnan().all()


@pytest.mark.parametrize("rows,V", [(1, 700), (16, 1900), (100, 3000), (300, 900), (700, 3000)])
def test_sums_of_wide_rows(rows, V):
    """fp32 logits of few rows are summed 128 columns at a time, and then these
    sums: a logit is off by at most 128 + D / 128 + 2 times e of its magnitudes.
    In one chain of D additions the target's products, 2^-6 (1 + 2^-14), would
    lose their last bits at every addition past 32, 0.002 in all; the other
    words' are 2^-6, whose sums are exact."""
    torch = T()
    D = 4096
    X = torch.ones(rows, D, device="cuda")
    W = torch.full((V, D), 2.0 ** -6, device="cuda")
    W[V // 2] = 2.0 ** -6 * (1 + 2.0 ** -14)
    y = torch.full((rows,), V // 2, dtype=torch.int32, device="cuda")
    net = H.HFVocab(V, D, rows, "fp32")
    want = torch.full((rows,), math.log1p((V - 1) * math.exp(-(2.0 ** -8))), dtype=torch.float64,
                      device="cuda")
    most = (128 + D / 128 + 2) * E32 * 64.01
    bound = torch.full_like(want, most + (512 + V // 128) * E32 + 256 * E32 * 10)
    assert bound[0] < 1e-3
    within(net.hf_vocab_loss_grad(X, W, y)[1], want, bound, "row losses")
    within(net.hf_vocab_loss(X, W, y)[1], want, bound, "row losses, alone")
    t = torch.zeros(rows, 1, device="cuda")
    within(net.hf_vocab_distill(X, W, y[:, None], t)[1], want, bound, "list's losses")
