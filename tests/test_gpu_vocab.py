"""The vocabulary calls on the GPU against their definitions in 64 bits.

Tolerances, derived from the operations (u: half a step of the type, 2^-8 for
bf16 and 2^-24 for fp32; e: 2^-24, the rounding of fp32 sums):
  logits   a sum of D products in fp32: off by at most D e sum_d |x_d w_d|;
           over tau, with one rounding more: that over tau + e |z|
  lse      moves by at most the largest logit error; the sums of exponentials
           run over at most 256 + tiles terms one after the other, and each
           exp is good to 8 e + e |z - max| (weighted by the term itself, so
           below 2 e): (512 + tiles) e covers it and the logarithm
  loss     both of these, twice the logit error for the target's own logit;
           times tau^2; the teacher's q as good as its exponentials
  delta    p relative by the error of z - lse and 64 e for the exp, rounded to
           the type by u (two terms of bf16: u^2), likewise at the targets; with
           bf16 and more than 128 rows exp(z - max) is rounded to fp16 before,
           2^-12 of it or, where fp16 has no smaller step, 2^-25 of the maximum:
           p is off by 2^-12 p + 2^-25 max p besides
  dX, dW   sum of K products in fp32: K e sum |terms|, terms off by delta's
           error, the result times a factor good to 2 e, rounded by u
  embedding  exact but for one rounding of the product by u (and e of it in
           fp32); its gradient n e sum |terms| for n tokens, rounded by u
The tests compare element by element with these bounds.
"""

import math

import pytest

from paper_1606_00511_amd import hf as H

pytestmark = pytest.mark.gpu
IGN = H.HF_IGNORE
E32 = 2.0 ** -24


def T():
    import torch
    return torch


def gen(seed):
    return T().Generator("cuda").manual_seed(seed)


def dt(name):
    return {"fp32": T().float32, "bf16": T().bfloat16}[name]


def unit(name):
    return T().finfo(dt(name)).eps / 2


def head_inputs(name, rows, V, D, seed=0, gain=1.0):
    """Rows whose labels stand out by 0 to ln V + 3, weights of unit rows."""
    torch, g = T(), gen(seed)
    W = (torch.randn(V, D, generator=g, device="cuda") * D ** -0.5).to(dt(name))
    y = torch.randint(0, V, (rows,), generator=g, device="cuda")
    X = torch.randn(rows, D, generator=g, device="cuda")
    X += W[y].float() * torch.rand(rows, 1, generator=g, device="cuda") * (math.log(V) + 3)
    return (X * gain).to(dt(name)), W, y.int()


def teacher(rows, V, K, seed=1):
    torch, g = T(), gen(seed)
    K = min(K, V)
    start = torch.randint(0, V, (rows, 1), generator=g, device="cuda")
    step = torch.randint(1, max(2, V // K + 1), (rows, 1), generator=g, device="cuda")
    step = torch.clamp(step, max=max(1, V // K))
    ids = (start + step * torch.arange(K, device="cuda")) % V
    t = torch.randn(rows, K, generator=g, device="cuda") * 3
    return ids.int(), t


def reference(X, W, q_of, tau, rows_used, denom, chunk=2048):
    """Losses, gradients and their bounds' parts in 64 bits; q_of(a, b): dense
    targets of rows a .. b."""
    torch = T()
    Xd, Wd = X.double(), W.double()
    n = X.shape[0]
    V = W.shape[0]
    scale = tau / denom if denom else 0.0
    r = dict(rows=[], erow=[], dX=[], bX=[])
    dW = torch.zeros_like(Wd)
    bW = torch.zeros_like(Wd)
    r["K_W"] = n
    for a in range(0, n, chunk):
        b = min(n, a + chunk)
        use = rows_used[a:b, None]
        x = torch.where(use, Xd[a:b], torch.zeros((), dtype=torch.float64, device="cuda"))
        z = x @ Wd.t() / tau
        ez = X.shape[1] * E32 * (x.abs() @ Wd.abs().t()) / tau + E32 * z.abs()
        lp = torch.log_softmax(z, 1)
        q = q_of(a, b)
        p = lp.exp()
        rows = tau ** 2 * (torch.special.xlogy(q, q) - q * lp).sum(1)
        most = ez.amax(1)
        elp = 2 * most + (512 + V // 128) * E32
        size = (q * lp.abs() + torch.special.xlogy(q, q).abs()).sum(1)
        r["rows"].append(torch.where(use[:, 0], rows, 0.0))
        # q: differences of logits up to ~60 in size, exp and quotient
        r["erow"].append(tau ** 2 * (elp + 256 * E32 * (1 + size)))
        d = torch.where(use, p - q, 0.0)
        ed = torch.where(use, p * (elp[:, None] + 64 * E32) + q * 256 * E32, 0.0)
        if X.dtype == torch.bfloat16 and n > 128:
            ed = ed + torch.where(use, 2.0 ** -12 * p + 2.0 ** -25 * p.amax(1, keepdim=True), 0.0)
        r["dX"].append(scale * (d @ Wd))
        for u, key in ((None, "bX"),):
            r[key].append((d, ed))
        dW += scale * (d.t() @ x)
        bW += abs(scale) * (ed.t() @ x.abs())
        r.setdefault("dabs_W", torch.zeros_like(Wd)).add_(abs(scale) * (d.abs().t() @ x.abs()))
    r["bX"] = [(abs(scale) * (ed @ Wd.abs()), abs(scale) * (d.abs() @ Wd.abs()))
               for d, ed in r["bX"]]
    out = {"rows": torch.cat(r["rows"]), "erow": torch.cat(r["erow"]),
           "dX": torch.cat(r["dX"]), "dW": dW}
    out["edX"] = torch.cat([a for a, _ in r["bX"]])
    out["adX"] = torch.cat([a for _, a in r["bX"]])
    out["edW"], out["adW"] = bW, r["dabs_W"]
    out["loss"] = out["rows"].sum() / denom if denom else out["rows"].sum() * 0
    out["eloss"] = out["erow"].sum() / denom if denom else out["erow"].sum() * 0
    return out


def label_targets(y, V):
    torch = T()

    def q_of(a, b):
        q = torch.zeros(b - a, V, dtype=torch.float64, device="cuda")
        keep = y[a:b] >= 0
        q.scatter_(1, y[a:b].long().clamp(min=0)[:, None], keep[:, None].double())
        return q
    return q_of, y >= 0


def list_targets(ids, t, tau, V):
    torch = T()
    use = (ids >= 0) & (t != -math.inf)
    some = use.any(1)
    td = torch.where(use, t.double(), -math.inf)
    top = torch.where(some[:, None], td.amax(1, keepdim=True), 0.0)
    e = torch.where(use, ((td - top) / tau).exp(), 0.0)
    qk = torch.where(some[:, None], e / e.sum(1, keepdim=True), 0.0)

    def q_of(a, b):
        q = torch.zeros(b - a, V, dtype=torch.float64, device="cuda")
        return q.scatter_add_(1, ids[a:b].long().clamp(min=0), qk[a:b])
    return q_of, some


def within(got, want, bound, what):
    torch = T()
    assert got.shape == want.shape, what
    d = (got.double() - want).abs()
    assert torch.isfinite(got).all(), "%s: not finite" % what
    over = (d > bound).sum().item()
    worst = (d / bound.clamp(min=1e-300)).max().item() if d.numel() else 0.0
    assert over == 0, "%s: %d of %d past their bounds, worst %.2f times" % (
        what, over, d.numel(), worst)


def check_head(name, ref, V, got, two=False):
    loss, rows, dX, dW = got
    u = unit(name)
    ud = u * u if two else u
    within(rows, ref["rows"], ref["erow"] + E32, "row losses")
    within(loss[0], ref["loss"], ref["eloss"] + 4 * E32 * (1 + ref["loss"].abs()), "loss")
    n = rows.numel()
    if dX is not None:
        b = ref["edX"] * (1 + u) + ref["adX"] * (ud + (V + 64) * E32) * (1 + 2 * u)
        within(dX, ref["dX"], b + (u + 4 * E32) * ref["dX"].abs() + 1e-38, "dX")
    if dW is not None:
        b = ref["edW"] * (1 + u) + ref["adW"] * (ud + (2 * n + 64) * E32) * (1 + 2 * u)
        within(dW, ref["dW"], b + (u + 4 * E32) * ref["dW"].abs() + 1e-38, "dW")


def mask_rows(y, how, seed=5):
    torch = T()
    if how == "none":
        return y
    if how == "all":
        return torch.full_like(y, IGN)
    share = 0.95 if how == "most" else 0.4
    gone = torch.rand(y.shape, generator=gen(seed), device="cuda") < share
    return torch.where(gone, IGN, y)


# one row; sizes below, at and past tiles of 128 and 256, K blocks of 64 and
# the 128 rows of the two-term form; odd widths and vocabularies; thousands of
# statistics entries for few rows; enough tiles of 256 for every product; 1,024
# rows, up to which tiles of 32 and 64 are taken, on few columns
SHAPES = [(1, 1, 1), (1, 1000, 64), (3, 7, 5), (64, 130, 64), (65, 129, 63), (127, 1000, 96),
          (128, 257, 128), (129, 1000, 96), (256, 256, 64), (300, 515, 200), (257, 2049, 321),
          (1000, 513, 130), (300, 1360, 520), (1024, 900, 260), (1025, 900, 260),
          (2100, 300, 66), (5, 20000, 1024), (100, 140000, 64), (2049, 8200, 512),
          (4101, 4099, 1100)]


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D", SHAPES)
def test_loss_and_gradient(name, rows, V, D):
    X, W, y = head_inputs(name, rows, V, D, seed=rows + V)
    net = H.HFVocab(V, D, rows, name)
    for how in ("none", "some", "all"):
        yy = mask_rows(y, how)
        q_of, used = label_targets(yy, V)
        ref = reference(X, W, q_of, 1.0, used, int(used.sum()))
        check_head(name, ref, V, net.hf_vocab_loss_grad(X, W, yy),
                   two=name == "bf16" and rows <= 128)
        loss, rl = net.hf_vocab_loss(X, W, yy)
        check_head(name, ref, V, (loss, rl, None, None))
    net.hf_vocab_check()


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D,left", [
    (3000, 1500, 260, 300), (3000, 1500, 260, 1), (1500, 9000, 300, 700), (5000, 2000, 1024, 257),
    (20000, 1100, 520, 4000), (2300, 14000, 1200, 2300)])
def test_mostly_masked(name, rows, V, D, left):
    """A few counted rows of many: the row gradients' products take more splits
    than the grid was made for; and a matrix gradient with a last round of few
    tiles."""
    torch = T()
    X, W, y = head_inputs(name, rows, V, D, seed=left)
    at = torch.randperm(rows, generator=gen(left), device="cuda")[left:]
    y[at] = IGN
    X[at] = math.nan                       # what stands there must not matter
    net = H.HFVocab(V, D, rows, name)
    q_of, used = label_targets(y, V)
    ref = reference(X, W, q_of, 1.0, used, left)
    check_head(name, ref, V, net.hf_vocab_loss_grad(X, W, y))
    got = net.hf_vocab_loss_grad(X, W, y, need_dW=False)
    check_head(name, ref, V, (got[0], got[1], got[2], None))


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D,K,tau", [
    (1, 5, 3, 5, 1.0), (2, 1000, 64, 1, 2.0), (64, 130, 64, 16, 2.0), (129, 700, 63, 65, 0.5),
    (300, 2000, 128, 128, 4.0), (513, 257, 72, 100, 1.0), (700, 900, 256, 57, 1.0),
    (200, 600, 513, 70, 1.0)])
def test_distillation(name, rows, V, D, K, tau):
    torch = T()
    X, W, _ = head_inputs(name, rows, V, D, seed=rows)
    ids, t = teacher(rows, V, K)
    net = H.HFVocab(V, D, rows, name)
    for how in ("whole", "ragged"):
        if how == "ragged":
            end = torch.randint(0, ids.shape[1] + 1, (rows, 1), generator=gen(3), device="cuda")
            past = torch.arange(ids.shape[1], device="cuda")[None] >= end
            # what stands in masked places must not matter
            ids = torch.where(past, IGN, ids)
            t = torch.where(past, torch.where(ids == IGN, math.nan, t), t)
            clean = torch.where(past, 0.0, t)
        else:
            clean = t
        q_of, used = list_targets(ids, clean, tau, V)
        ref = reference(X, W, q_of, tau, used, int(used.sum()))
        check_head(name, ref, V, net.hf_vocab_distill_grad(X, W, ids, t, tau),
                   two=name == "bf16" and rows <= 128)
        loss, rl = net.hf_vocab_distill(X, W, ids, t, tau)
        check_head(name, ref, V, (loss, rl, None, None))
    net.hf_vocab_check()


def test_distillation_lists_with_repeats_and_lowest_values():
    """Ids listed two and three times, logits of -inf (masked) and of the
    type's lowest value (a place that counts: alone in its list, or against
    its like, it has all the probability), in any place."""
    torch = T()
    V, D, K = 50, 64, 8
    low = torch.finfo(torch.float32).min
    ids = torch.tensor([[3, 3, 4, 5, 3, 6, 6, 7], [9] * 8, [1, 2, 3, 4, 5, 6, 7, 8],
                        [0, 1, IGN, IGN, IGN, IGN, IGN, IGN], [10] + [IGN] * 7,
                        [11, 12, 13, 14, 15, 16, 17, 18], [20, 21, 22, 23, 24, 25, 26, 27]],
                       dtype=torch.int32, device="cuda")
    t = torch.randn(7, K, generator=gen(0), device="cuda")
    t[2, ::2] = -math.inf
    t[3, :2] = low
    t[4, 0] = low
    t[5] = -math.inf                       # nothing left: the row does not count
    t[6, 3] = low
    for name in ("fp32", "bf16"):
        for tau in (0.25, 1.0):
            X, W, _ = head_inputs(name, 7, V, D)
            net = H.HFVocab(V, D, 7, name)
            q_of, used = list_targets(ids, t, tau, V)
            assert int(used.sum()) == 6
            ref = reference(X, W, q_of, tau, used, 6)
            check_head(name, ref, V, net.hf_vocab_distill_grad(X, W, ids, t, tau),
                       two=name == "bf16")


@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_logits_in_pieces(name):
    """More logits than are kept: statistics first, then pieces of the
    vocabulary (with W packed, as its width is no multiple of 64, or not), for
    labels and lists."""
    torch = T()
    for rows, V, D in ((8000, 50257, 72), (4097, 100003, 64), (8000, 131075, 64)):
        X, W, y = head_inputs(name, rows, V, D)
        y = mask_rows(y, "some")
        net = H.HFVocab(V, D, rows, name)
        q_of, used = label_targets(y, V)
        ref = reference(X, W, q_of, 1.0, used, int(used.sum()), chunk=512)
        check_head(name, ref, V, net.hf_vocab_loss_grad(X, W, y))
        ids, t = teacher(rows, V, 20)
        q_of, used = list_targets(ids, t, 2.0, V)
        ref = reference(X, W, q_of, 2.0, used, int(used.sum()), chunk=512)
        check_head(name, ref, V, net.hf_vocab_distill_grad(X, W, ids, t, 2.0))
        del ref, net
        torch.cuda.empty_cache()


def test_matrix_packed_in_pieces():
    """A width that is no multiple of 64 and a matrix past what is packed at a
    time, with kept logits."""
    rows, V, D = 130, 50257, 1500
    X, W, y = head_inputs("fp32", rows, V, D)
    net = H.HFVocab(V, D, rows, "fp32")
    q_of, used = label_targets(y, V)
    check_head("fp32", reference(X, W, q_of, 1.0, used, rows), V,
               net.hf_vocab_loss_grad(X, W, y))


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [100, 300])
def test_masked_rows_reach_nothing(name, rows):
    """NaN and infinities in rows that do not count change no bit of any
    output."""
    torch = T()
    X, W, y = head_inputs(name, rows, 517, 96)
    y = mask_rows(y, "some")
    net = H.HFVocab(517, 96, rows, name)
    want = [o.clone() for o in net.hf_vocab_loss_grad(X, W, y)]
    Z = X.clone()
    Z[y < 0] = math.nan
    Z[(y < 0).nonzero()[::2, 0]] = math.inf
    for a, b in zip(want, net.hf_vocab_loss_grad(Z, W, y)):
        assert torch.equal(a, b)
    assert (want[2][y < 0] == 0).all() and (want[1][y < 0] == 0).all()


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D", [(50, 300, 64), (200, 300, 64), (200, 301, 100)])
def test_strides_and_alignment(name, rows, V, D):
    """Rows apart by odd and even strides, starting at any element: the bits of
    the contiguous call, and nothing written beside the outputs."""
    torch = T()
    X, W, y = head_inputs(name, rows, V, D)
    net = H.HFVocab(V, D, rows, name)
    want = [o.clone() for o in net.hf_vocab_loss_grad(X, W, y)]
    for pad, at in ((1, 1), (8, 8), (3, 0), (64, 3)):
        def wide(t):
            w = torch.full((t.shape[0], D + pad + at), 7.0, device="cuda", dtype=t.dtype)
            w[:, at:at + D] = t
            return w
        xs, ws = wide(X), wide(W)
        dxs, dws = wide(X * 0), wide(W * 0)
        got = net.hf_vocab_loss_grad(xs[:, at:at + D], ws[:, at:at + D], y,
                                     dX=dxs[:, at:at + D], dW=dws[:, at:at + D])
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        for w in (dxs, dws):
            assert (w[:, :at] == 7).all() and (w[:, at + D:] == 7).all()


def test_partial_gradients_denominator_and_accumulation():
    torch = T()
    rows, V, D = 150, 400, 64
    for name in ("fp32", "bf16"):
        X, W, y = head_inputs(name, rows, V, D)
        y = mask_rows(y, "some")
        n = int((y >= 0).sum())
        net = H.HFVocab(V, D, rows, name)
        loss, rl, dX, dW = net.hf_vocab_loss_grad(X, W, y)
        _, _, a, b = net.hf_vocab_loss_grad(X, W, y, need_dW=False)
        assert b is None and torch.equal(a, dX)
        _, _, a, b = net.hf_vocab_loss_grad(X, W, y, need_dX=False)
        assert a is None and torch.equal(b, dW)
        # denom given: 2 n halves everything (by a power of two)
        half = net.hf_vocab_loss_grad(X, W, y, denom=2.0 * n)
        assert torch.equal(half[0] * 2, loss) and torch.equal(half[1], rl)
        assert torch.equal(half[2].float() * 2, dX.float())
        assert torch.equal(half[3].float() * 2, dW.float())
        # dW += : one rounding of the sum
        q_of, used = label_targets(y, V)
        ref = reference(X, W, q_of, 1.0, used, n)
        old = torch.randn(V, D, generator=gen(9), device="cuda").to(dt(name)) * 0.1
        got = net.hf_vocab_loss_grad(X, W, y, dW=old.clone(), accumulate=True)[3]
        u = unit(name)
        sum_ = ref["dW"] + old.double()
        within(got, sum_, ref["edW"] * 2 + ref["adW"] * (u + 512 * E32) * 2 +
               (u + 4 * E32) * sum_.abs() + E32 * old.double().abs(), "dW +=")
        with pytest.raises(ValueError):
            net.hf_vocab_loss_grad(X, W, y, accumulate=True)


@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_no_rows(name):
    torch = T()
    V, D = 100, 70
    net = H.HFVocab(V, D, 16, name)
    W = torch.randn(V, D, device="cuda").to(dt(name))
    X = torch.empty(0, D, device="cuda", dtype=dt(name))
    y = torch.empty(0, dtype=torch.int32, device="cuda")
    loss, rl, dX, dW = net.hf_vocab_loss_grad(X, W, y)
    assert loss.item() == 0 and rl.numel() == 0 and dX.shape == (0, D) and (dW == 0).all()
    kept = torch.ones_like(W)
    net.hf_vocab_loss_grad(X, W, y, dW=kept, accumulate=True)
    assert (kept == 1).all()
    assert net.hf_vocab_embed(W, y).shape == (0, D)
    assert (net.hf_vocab_embed_grad(y, X) == 0).all()
    net.hf_vocab_check()


def test_labels_outside_are_reported():
    torch = T()
    X, W, y = head_inputs("fp32", 40, 30, 64)
    net = H.HFVocab(30, 64, 40, "fp32")
    for bad in (30, -1, -101, 2 ** 31 - 1):
        yy = y.clone()
        yy[7] = bad
        got = [o.clone() for o in net.hf_vocab_loss_grad(X, W, yy)]
        with pytest.raises(H.HFError) as e:
            net.hf_vocab_check()
        assert e.value.code == H.HF_ELABEL
        net.hf_vocab_check()               # reported once
        yy[7] = IGN                        # counts as masked
        for a, b in zip(got, net.hf_vocab_loss_grad(X, W, yy)):
            assert torch.equal(a, b)
        net.hf_vocab_check()
        ids = y[:, None].repeat(1, 3).clone()
        ids[5, 1] = bad
        net.hf_vocab_distill(X, W, ids, torch.zeros(40, 3, device="cuda"))
        with pytest.raises(H.HFError):
            net.hf_vocab_check()
        tok = y.clone()
        tok[0] = bad
        assert (net.hf_vocab_embed(W, tok)[0] == 0).all()
        with pytest.raises(H.HFError):
            net.hf_vocab_check()
        net.hf_vocab_embed_grad(tok, X)
        with pytest.raises(H.HFError):
            net.hf_vocab_check()


def test_binding_refuses():
    torch = T()
    X, W, y = head_inputs("bf16", 8, 20, 64)
    net = H.HFVocab(20, 64, 8, "bf16")
    for args in ((X.float(), W, y), (X, W.float(), y), (X, W, y.long()), (X.cpu(), W, y),
                 (X, W, y.cpu())):
        with pytest.raises(TypeError):
            net.hf_vocab_loss_grad(*args)
    for args in ((X[:, :32], W, y), (X, W[:10], y), (X, W, y[:5]),
                 (X.t().contiguous().t(), W, y)):
        with pytest.raises(ValueError):
            net.hf_vocab_loss_grad(*args)
    with pytest.raises(H.HFError) as e:
        net.hf_vocab_loss_grad(X.repeat(2, 1), W, y.repeat(2))
    assert e.value.code == H.HF_EINVAL
    small = H.HFVocab(20, 64, 4096, "bf16", ws_rows=8)
    small.hf_vocab_loss(X, W, y)
    with pytest.raises(H.HFError) as e:
        small.hf_vocab_loss(X.repeat(512, 1), W, y.repeat(512))
    assert e.value.code == H.HF_EWORKSPACE
    for kw in (dict(need_dX=False, need_dW=False), dict(dX=X), dict(dW=W)):
        with pytest.raises(H.HFError) as e:       # nothing to do, or in place
            net.hf_vocab_loss_grad(X, W, y, **kw)
        assert e.value.code == H.HF_EINVAL
    with pytest.raises(H.HFError):
        net.hf_vocab_embed(W, y, out=W[:8])


def test_gradient_against_differences():
    """<grad, U> against (f(+hU) - f(-hU)) / 2h in fp32.  The difference is off
    by h^2 / 6 times the third derivative along U and by the losses' own bounds
    over h.  That derivative is tau^2 times the third cumulant of the logits'
    movement over tau under p; for a movement within +-m it is at most
    (2 m)^3 / (6 sqrt 3)."""
    torch = T()
    rows, V, D, h = 40, 200, 64, 2.0 ** -5
    X, W, y = head_inputs("fp32", rows, V, D, seed=4)
    ids, t = teacher(rows, V, 10)
    net = H.HFVocab(V, D, rows, "fp32")
    U = torch.randn(rows, D, generator=gen(1), device="cuda")
    U /= U.norm(dim=1, keepdim=True)
    Y = torch.randn(V, D, generator=gen(2), device="cuda")
    Y /= Y.norm(dim=1, keepdim=True) * X.norm(dim=1).max()
    for f, targets in ((net.hf_vocab_loss, (y,)), (net.hf_vocab_distill, (ids, t, 2.0))):
        hard = len(targets) == 1
        grad = net.hf_vocab_loss_grad if hard else net.hf_vocab_distill_grad
        loss, _, dX, dW = grad(X, W, *targets)
        q_of, used = label_targets(y, V) if hard else list_targets(ids, t, 2.0, V)
        tau = 1.0 if hard else 2.0
        err = reference(X, W, q_of, tau, used, rows)["eloss"].item() + 4 * E32 * 10
        for G, A, B in ((dX, (X + h * U, W), (X - h * U, W)), (dW, (X, W + h * Y), (X, W - h * Y))):
            D_ = U if G is dX else Y
            num = (f(*A, *targets)[0].double() - f(*B, *targets)[0].double()).item() / (2 * h)
            ana = (G.double() * D_.double()).sum().item()
            # inputs X +- hU are rounded too: their relative e over h, times |grad|
            rnd = E32 / h * (G.double().abs() * (X if G is dX else W).double().abs()).sum().item()
            m = max((U @ W.t()).abs().max(), (X @ Y.t()).abs().max()).item() / tau
            third = tau ** 2 * (2 * m) ** 3 / (6 * math.sqrt(3))
            assert abs(num - ana) <= h * h / 6 * third + err / h + rnd, (num, ana)


def test_large_logits():
    """Logits of thousands: probabilities of 0 and 1, no overflow."""
    for name in ("fp32", "bf16"):
        X, W, y = head_inputs(name, 70, 300, 64, gain=600.0)
        net = H.HFVocab(300, 64, 70, name)
        q_of, used = label_targets(y, 300)
        ref = reference(X, W, q_of, 1.0, used, 70)
        check_head(name, ref, 300, net.hf_vocab_loss_grad(X, W, y), two=name == "bf16")


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D", [(100, 1000, 128), (700, 1500, 200), (4200, 70000, 64),
                                      (8200, 131100, 64)])
def test_same_bits(name, rows, V, D):
    """Repeated calls, another workspace, another stream."""
    torch = T()
    X, W, y = head_inputs(name, rows, V, D)
    net = H.HFVocab(V, D, rows, name)
    want = [o.clone() for o in net.hf_vocab_loss_grad(X, W, y)]
    for a, b in zip(want, net.hf_vocab_loss_grad(X, W, y)):
        assert torch.equal(a, b)
    big = H.HFVocab(V, D, 3 * rows, name)
    big.workspace.fill_(0xff)              # NaN wherever nothing is written first
    big._check(H.lib().hf_vocab_set_workspace(big._h, big.workspace.data_ptr(),
                                              big.workspace.numel()))
    for a, b in zip(want, big.hf_vocab_loss_grad(X, W, y)):
        assert torch.equal(a, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = net.hf_vocab_loss_grad(X, W, y)
    # back on the first stream at once: the context orders its workspace's use
    again = net.hf_vocab_loss_grad(X, W, y)
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [200, 3000])
def test_captured_and_replayed(name, rows):
    """Loss, distillation, embedding and their gradients in one graph, replayed
    on new inputs and masks between eager calls of the same context."""
    torch = T()
    V, D, K = 1100, 96, 12
    net = H.HFVocab(V, D, rows, name)
    X, W, y = head_inputs(name, rows, V, D)
    ids, t = teacher(rows, V, K)

    def work():
        a = net.hf_vocab_embed(W, y, 3.0)
        b = net.hf_vocab_loss_grad(X, W, y)
        c = net.hf_vocab_distill_grad(X, W, ids, t, 2.0)
        d = net.hf_vocab_embed_grad(y, X, 3.0)
        return [a, *b, *c, d]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        work()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = work()
    for seed in range(4):
        nX, nW, ny = head_inputs(name, rows, V, D, seed=20 + seed)
        X.copy_(nX)
        W.copy_(nW)
        y.copy_(mask_rows(ny, ("none", "some", "most", "all")[seed]))
        g.replay()
        got = [o.clone() for o in outs]
        torch.cuda.synchronize()
        for a, b in zip(got, work()):
            assert torch.equal(a, b), seed
        torch.cuda.synchronize()


# ---------------------------------------------------------------- embedding

def zipf(n, V, seed=0):
    torch = T()
    r = torch.rand(n, generator=gen(seed), device="cuda")
    return (torch.exp(r * math.log(V + 1.0)) - 1).long().clamp_(0, V - 1).int()


@pytest.mark.parametrize("name", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,D", [(1, 1, 1), (1, 100, 4096), (5, 10, 3), (63, 50, 257),
                                      (1000, 5000, 64), (1024, 4096, 520), (1025, 4095, 130),
                                      (500, 80, 8), (500, 80, 9), (2000, 70, 255), (1200, 90, 511),
                                      (1200, 90, 513), (1200, 90, 519), (1100, 60, 1021),
                                      (20000, 1000, 72), (30011, 200003, 24), (30011, 120000, 1024),
                                      (20000, 140000, 1021)])
def test_embedding_and_gradient(name, rows, V, D):
    torch = T()
    u = unit(name)
    E = torch.randn(V, D, generator=gen(rows), device="cuda").to(dt(name))
    dout = torch.randn(rows, D, generator=gen(rows + 1), device="cuda").to(dt(name))
    net = H.HFVocab(V, D, rows, name)
    for how in ("zipf", "masked", "one", "none"):
        tok = {"zipf": lambda: zipf(rows, V), "masked": lambda: mask_rows(zipf(rows, V), "some"),
               "one": lambda: torch.full((rows,), V - 1, dtype=torch.int32, device="cuda"),
               "none": lambda: torch.full((rows,), IGN, dtype=torch.int32, device="cuda")}[how]()
        keep = tok >= 0
        at = tok.long().clamp(min=0)
        for scale in (1.0, -2.7):
            s32 = float(torch.tensor(scale, dtype=torch.float32))
            want = E[at].double() * s32 * keep[:, None]
            within(net.hf_vocab_embed(E, tok, scale), want, (u + E32) * want.abs(), "embedding")
            want = torch.zeros(V, D, dtype=torch.float64, device="cuda")
            size, n = want.clone(), torch.zeros(V, 1, dtype=torch.float64, device="cuda")
            want.index_add_(0, at[keep], dout[keep].double() * s32)
            size.index_add_(0, at[keep], dout[keep].double().abs() * abs(s32))
            n.index_add_(0, at[keep], torch.ones(int(keep.sum()), 1, dtype=torch.float64,
                                                 device="cuda"))
            got = net.hf_vocab_embed_grad(tok, dout, scale)
            bound = size * (n + 2) * E32 * (1 + 2 * u) + u * want.abs()
            within(got, want, bound, "embedding gradient, " + how)
            assert torch.equal(got, net.hf_vocab_embed_grad(tok, dout, scale))
            old = torch.randn(V, D, generator=gen(3), device="cuda").to(dt(name))
            got = net.hf_vocab_embed_grad(tok, dout, scale, dE=old.clone(), accumulate=True)
            sum_ = want + old.double()
            within(got, sum_, bound + u * sum_.abs() + E32 * old.double().abs(), "dE +=")
            absent = torch.ones(V, dtype=torch.bool, device="cuda")
            absent[at[keep]] = False
            assert torch.equal(got[absent], old[absent])
    net.hf_vocab_check()


@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_embedding_strides(name):
    torch = T()
    rows, V, D = 1500, 300, 100
    E = torch.randn(V, D, generator=gen(0), device="cuda").to(dt(name))
    dout = torch.randn(rows, D, generator=gen(1), device="cuda").to(dt(name))
    tok = mask_rows(zipf(rows, V), "some")
    net = H.HFVocab(V, D, rows, name)
    want, grad = net.hf_vocab_embed(E, tok, 1.5), net.hf_vocab_embed_grad(tok, dout, 1.5)
    for pad, at in ((1, 1), (12, 8), (3, 0)):
        def wide(t, fill=False):
            w = torch.full((t.shape[0], D + pad + at), 7.0, device="cuda", dtype=t.dtype)
            if not fill:
                w[:, at:at + D] = t
            return w
        o, de = wide(want, True), wide(E, True)
        net.hf_vocab_embed(wide(E)[:, at:at + D], tok, 1.5, out=o[:, at:at + D])
        net.hf_vocab_embed_grad(tok, wide(dout)[:, at:at + D], 1.5, dE=de[:, at:at + D])
        assert torch.equal(o[:, at:at + D], want) and torch.equal(de[:, at:at + D], grad)
        for w in (o, de):
            assert (w[:, :at] == 7).all() and (w[:, at + D:] == 7).all()


def test_masked_gradient_rows_reach_nothing():
    torch = T()
    rows, V, D = 3000, 40, 64
    tok = mask_rows(zipf(rows, V), "some")
    dout = torch.randn(rows, D, generator=gen(0), device="cuda")
    net = H.HFVocab(V, D, rows, "fp32")
    want = net.hf_vocab_embed_grad(tok, dout)
    dout[tok < 0] = math.nan
    assert torch.equal(want, net.hf_vocab_embed_grad(tok, dout))


@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_limits(name):
    """The widest rows, the largest vocabulary, the most rows."""
    torch = T()
    for rows, V, D in ((3, 9, H.HF_VOCAB_MAX_WIDTH), (5, H.HF_VOCAB_MAX, 8),
                       (H.HF_VOCAB_MAX_ROWS, 3, 4)):
        X, W, y = head_inputs(name, rows, V, D)
        y = mask_rows(y, "some") if rows > 100 else y
        net = H.HFVocab(V, D, rows, name)
        q_of, used = label_targets(y, V)
        ref = reference(X, W, q_of, 1.0, used, int(used.sum()), chunk=1 << 18)
        check_head(name, ref, V, net.hf_vocab_loss_grad(X, W, y), two=rows <= 128)
        emb = net.hf_vocab_embed(W, y, 2.0)
        keep = y >= 0
        assert torch.equal(emb, W[y.long().clamp(min=0)] * 2 * keep[:, None])
        # whole numbers: their sums are exact in fp32, in any order
        whole = torch.randint(-2, 3, X.shape, generator=gen(1), device="cuda").to(X.dtype)
        want = torch.zeros(V, D, dtype=torch.float64, device="cuda")
        want.index_add_(0, y[keep].long(), whole[keep].double())
        assert torch.equal(net.hf_vocab_embed_grad(y, whole), want.to(X.dtype))
        del net, ref, want
        torch.cuda.empty_cache()


def test_two_contexts_on_two_streams():
    """Contexts share nothing: both working at once give the bits of each
    alone."""
    torch = T()
    jobs = []
    for k, (rows, V, D) in enumerate(((900, 5000, 256), (60, 9000, 320))):
        X, W, y = head_inputs("bf16", rows, V, D, seed=k)
        net = H.HFVocab(V, D, rows, "bf16")
        want = [o.clone() for o in net.hf_vocab_loss_grad(X, W, y)]
        want.append(net.hf_vocab_embed_grad(y, X).clone())
        jobs.append((net, X, W, y, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, (net, X, W, y, want, s) in enumerate(jobs):
            with torch.cuda.stream(s):
                got[k] = [*net.hf_vocab_loss_grad(X, W, y), net.hf_vocab_embed_grad(y, X)]
    torch.cuda.synchronize()
    for k in range(2):
        for a, b in zip(jobs[k][4], got[k]):
            assert torch.equal(a, b)


# ------------------------------------------------------------- all together

@pytest.mark.parametrize("name", ["fp32", "bf16"])
def test_tied_token_model(name):
    """Tokens to their embeddings, the rows through the head with the next
    token as label, and both gradients into the one tied matrix, against the
    same in 64 bits from the bits the calls pass on."""
    torch = T()
    rows, V, D = 400, 900, 128
    s = math.sqrt(D)
    E = (torch.randn(V, D, generator=gen(0), device="cuda") * D ** -0.5).to(dt(name))
    tok = zipf(rows, V, 1)
    y = mask_rows(zipf(rows, V, 2), "some")
    net = H.HFVocab(V, D, rows, name)
    X = net.hf_vocab_embed(E, tok, s)
    loss, rl, dX, dE = net.hf_vocab_loss_grad(X, E, y)
    head = dE.clone()
    net.hf_vocab_embed_grad(tok, dX, s, dE=dE, accumulate=True)
    net.hf_vocab_check()
    q_of, used = label_targets(y, V)
    check_head(name, reference(X, E, q_of, 1.0, used, int(used.sum())), V,
               (loss, rl, dX, head))
    s32 = float(torch.tensor(s, dtype=torch.float32))
    u = unit(name)
    want = head.double().index_add_(0, tok.long(), dX.double() * s32)
    size = torch.zeros_like(want).index_add_(0, tok.long(), dX.double().abs() * s32)
    within(dE, want, size * (rows + 2) * E32 + (u + E32) * want.abs() +
           E32 * head.double().abs(), "tied gradient")
    # a step down the gradient of the whole model lowers its loss (a small one:
    # by about its length times the gradient's)
    if name == "fp32":
        h = 1e-2 / dE.norm()
        E2 = E - h * dE
        new = net.hf_vocab_loss(net.hf_vocab_embed(E2, tok, s), E2, y)[0]
        assert new.item() < loss.item()


def test_head_matches_the_net(tmp_path):
    """A vocabulary within HF_MAX_CLASSES: the head against HFNet's output
    layer (one weight layer, its bias zero), loss and gradient, within both
    calls' bounds."""
    torch = T()
    rows, V, D = 300, 700, 96
    X, W, y = head_inputs("fp32", rows, V, D)
    net = H.HFNet((D, V), "tanh", rows)
    theta = torch.cat([W.reshape(-1), torch.zeros(V, device="cuda")])
    f, g = net.hf_loss_grad(theta, X, y)
    loss, _, _, dW = H.HFVocab(V, D, rows, "fp32").hf_vocab_loss_grad(X, W, y)
    q_of, used = label_targets(y, V)
    ref = reference(X, W, q_of, 1.0, used, rows)
    within(loss, f.double(), 2 * ref["eloss"] + 8 * E32 * f.double(), "loss")
    b = 2 * (ref["edW"] + ref["adW"] * (2 * rows + 64) * E32) + 8 * E32 * ref["dW"].abs() + 1e-38
    within(dW, g[:V * D].view(V, D).double(), b, "dW")
