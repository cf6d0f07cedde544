"""The vocabulary ends of a token model, as cases that can be timed: the token
embedding and its gradient, the softmax cross-entropy head over a large
vocabulary, and distillation from a teacher's top logits.

A case: ``op`` ("xent", "xent_grad", "distill_grad", "embed" or "embed_grad"),
``type`` ("fp32" or "bf16", of the rows, the matrices and their gradients),
``rows`` (tokens), ``vocab`` and ``width``; for distillation ``top`` logits per
row and the temperature ``tau``; ``masked``, the share of rows (and, for the
teacher's lists, of slots) that are padding.
"""

import math

import torch

own = False

IGNORE = -100
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _case(op, type, rows, vocab, width, top=0, tau=1.0, masked=0.0, name=None):
    c = dict(op=op, type=type, rows=rows, vocab=vocab, width=width, top=top,
             tau=tau, masked=masked)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the few target tokens of a short answer under a masked prompt
        _case("xent_grad", "bf16", 5, 32000, 1024, name="xent_grad_few"),
        # evaluation: the loss alone, on a vocabulary of odd size
        _case("xent", "bf16", 4096, 50257, 768, name="xent_eval"),
        # a ragged minibatch with a quarter of its rows padding, on a width
        # that no vector load divides
        _case("xent_grad", "bf16", 3001, 50257, 1021, masked=0.25,
              name="xent_grad_ragged"),
        # the head of a large model on a full minibatch
        _case("xent_grad", "bf16", 8192, 131072, 4096, name="xent_grad_large"),
        # the output layer of the speech-frame net on its full minibatch
        _case("xent_grad", "fp32", 16384, 1973, 2048, name="xent_grad_speech_fp32"),
        # fine-tuning a student on a short prompt's answers
        _case("distill_grad", "bf16", 64, 32000, 1024, top=16, tau=2.0,
              name="distill_grad_short"),
        # a single-precision student with ragged teacher lists
        _case("distill_grad", "fp32", 777, 50257, 512, top=32, tau=1.0, masked=0.2,
              name="distill_grad_fp32"),
        # a distillation minibatch
        _case("distill_grad", "bf16", 4096, 65536, 2048, top=64, tau=2.0,
              masked=0.1, name="distill_grad_large"),
        # one decoded token's embedding
        _case("embed", "bf16", 1, 32000, 1024, name="embed_one"),
        # a large minibatch's embeddings
        _case("embed", "bf16", 65536, 131072, 4096, masked=0.1, name="embed_large"),
        # the embedding gradient of a small minibatch of ragged length
        _case("embed_grad", "fp32", 10007, 50257, 768, masked=0.1,
              name="embed_grad_fp32"),
        # and of a large one
        _case("embed_grad", "bf16", 131072, 131072, 2048, masked=0.1,
              name="embed_grad_large"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("xent", "xent_grad", "xent_grad", "distill_grad",
                     "distill_grad", "embed", "embed_grad"))
    type = rng.choice(("bf16", "bf16", "fp32"))
    masked = rng.choice((0.0, 0.0, 0.1, 0.5))
    vocab = _log_int(rng, 1000, 131072)
    width = _log_int(rng, 64, 4096)
    if rng.random() < 0.7:      # most models' widths are multiples of 64
        width = max(64, width // 64 * 64)
    if op in ("embed", "embed_grad"):
        return _case(op, type, _log_int(rng, 1, 65536), vocab, width, masked=masked)
    # the plain form computes in 32 bits for either type
    most = 4e12 / (vocab * width)
    rows = _log_int(rng, 1, max(1, min(16384, most, 1e9 / vocab)))
    if op == "distill_grad":
        return _case(op, type, rows, vocab, width, top=_log_int(rng, 4, 128),
                     tau=rng.choice((1.0, 2.0, 4.0)), masked=masked)
    return _case(op, type, rows, vocab, width, masked=masked)


# ------------------------------------------------------------------- inputs

def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    T, V, D = case["rows"], case["vocab"], case["width"]
    dt = TYPES[case["type"]]
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")     # noqa: E731
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    # tokens as text has them: the r-th commonest about as often as 1 / r
    zipf = lambda n: (torch.exp(rand(n) * math.log(V + 1.0)) - 1).long().clamp_(0, V - 1)   # noqa: E731
    gone = rand(T) < case["masked"]
    tok = zipf(T)
    s = {}
    if case["op"] in ("embed", "embed_grad"):
        s["tok"] = torch.where(gone, IGNORE, tok).int()
        s["scale"] = math.sqrt(D)
        if case["op"] == "embed":
            s["E"] = (randn(V, D) * D ** -0.5).to(dt)
        else:
            s["dout"] = (randn(T, D) / T).to(dt)
        return s
    # rows of unit size; the label's logit stands out by up to ln V + 3, so
    # that some rows are learnt and some are not
    W = (randn(V, D) * D ** -0.5).to(dt)
    X = randn(T, D) + W[tok].float() * (rand(T, 1) * (math.log(V) + 3))
    s["W"], s["X"] = W, X.to(dt)
    if case["op"] != "distill_grad":
        s["y"] = torch.where(gone, IGNORE, tok).int()
        return s
    K = case["top"]
    # K different tokens a row, the first of them the likeliest
    step = (rand(T, 1) * (V // K - 1)).long() + 1
    ids = (tok[:, None] + step * torch.arange(K, device="cuda")) % V
    t = (randn(T, K) * 3).sort(1, descending=True)[0]
    # lists end early, and whole rows are padding
    n = torch.where(rand(T) < case["masked"], rand(T) * K, K + 1.0)
    empty = (torch.arange(K, device="cuda")[None] >= n[:, None]) | gone[:, None]
    s["ids"] = torch.where(empty, IGNORE, ids).int()
    s["t"] = t
    return s


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    if own:
        from paper_1606_00511_amd.hf import HFVocab
        s["net"] = HFVocab(case["vocab"], case["width"], case["rows"], case["type"])
    return s


# ------------------------------------------------------------- one pass

def _own(s):
    case, net = s["case"], s["net"]
    if case["op"] == "xent":
        loss, rows = net.hf_vocab_loss(s["X"], s["W"], s["y"])
        return {"loss": loss, "rows": rows}
    if case["op"] == "embed":
        return {"out": net.hf_vocab_embed(s["E"], s["tok"], s["scale"])}
    if case["op"] == "embed_grad":
        return {"dE": net.hf_vocab_embed_grad(s["tok"], s["dout"], s["scale"])}
    if case["op"] == "xent_grad":
        loss, rows, dX, dW = net.hf_vocab_loss_grad(s["X"], s["W"], s["y"])
    else:
        loss, rows, dX, dW = net.hf_vocab_distill_grad(s["X"], s["W"], s["ids"], s["t"],
                                                       case["tau"])
    return {"loss": loss, "rows": rows, "dX": dX, "dW": dW}


def run(s):
    if own:
        return _own(s)
    case = s["case"]
    op, dt = case["op"], TYPES[case["type"]]
    if op == "embed":
        keep = s["tok"] >= 0
        rows = s["E"][s["tok"].clamp(min=0)].float() * s["scale"]
        return {"out": (rows * keep[:, None]).to(dt)}
    if op == "embed_grad":
        keep = s["tok"] >= 0
        rows = s["dout"].float() * (keep[:, None] * s["scale"])
        dE = torch.zeros(case["vocab"], case["width"], device="cuda")
        return {"dE": dE.index_add_(0, s["tok"].clamp(min=0), rows).to(dt)}
    X, W, tau = s["X"].float(), s["W"].float(), case["tau"]
    z = X @ W.t()
    if tau != 1:
        z = z / tau
    m = z.amax(1, keepdim=True)
    p = torch.exp(z - m)
    total = p.sum(1, keepdim=True)
    lse = m + torch.log(total)
    if op == "distill_grad":
        have = s["ids"] >= 0
        ids = s["ids"].long().clamp(min=0)
        keep = have.any(1)
        t = torch.where(have, s["t"] / tau, -math.inf)
        top = torch.where(keep[:, None], t.amax(1, keepdim=True), 0.0)
        e = torch.exp(t - top)
        sum_e = torch.where(keep[:, None], e.sum(1, keepdim=True), 1.0)
        q = e / sum_e
        log_q = torch.where(have, t - top - torch.log(sum_e), 0.0)
        rows = tau * tau * (q * (log_q - (z.gather(1, ids) - lse))).sum(1)
    else:
        keep = s["y"] >= 0
        ids = s["y"].long().clamp(min=0)[:, None]
        q = keep[:, None].float()
        rows = (lse - z.gather(1, ids))[:, 0] * keep
    n = keep.sum().clamp(min=1)
    loss = (rows.double().sum() / n).float().reshape(1)
    if op == "xent":
        return {"loss": loss, "rows": rows}
    p = p * (keep[:, None] / total)
    p.scatter_add_(1, ids, -q)
    p *= tau / n
    return {"loss": loss, "rows": rows, "dX": (p @ W).to(dt), "dW": (p.t() @ X).to(dt)}


# -------------------------------------------------------------------- work

def work(case):
    T, V, D, K = case["rows"], case["vocab"], case["width"], case["top"]
    b = 4 if case["type"] == "fp32" else 2
    if case["op"] == "embed":
        return {"bytes": 4 * T + 2 * b * T * D, "flops": T * D}
    if case["op"] == "embed_grad":
        return {"bytes": 4 * T + b * (T + V) * D, "flops": 2 * T * D}
    targets = 8 * T * K if K else 4 * T
    if case["op"] == "xent":
        return {"bytes": b * (T + V) * D + targets + 4 * T, "flops": 2 * T * V * D}
    return {"bytes": 2 * b * (T + V) * D + targets + 4 * T, "flops": 6 * T * V * D}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    """The definitions in 64 bits, a block of rows at a time."""
    s = _inputs(case, seed)
    op, T, V, D = case["op"], case["rows"], case["vocab"], case["width"]
    if op == "embed":
        out = torch.zeros(T, D, dtype=torch.float64, device="cuda")
        at = torch.nonzero(s["tok"] != IGNORE)[:, 0]
        out[at] = s["E"].index_select(0, s["tok"][at]).double() * s["scale"]
        return {"out": out}
    if op == "embed_grad":
        dE = torch.zeros(V, D, dtype=torch.float64, device="cuda")
        at = torch.nonzero(s["tok"] != IGNORE)[:, 0]
        dE.index_add_(0, s["tok"][at], s["dout"][at].double())
        return {"dE": dE * s["scale"]}
    tau = case["tau"]
    W = s["W"].double()
    if op == "distill_grad":
        use = (s["ids"] != IGNORE)
        logits = torch.where(use, s["t"].double() / tau, -torch.inf)
        some = use.any(1)
        q = torch.zeros_like(logits)
        q[some] = torch.softmax(logits[some], 1)
        at = torch.where(use, s["ids"].long(), 0)
    else:
        some = s["y"] != IGNORE
        at = torch.where(some, s["y"].long(), 0)[:, None]
        q = some[:, None].double()
    n = max(1, int(some.sum()))
    rows = torch.zeros(T, dtype=torch.float64, device="cuda")
    grad = op != "xent"
    if grad:
        dX = torch.zeros(T, D, dtype=torch.float64, device="cuda")
        dW = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for b in range(0, T, 1024):
        e = min(T, b + 1024)
        X = s["X"][b:e].double()
        log_p = torch.log_softmax(X @ W.t() / tau, 1)
        qb = q[b:e]
        rows[b:e] = tau ** 2 * (torch.special.xlogy(qb, qb) - qb * log_p.gather(1, at[b:e])).sum(1)
        if grad:
            d = log_p.exp_()
            d[~some[b:e]] = 0
            d.scatter_add_(1, at[b:e], -qb)
            d *= tau / n
            dX[b:e] = d @ W
            dW += d.t() @ X
    out = {"loss": (rows.sum() / n).reshape(1), "rows": rows}
    if grad:
        out.update(dX=dX, dW=dW)
    return out
