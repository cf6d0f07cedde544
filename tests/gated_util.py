"""Plain forms of the gated block in 64 bits, and bounds of what the types may
cost.

A rounding to a type is off by at most U[type] of the value.  A sum of n
products in fp32 is off by at most n 2^-24 of the sum of magnitudes (n 2^-24
also covers the sums' own rounding); the bounds below count every rounding with
the magnitudes it acts on, so they hold element by element.
"""

import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
S = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
# an activation and its slope are off by at most so much of their scale
# (|z| + 1, and 1): fp32's exp, tanh and erfc are within a few units of the last
# place (8 with the products around them); what is rounded to bf16 afterwards
# uses exp2 and reciprocals of one unit on arguments rounded once, |z| 2^-24 of
# them for |z| up to 20 (beyond, the sigmoid is 0 or 1 to 2^-24): 64 units
ACT_OFF = {torch.float32: 8 * S, torch.bfloat16: 64 * S}
# bounds of the slopes of the activations and of their slopes' slopes
SLOPE, BEND = 1.13, 1.2


def act(name, z):
    f = torch.nn.functional
    return {"silu": f.silu, "gelu": f.gelu, "sigmoid": torch.sigmoid, "tanh": torch.tanh,
            "relu": torch.relu, "gelu_tanh": lambda v: f.gelu(v, approximate="tanh")}[name](z)


def slope(name, z):
    z = z.detach().clone().requires_grad_()
    return torch.autograd.grad(act(name, z).sum(), z)[0]


def block(name, X, Wg, Wu, Wd):
    """(Y, G, U, H) in 64 bits."""
    X, Wg, Wu, Wd = (t.double() for t in (X, Wg, Wu, Wd))
    G, U_ = X @ Wg.t(), X @ Wu.t()
    H = act(name, G) * U_
    return H @ Wd.t(), G, U_, H


def block_bound(name, X, Wg, Wu, Wd, two_term=False):
    """Elementwise bounds (of Y, G, U) for X's type."""
    dt = X.dtype
    D, F = Wg.shape[1], Wg.shape[0]
    Y, G, U_, H = block(name, X, Wg, Wu, Wd)
    aX, aG, aU, aD = (t.double().abs() for t in (X, Wg, Wu, Wd))
    dg, du = (D * S) * (aX @ aG.t()), (D * S) * (aX @ aU.t())
    A = act(name, G).abs() + ACT_OFF[dt] * (G.abs() + 1)
    dA = SLOPE * dg + ACT_OFF[dt] * (G.abs() + 1)
    dH = dA * (U_.abs() + du) + A * du + S * H.abs()
    # h is rounded to the type (twice, if two terms: 2^-16 of it is left)
    dH = dH + (U[dt] if not two_term else 2.0 ** -16) * (H.abs() + dH)
    dY = dH @ aD.t() + (2 * F * S) * (H.abs() @ aD.t())
    return dY + U[dt] * (Y.abs() + dY), dg + U[dt] * (G.abs() + dg), du + U[dt] * (U_.abs() + du)


def grads(name, X, Wg, Wu, Wd, G, U_, dY):
    """(dX, dWg, dWu, dWd) in 64 bits from what was kept, and their bounds."""
    dt = dY.dtype
    T, (F, D) = X.shape[0], Wg.shape
    X, Wg, Wu, Wd, G, U_, dY = (t.double() for t in (X, Wg, Wu, Wd, G, U_, dY))
    A, sl = act(name, G), slope(name, G)
    H, dH = A * U_, dY @ Wd
    dG, dU = dH * U_ * sl, dH * A
    out = (dG @ Wg + dU @ Wu, dG.t() @ X, dU.t() @ X, dY.t() @ H)
    off = ACT_OFF[dt]
    eA, eS = off * (G.abs() + 1), off * (G.abs() + 2)
    eH = eA * U_.abs() + U[dt] * H.abs() + 2 * S * H.abs()
    edH = (D * S) * (dY.abs() @ Wd.abs())
    edG = edH * U_.abs() * SLOPE + (dH.abs() + edH) * U_.abs() * eS + 4 * S * dG.abs()
    edU = edH * (A.abs() + eA) + dH.abs() * eA + 2 * S * dU.abs()
    edG = edG + U[dt] * (dG.abs() + edG)
    edU = edU + U[dt] * (dU.abs() + edU)
    aX, aY = X.abs(), dY.abs()
    bounds = [edG @ Wg.abs() + edU @ Wu.abs()
              + 4 * F * S * (dG.abs() @ Wg.abs() + dU.abs() @ Wu.abs()),
              edG.t() @ aX + 2 * T * S * (dG.abs().t() @ aX),
              edU.t() @ aX + 2 * T * S * (dU.abs().t() @ aX),
              aY.t() @ eH + 2 * T * S * (aY.t() @ H.abs())]
    return out, tuple(b + U[dt] * (o.abs() + b) for b, o in zip(bounds, out))


def pack(x):
    """(codes, scale bytes) of a checkpoint, from the definition in 64 bits."""
    x = x.double()
    R, C = x.shape
    n = (C + 31) // 32
    v = torch.zeros(R, n * 32, dtype=torch.float64, device=x.device)
    v[:, :C] = x
    v = v.view(R, n, 32)
    big = v.abs().amax(2)
    bad = ~torch.isfinite(v).all(2)
    safe = torch.where(bad | (big == 0), 1.0, big)
    mant, e = torch.frexp(safe)                # big = mant 2^e, mant in [1/2, 1)
    e = e - 1 + (mant >= 127.5 / 128).int()
    byte = torch.where(big == 0, 0, (127 + e - 6).clamp(min=0))
    byte = torch.where(bad, 255, byte)
    step = torch.where(bad, 1.0, torch.exp2((byte - 127).double()))
    q = torch.where(bad[:, :, None], 0.0, (v / step[:, :, None]).round())
    return q.to(torch.int8).view(R, -1)[:, :C], byte.to(torch.uint8)


def values(codes, scale):
    """What a checkpoint stands for, in 64 bits."""
    at = torch.arange(codes.shape[1], device=codes.device) // 32
    step = torch.where(scale == 255, math.nan, torch.exp2(scale.double() - 127))
    return codes.double() * step[:, at]


def row_codes(x):
    """(codes, fp32 scales) of rows, from the definition in 64 bits."""
    s = (x.float().abs().amax(1).double() / 127).float()
    bad = ~torch.isfinite(x).all(1)
    q = (x.double() / torch.where(s > 0, s, 1.0).double()[:, None]).round()
    q = torch.where(bad[:, None] | (s == 0)[:, None], 0.0, q)
    return q.to(torch.int8), torch.where(bad, math.nan, s)


def inputs(T, D, F, dt, seed=0, device="cuda"):
    """X, Wg, Wu, Wd, dY of a block."""
    g = torch.Generator(device).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=device)     # noqa: E731
    X = r(T, D) * torch.exp(0.5 * r(D))
    return tuple(t.to(dt) for t in (X, r(F, D) * D ** -0.5, r(F, D) * D ** -0.5,
                                    r(D, F) * F ** -0.5, r(T, D)))


def strided(t, gap=5, shift=3, fill=float("nan")):
    """A copy of t whose rows lie `gap` elements further apart, `shift` into
    their buffer, and that buffer (`fill` around the rows)."""
    rows, cols = t.shape
    if t.dtype in (torch.int8, torch.uint8):
        fill = 77
    buf = torch.full((rows * (cols + gap) + shift,), fill, dtype=t.dtype, device=t.device)
    view = buf[shift:].view(rows, cols + gap)[:, :cols]
    view.copy_(t)
    return view, buf


def close(got, want, bound, what):
    """got within `bound` of want, element by element."""
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d off, the worst %.3g times the bound at %s" % (
        what, int(bad.sum()), bad.numel(), float((off / bound.clamp(min=1e-300)).max()),
        bad.nonzero()[0].tolist())
