"""That the 2-norms of tests/gated_norms.py tell a rounding too many, with the mistakes
planted in results in 64 bits.  No GPU."""

import pytest
import torch

from tests import gated_norms as N
from tests import gated_util as G

BF16, F32 = torch.bfloat16, torch.float32


def inputs(T, dt):
    X, Wg, Wu, Wd, dY = G.inputs(T, 96, 160, dt, device="cpu")
    g, u = X.double() @ Wg.double().t(), X.double() @ Wu.double().t()
    return X, Wg, Wu, Wd, g.to(dt), u.to(dt), dY


def results(X, Wg, Wu, Wd, g, u, dY, dt, round_h, round_d, round_dh=lambda t: t):
    """(Y, dX, dWg, dWu, dWd), with h, dg and du, and dh rounded by these."""
    x, wg, wu, wd, g, u, dy = (t.double() for t in (X, Wg, Wu, Wd, g, u, dY))
    hY = round_h(G.act("silu", x @ wg.t()) * (x @ wu.t()))
    a, s, dh = G.act("silu", g), G.slope("silu", g), round_dh(dy @ wd)
    h, dg, du = round_h(a * u), round_d(dh * u * s), round_d(dh * a)
    out = (hY @ wd.t(), dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ h)
    return [N.rounded(t, dt) for t in out]


def fails(got, args, dt):
    X, Wg, Wu, Wd, g, u, dY = args
    checks = [N.forward("silu", X, Wg, Wu, Wd)]
    checks += list(zip(*N.grads("silu", X, Wg, Wu, Wd, g, u, dY, dt)))
    bad = []
    for t, (want, model, rest), what in zip(got, checks, ("Y", "dX", "dWg", "dWu", "dWd")):
        try:
            N.close(t, want, model, rest, what)
        except AssertionError:
            bad.append(what)
    return bad


def terms(n):
    return lambda t: N.rounded(t, BF16, n)


def exact(t):
    return t


ALL = ["Y", "dX", "dWg", "dWu", "dWd"]


@pytest.mark.parametrize("T,dt,n", [(100, F32, 0), (400, F32, 0), (100, BF16, 2), (400, BF16, 1)])
def test_the_calls_roundings_pass(T, dt, n):
    args = inputs(T, dt)
    r = terms(n) if n else exact
    assert fails(results(*args, dt, r, r), args, dt) == []


@pytest.mark.parametrize("T", [100, 400])
def test_bf16_in_fp32_calls(T):
    args = inputs(T, F32)
    assert fails(results(*args, F32, terms(1), terms(1)), args, F32) == ALL
    assert fails(results(*args, F32, terms(1), exact), args, F32) == ["Y", "dWd"]
    assert fails(results(*args, F32, exact, terms(1)), args, F32) == ["dX", "dWg", "dWu"]


def test_one_term_where_two_are_due():
    args = inputs(100, BF16)
    assert fails(results(*args, BF16, terms(1), terms(1)), args, BF16) == ALL


def test_a_rounding_too_many():
    """dh rounded as well."""
    args = inputs(400, BF16)
    got = results(*args, BF16, terms(1), terms(1), terms(1))
    assert fails(got, args, BF16) == ["dX", "dWg", "dWu"]
