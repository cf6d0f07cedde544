"""What the gated block's results may be off by in the 2-norm, and the sizes at which its
calls run every kernel of theirs.

Element by element a bound has to count each rounding at its worst, K roundings of a sum in
one direction among them, and a rounding too many can hide behind it.  In the 2-norm the
roundings add up as they are: those of a type are taken from the 64-bit results, rounded
where the calls say that they round (`model`), and fp32 sums of K terms of any sign are off
by 2^-24 sqrt(K / 6) of themselves (K roundings of partial sums, whose squares grow from 0
to the whole one's, each of a third of 2^-48).
"""

import math

import torch

from tests import gated_util as G

S = G.S

# (rows, width, hidden) at which all six activations are run: tiles of 256, 128, 128 x 64
# and 128 x 32 of "up" and "dh" in both types and in codes, whole and cut ones, operands in
# place and copied, last columns of their own
ACT_SIZES = [(2500, 1000, 2500), (2000, 512, 512), (700, 512, 1365), (8192, 768, 2048),
             (4096, 1024, 2731), (900, 900, 1800), (45, 2100, 70)]
# and with one activation each: one row, few rows (16, 32, 64; 32 rows of long matrices a
# workgroup; Wd in tiles and in place), down and the gradients in tiles of 256, dh by
# partials in every tile, shares of K
SIZES = [(1, 1300, 1100), (1, 90, 70), (1, 70, 2600), (1, 2100, 2300), (9, 1030, 300), (9, 4097, 90),
         (24, 320, 640), (24, 321, 643), (48, 128, 640), (48, 321, 643), (20, 64, 8208),
         (20, 70, 8209), (40, 70, 8209), (64, 128, 8256), (520, 1024, 4096),
         (1100, 2048, 4096), (5536, 1575, 40), (600, 2048, 2048), (690, 8102, 70),
         (1032, 1053, 60), (896, 256, 7466), (7124, 3566, 565)]
# (rows, channels, columns) of products of codes
PRODUCTS = [(1, 300, 128), (1, 300, 2100), (9, 257, 1000), (24, 257, 1000), (48, 257, 1000),
            (48, 256, 1024), (100, 512, 4096), (700, 1000, 512), (2500, 2500, 1000),
            (2500, 10000, 1000)]
# (rows, columns) of checkpoints: in the caches and past them; of rows that become codes: a
# wave and a workgroup a row, held and read twice
PACKS = [(700, 1973), (8200, 8192)]
ROW_CODES = [(9, 1000), (9, 2056), (9, 9000), (9, 1001), (3, 20001)]


def sums(K):
    return S * (math.sqrt(K / 6) + 4)


def rounded(t, dt, terms=1):
    """t as `terms` numbers of the type, in 64 bits (fp32: as it is)."""
    if dt != torch.bfloat16:
        return t
    a = t.to(dt).double()
    return a if terms == 1 else a + (t - a).to(dt).double()


def forward(name, X, Wg, Wu, Wd):
    """(Y in 64 bits, Y with the roundings of the type's calls, what fp32 leaves)."""
    T, (F, D) = X.shape[0], Wg.shape
    dt = X.dtype
    Y, _, _, h = G.block(name, X, Wg, Wu, Wd)
    model = rounded(h, dt, 2 if T <= 128 else 1) @ Wd.double().t()
    # g and u, either of which h has once (of an activation's slope up to 1.13 where its
    # value is half of g); the activation; h's sum; twice of all
    return Y, rounded(model, dt), 2 * (4 * sums(D) + sums(F) + 16 * S)


def grads(name, X, Wg, Wu, Wd, g, u, dY, dt):
    """((dX, dWg, dWu, dWd) in 64 bits, the same with the roundings, what fp32 leaves)."""
    T, (F, D) = X.shape[0], Wg.shape
    X, Wg, Wu, Wd, g, u, dY = (t.double() for t in (X, Wg, Wu, Wd, g, u, dY))
    a, s, dh = G.act(name, g), G.slope(name, g), dY @ Wd
    h, dg, du = a * u, dh * u * s, dh * a
    terms = 2 if T <= 128 else 1
    h2, dg2, du2 = (rounded(t, dt, terms) for t in (h, dg, du))
    f = lambda h, dg, du: (dg @ Wg + du @ Wu, dg.t() @ X, du.t() @ X, dY.t() @ h)   # noqa: E731
    rest = [2 * (sums(D) + sums(K) + 16 * S) for K in (2 * F, T, T, T)]
    return f(h, dg, du), [rounded(t, dt) for t in f(h2, dg2, du2)], rest


def close(got, want, model, rest, what):
    """got is no further from want than its model, to a tenth, and what fp32 leaves.  (One
    rounding more is 22% or more: of two equal ones that are independent a third.)"""
    off, most = float((got.double() - want).norm()), float((model - want).norm())
    most = 1.1 * most + rest * float(want.norm())
    assert off <= most, "%s: off by %.3g, %.3g times what its roundings make" % (
        what, off, off / max(most, 1e-300))
