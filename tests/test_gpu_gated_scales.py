"""Products of codes whose scales' product leaves fp32's normal numbers where the result
does not, in every form of the products: one row, few rows, tiles, partials."""

import pytest
import torch

from paper_1606_00511_amd import hf as H
from tests import gated_util as G

pytestmark = pytest.mark.gpu

# one row by a wave a row and by few rows; few rows at odd and whole widths; tiles; tiles
# whose sums are partials (few channels of long rows)
SIZES = [(1, 50, 4096), (1, 70, 1000), (5, 33, 515), (40, 70, 300), (24, 128, 1024),
         (129, 257, 1000), (300, 640, 512), (96, 64, 8192)]
# powers of two of the rows' and of the channels' scales
SCALES = [(-100, -44), (-44, -100), (-126, -20), (-20, -126), (-140, -6), (-6, -140), (124, -140),
          (-140, 124), (126, -60), (-60, 126), (-149, 120), (110, -149)]


def operands(T, N, K, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    r = lambda *s: torch.randint(-127, 128, s, generator=g, device="cuda").to(torch.int8)   # noqa: E731
    one = lambda n: 1 + torch.rand(n, generator=g, device="cuda", dtype=torch.float64)      # noqa: E731
    return r(T, K), r(N, K), one(T), one(N)


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("T,N,K", SIZES)
def test_product_scales(type, T, N, K):
    """y = sa sb sum to three roundings and the type's, wherever y is in range; below
    fp32's normal numbers to half its step there, 2^-150, and bf16's, 2^-134."""
    A, B, one_a, one_b = operands(T, N, K)
    n = H.HFGated(K, 64, T, dtype=type)
    sums = A.double() @ B.double().t()
    for ea, eb in SCALES:
        sa, sb = (one_a * 2.0 ** ea).float(), (one_b * 2.0 ** eb).float()
        Y = n.hf_gated_product(A, sa, B, sb)
        want = sums * (sa.double()[:, None] * sb.double())
        ok = want.abs() < 2.0 ** 127.9
        low = 2.0 ** -150 + (2.0 ** -134 if type == "bf16" else 0)
        bound = (3.01 * G.S + G.U[Y.dtype] * (1 + 4 * G.S)) * want.abs() + low
        off = (Y.double() - want).abs()
        assert ((off <= bound) | ~ok).all(), (ea, eb, float((off / bound)[ok].max()))
        assert torch.equal(Y.signbit()[ok & (want != 0)], want.signbit()[ok & (want != 0)])


@pytest.mark.parametrize("T,N,K", SIZES)
def test_sums_of_zero(T, N, K):
    """A sum of 0 is 0 whatever the scales, of either sign."""
    A, B, one_a, one_b = operands(T, N, K, 1)
    A[T // 2] = 0
    B[N // 3] = 0
    n = H.HFGated(K, 64, T, dtype="fp32")
    for ea, eb in ((100, 60), (60, 100), (127, 127), (-149, -149)):
        for sign in (1, -1):
            Y = n.hf_gated_product(A, sign * (one_a * 2.0 ** ea).clamp(max=3e38).float(), B,
                                   (one_b * 2.0 ** eb).clamp(max=3e38).float())
            assert (Y[T // 2] == 0).all() and (Y[:, N // 3] == 0).all(), (ea, eb)
    # scales without a number stay so
    sa, sb = one_a.float(), one_b.float()
    sa[T - 1], sb[N - 1] = float("nan"), float("nan")
    Y = n.hf_gated_product(A, sa, B, sb)
    assert torch.isnan(Y[T - 1]).all() and torch.isnan(Y[:, N - 1]).all()
    assert torch.isfinite(Y[:T - 1, :N - 1]).all()


@pytest.mark.parametrize("T,D,F", [(1, 4096, 70), (1, 1024, 200), (20, 4096, 128), (40, 2000, 99),
                                   (100, 4096, 256)])
def test_block_scales(T, D, F):
    """The block on codes with small rows and gates: the products of their scales are next
    to 2^-147, g next to 2^-123, and u large.  g's digits show in h's codes: with g, u and h
    off by 5 roundings of 2^-24 a code changes only next to a border, 2^-13 of all places at
    127 steps; a step is at most 1 / 127 of a row's largest, which is at most 30 times its
    mean of F >= 70 numbers."""
    g = torch.Generator("cuda").manual_seed(T)
    r = lambda *s: torch.rand(*s, generator=g, device="cuda") + 0.1      # noqa: E731
    X, Wg = r(T, D) * 2.0 ** -90, r(F, D) * 2.0 ** -43
    Wu, Wd = r(F, D) * 2.0 ** 100, torch.randn(D, F, generator=g, device="cuda")
    n = H.HFGated(D, F, T, act="relu", dtype="fp32")
    q = [n.hf_gated_codes(w) for w in (Wg, Wu, Wd)]
    Y = n.hf_gated_forward_codes(X, *q)
    qx, sx = G.row_codes(X)
    times = lambda a, sa, m: (a.double() @ m[0].double().t()) * (   # noqa: E731
        sa.double()[:, None] * m[1].double())
    h = times(qx, sx, q[0]).clamp(min=0) * times(qx, sx, q[1])
    sh = (h.abs().amax(1) / 127).float().double()
    want = times((h / sh[:, None]).round(), sh, q[2])
    assert float((Y.double() - want).norm()) <= 0.01 * float(want.norm())


@pytest.mark.parametrize("cols", [100, 1024])
def test_codes_of_the_smallest_numbers(cols):
    """Rows whose scale is below fp32's normal numbers, rounded to few digits: codes of the
    quotient by it, within 127."""
    g = torch.Generator("cuda").manual_seed(cols)
    X = torch.randn(40, cols, generator=g, device="cuda", dtype=torch.float64)
    X = (X * torch.exp2(-115.0 - torch.arange(40, device="cuda").double())[:, None]).float()
    codes, s = H.HFGated(64, 64, 1, dtype="fp32").hf_gated_codes(X)
    want = (X.abs().amax(1).double() / 127).float()
    assert torch.equal(s, want)
    q = (X.double() / torch.where(want > 0, want, 1.0).double()[:, None]).round()
    q = torch.where(want[:, None] > 0, q, 0.0).clamp(-127, 127)
    assert torch.equal(codes.double(), q) and (s == 0).any() and (q.abs().amax(1) == 127).any()
