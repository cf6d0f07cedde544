"""Every kernel of the gated block against the definitions in 64 bits, element by element
(tests/gated_util.py) and by the 2-norm (tests/gated_norms.py): at the sizes there, which
tests/test_gated_kernels_cpu.py finds to run all of them."""

import pytest
import torch

from paper_1606_00511_amd import hf as H
from tests import gated_norms as N
from tests import gated_util as G

pytestmark = pytest.mark.gpu

ACTS = ["silu", "gelu", "gelu_tanh", "sigmoid", "tanh", "relu"]
BLOCKS = [(s, a) for s in N.ACT_SIZES for a in ACTS] + [
    (s, ACTS[sum(s) % 6]) for s in N.SIZES]


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("size,act", BLOCKS, ids=["%dx%dx%d-%s" % (*s, a) for s, a in BLOCKS])
def test_block(type, size, act):
    T, D, F = size
    dt = G.TYPES[type]
    X, Wg, Wu, Wd, dY = G.inputs(T, D, F, dt, seed=T + F)
    n = H.HFGated(D, F, T, act=act, dtype=type)
    Y, _ = n.hf_gated_forward(X, Wg, Wu, Wd)
    Yf, full = n.hf_gated_forward(X, Wg, Wu, Wd, keep="full")
    Y8, (codes, scale) = n.hf_gated_forward(X, Wg, Wu, Wd, keep="int8")
    assert torch.equal(Y, Yf) and torch.equal(Y, Y8)
    N.close(Y, *N.forward(act, X, Wg, Wu, Wd), "Y")
    _, g, u, _ = G.block(act, X, Wg, Wu, Wd)
    by, bg, bu = G.block_bound(act, X, Wg, Wu, Wd, two_term=type == "bf16" and T <= 128)
    G.close(Y, G.block(act, X, Wg, Wu, Wd)[0], by, "Y")
    nb = (F + 31) // 32
    at = torch.arange(F, device="cuda") // 32
    for i, (t, b, what) in enumerate(((g, bg, "g"), (u, bu, "u"))):
        kept = full[:, i * F:(i + 1) * F]
        N.close(kept, t, N.rounded(t, dt), 2 * N.sums(D), what)
        G.close(kept, t, b, what)
        c, s = codes[:, i * F:(i + 1) * F], scale[:, i * nb:(i + 1) * nb]
        # half a step, and what the sum was off by
        step = torch.exp2(s.double() - 127)[:, at]
        G.close(G.values(c, s), t, step / 2 + b, what + "'s codes")

    # from what was kept in full, and from checkpoints of it and of X
    x8 = n.hf_gated_pack(X)
    g8, u8 = (G.values(codes[:, i * F:(i + 1) * F], scale[:, i * nb:(i + 1) * nb])
              for i in (0, 1))
    for x, kept, xv, g, u in ((X, full, X, full[:, :F], full[:, F:]),
                              (x8, (codes, scale), G.values(*x8), g8, u8)):
        got = n.hf_gated_grad(x, Wg, Wu, Wd, kept, dY)
        elements = G.grads(act, xv, Wg, Wu, Wd, g, u, dY)
        norms = N.grads(act, xv, Wg, Wu, Wd, g, u, dY, dt)
        for a, w, b, m, r, what in zip(got, *elements, *norms[1:], ("dX", "dWg", "dWu", "dWd")):
            G.close(a, w, b, what)
            N.close(a, w, m, r, what)


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("size,act", BLOCKS, ids=["%dx%dx%d-%s" % (*s, a) for s, a in BLOCKS])
def test_block_on_codes(type, size, act):
    """Element by element: as far as h's codes next to a border between two may be on its
    other side."""
    T, D, F = size
    dt = G.TYPES[type]
    X, Wg, Wu, Wd, _ = G.inputs(T, D, F, dt, seed=T)
    n = H.HFGated(D, F, T, act=act, dtype=type)
    q = [n.hf_gated_codes(w) for w in (Wg, Wu, Wd)]
    Y = n.hf_gated_forward_codes(X, *q)
    qx, sx = G.row_codes(X)
    times = lambda a, sa, m: (a.double() @ m[0].double().t()) * (   # noqa: E731
        sa.double()[:, None] * m[1].double())
    g, u = times(qx, sx, q[0]), times(qx, sx, q[1])
    h = G.act(act, g) * u
    sh = (h.abs().amax(1).float().double() / 127).float().double()
    safe = torch.where(sh > 0, sh, 1.0)[:, None]
    steps = h / safe
    want = times(steps.round(), sh, q[2])
    # h in fp32: g and u are off by 4 roundings each, the activation and the product by 8; a
    # code changes by one step where that crosses a border.  A scale off by a rounding:
    # 2^-23 of the row.
    off = G.SLOPE * 4 * G.S * g.abs() * u.abs() + 8 * G.S * (g.abs() + 1) * u.abs() \
        + 8 * G.S * h.abs()
    off = off / safe + 4 * G.S * steps.abs()
    near = ((steps - steps.floor() - 0.5).abs() <= off).double()
    w = (q[2][0].double() * q[2][1].double()[:, None]).abs()
    bound = (near * safe) @ w.t() + 8 * G.S * (steps.abs() * safe) @ w.t()
    G.close(Y, want, bound + G.U[dt] * (want.abs() + bound), "Y")


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("T,C,K", N.PRODUCTS)
def test_product(type, T, C, K):
    """Three roundings of the exact sum and its two scales, and that to the type."""
    g = torch.Generator("cuda").manual_seed(T + C + K)
    r = lambda *s: torch.randint(-127, 128, s, generator=g, device="cuda").to(torch.int8)   # noqa: E731
    A, B = r(T, K), r(C, K)
    sa, sb = (torch.rand(n, generator=g, device="cuda") + 0.1 for n in (T, C))
    Y = H.HFGated(K, 64, T, dtype=type).hf_gated_product(A, sa, B, sb)
    want = (A.double() @ B.double().t()) * (sa.double()[:, None] * sb.double())
    G.close(Y, want, (3.01 * G.S + G.U[Y.dtype] * (1 + 4 * G.S)) * want.abs(), "Y")


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("R,C", N.PACKS)
def test_pack(type, R, C):
    """Bit by bit, also of what is past the caches."""
    g = torch.Generator("cuda").manual_seed(R)
    X = torch.randn(R, C, generator=g, device="cuda")
    X = (X * torch.exp(3 * torch.randn(R, C, generator=g, device="cuda"))).to(G.TYPES[type])
    n = H.HFGated(64, 64, 1, dtype=type)
    codes, scale = n.hf_gated_pack(X)
    back = n.hf_gated_unpack(codes, scale)
    for i in range(0, R, 1000):             # (64 bits of all at once take much)
        part = slice(i, i + 1000)
        wc, ws = G.pack(X[part])
        assert torch.equal(codes[part], wc) and torch.equal(scale[part], ws)
        assert torch.equal(back[part].double(), G.values(wc, ws))


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("R,C", N.ROW_CODES)
def test_row_codes(type, R, C):
    g = torch.Generator("cuda").manual_seed(R + C)
    X = torch.randn(R, C, generator=g, device="cuda").to(G.TYPES[type])
    codes, s = H.HFGated(64, 64, 1, dtype=type).hf_gated_codes(X)
    wc, ws = G.row_codes(X)
    assert torch.equal(s, ws) and torch.equal(codes, wc)
