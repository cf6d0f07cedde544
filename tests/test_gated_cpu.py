"""Host-side checks of the gated block's calls that need no GPU: limits, the
workspace's size, and the refusals, all made before any device call."""

import ctypes
import os

import pytest

from paper_1606_00511_amd import hf as H

OK, EINVAL, EWS = H.HF_OK, H.HF_EINVAL, H.HF_EWORKSPACE
FAKE = ctypes.c_void_p(1 << 20)          # never dereferenced
FAKE2, FAKE3, FAKE4, FAKE5 = (ctypes.c_void_p((1 << 30) + (i << 24)) for i in range(4))
ODD = ctypes.c_void_p((1 << 20) + 1)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(H.LIB_PATH):
        from paper_1606_00511_amd.build import build_library
        build_library()
    return H.lib()


def create(L, width=64, hidden=96, act=H.HF_SILU, type=H.HF_TYPE_BF16, rows=256):
    h = ctypes.c_void_p()
    return L.hf_gated_create(width, hidden, act, type, rows, None, ctypes.byref(h)), h


def test_create_validates(L):
    most = H.HF_GATED_MAX_WIDTH
    for bad in (dict(width=0), dict(width=-1), dict(width=most + 1), dict(hidden=0),
                dict(hidden=most + 1), dict(act=-1), dict(act=6), dict(type=2), dict(type=-1),
                dict(rows=0), dict(rows=H.HF_GATED_MAX_ROWS + 1)):
        rc, h = create(L, **bad)
        assert rc == EINVAL and not h.value, bad
    assert L.hf_gated_create(4, 4, 0, 0, 4, None, None) == EINVAL
    for good in [dict(act=a) for a in H.GATED_ACTS.values()] + [
            dict(width=1, hidden=1, rows=1), dict(width=most, hidden=most),
            dict(rows=H.HF_GATED_MAX_ROWS)]:
        rc, h = create(L, **good)
        assert rc == OK and L.hf_gated_destroy(h) == OK, good


def test_the_nets_keep_their_activations(L):
    """The block's activations are not the nets'."""
    dims = (ctypes.c_int32 * 2)(4, 3)
    for act in (H.HF_SILU, H.HF_GELU, H.HF_GELU_TANH):
        h = ctypes.c_void_p()
        assert L.hf_create(dims, 2, act, H.HF_FP32, 16, None, ctypes.byref(h)) == EINVAL


def test_constants_are_the_headers():
    txt = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                            "include", "hf.h")).read()
    for name in ("HF_GATED_MAX_WIDTH", "HF_GATED_MAX_ROWS", "HF_GATED_MAX_OUT", "HF_CODE_BLOCK"):
        line = next(l for l in txt.splitlines() if l.startswith("#define " + name + " "))
        assert eval(line.split(None, 2)[2]) == getattr(H, name), name
    for name in ("HF_SILU", "HF_GELU", "HF_GELU_TANH", "HF_KEEP_NONE", "HF_KEEP_FULL",
                 "HF_KEEP_CODES"):
        assert "%s = %d" % (name, getattr(H, name)) in txt


@pytest.mark.parametrize("type", [H.HF_TYPE_FP32, H.HF_TYPE_BF16])
@pytest.mark.parametrize("width,hidden", [(1, 1), (768, 2050), (4096, 16384), (1021, 2731),
                                          (65536, 64), (64, 65536)])
def test_workspace_grows_with_rows(L, type, width, hidden):
    rc, h = create(L, width, hidden, type=type, rows=262144)
    assert rc == OK
    rows = [1, 2, 16, 17, 63, 64, 65, 127, 128, 129, 256, 257, 1000, 4096, 4097, 65536, 262143,
            262144]
    got = [L.hf_gated_workspace_bytes(h, r) for r in rows]
    assert all(0 < a <= b for a, b in zip(got, got[1:])), got
    assert L.hf_gated_workspace_bytes(h, 0) == got[-1]
    assert L.hf_gated_workspace_bytes(h, 262145) == 0
    assert L.hf_gated_destroy(h) == OK


def test_null_context(L):
    assert L.hf_gated_destroy(None) == OK
    assert L.hf_gated_set_stream(None, None) == EINVAL
    assert L.hf_gated_workspace_bytes(None, 1) == 0
    assert L.hf_gated_set_workspace(None, FAKE, 1 << 30) == EINVAL
    assert L.hf_gated_last_error(None) == b"null context"
    for fn, good, _ in CALLS:
        assert getattr(L, fn)(None, *good.values()) == EINVAL, fn


def test_workspace_refusals(L):
    rc, h = create(L)
    assert rc == OK
    assert L.hf_gated_set_workspace(h, None, 1 << 30) == EINVAL
    assert L.hf_gated_set_workspace(h, ctypes.c_void_p(4096 + 16), 1 << 30) == EINVAL
    assert b"256-byte" in L.hf_gated_last_error(h)
    need = L.hf_gated_workspace_bytes(h, 1)
    assert L.hf_gated_set_workspace(h, ctypes.c_void_p(4096), need - 1) == EWS
    assert L.hf_gated_destroy(h) == OK


W = dict(Wg=FAKE, ldg=64, Wu=FAKE, ldu=64, Wd=FAKE, ldd=96)
FWD = dict(X=FAKE, ldx=64, **W, rows=4, Y=FAKE2, ldy=64, keep=0, kept=None, ldk=0, scale=None,
           lds=0)
FULL = dict(FWD, keep=H.HF_KEEP_FULL, kept=FAKE3, ldk=192)
CODES = dict(FWD, keep=H.HF_KEEP_CODES, kept=FAKE3, ldk=192, scale=FAKE4, lds=6)
GRAD = dict(X=FAKE, ldx=64, xscale=None, ldxs=0, **W, keep=H.HF_KEEP_CODES, kept=FAKE3, ldk=192,
            scale=FAKE4, lds=6, dY=FAKE, lddy=64, rows=4, dX=FAKE2, lddx=64, dWg=FAKE2, lddg=64,
            dWu=FAKE5, lddu=64, dWd=FAKE2, lddd=96, accumulate=0)
PACK = dict(X=FAKE, ldx=40, rows=4, cols=40, codes=FAKE2, ldc=40, scale=FAKE3, lds=2)
UNPACK = dict(codes=FAKE, ldc=40, scale=FAKE3, lds=2, rows=4, cols=40, X=FAKE2, ldx=40)
ROWS = dict(X=FAKE, ldx=40, rows=4, cols=40, codes=FAKE2, ldc=40, scale=FAKE3)
PROD = dict(A=FAKE, lda=40, sa=FAKE, B=FAKE, ldb=40, sb=FAKE, rows=4, n=10, k=40, Y=FAKE2, ldy=10)
FWDC = dict(X=FAKE, ldx=64, Wg=FAKE, ldg=64, sg=FAKE, Wu=FAKE, ldu=64, su=FAKE, Wd=FAKE, ldd=96,
            sd=FAKE, rows=4, Y=FAKE2, ldy=64)
MATS = [dict(X=None), dict(X=ODD), dict(ldx=63), dict(ldx=(1 << 31) + 1), dict(Wg=None),
        dict(Wg=ODD), dict(ldg=63), dict(Wu=None), dict(Wu=ODD), dict(ldu=1), dict(Wd=None),
        dict(Wd=ODD), dict(ldd=95), dict(rows=-1), dict(rows=257)]
FWD_BAD = MATS + [dict(Y=None), dict(Y=ODD), dict(ldy=63), dict(Y=FAKE), dict(keep=3),
                  dict(keep=-1)]
CALLS = [
    ("hf_gated_forward", FWD, FWD_BAD),
    ("hf_gated_forward", FULL, FWD_BAD + [dict(kept=None), dict(kept=ODD), dict(ldk=191),
                                          dict(kept=FAKE), dict(kept=FAKE2)]),
    ("hf_gated_forward", CODES, FWD_BAD + [dict(kept=None), dict(ldk=191), dict(scale=None),
                                           dict(lds=5)]),
    ("hf_gated_grad", GRAD, MATS + [
        dict(ldxs=1, xscale=FAKE, ldx=64), dict(keep=0), dict(keep=3), dict(kept=None),
        dict(ldk=191), dict(scale=None), dict(lds=5), dict(keep=1, kept=ODD), dict(dY=None),
        dict(dY=ODD), dict(lddy=63), dict(dX=None, dWg=None, dWu=None, dWd=None), dict(dX=ODD),
        dict(lddx=63), dict(dWg=ODD), dict(lddg=63), dict(dWu=ODD), dict(lddu=63), dict(dWd=ODD),
        dict(lddd=95), dict(accumulate=2), dict(accumulate=-1),
        # outputs over inputs, and over each other
        dict(dX=FAKE), dict(dX=FAKE3), dict(dWg=FAKE), dict(dWu=FAKE), dict(dWd=FAKE),
        dict(dWu=FAKE2)]),
    ("hf_gated_pack", PACK, [dict(X=None), dict(X=ODD), dict(ldx=39), dict(rows=-1),
                             dict(rows=H.HF_GATED_MAX_ROWS + 1), dict(cols=0), dict(cols=65537),
                             dict(codes=None), dict(ldc=39), dict(scale=None), dict(lds=1),
                             dict(codes=FAKE)]),
    ("hf_gated_unpack", UNPACK, [dict(X=None), dict(X=ODD), dict(ldx=39), dict(rows=-1),
                                 dict(rows=H.HF_GATED_MAX_ROWS + 1), dict(cols=0),
                                 dict(codes=None), dict(ldc=39), dict(scale=None), dict(lds=1),
                                 dict(X=FAKE)]),
    ("hf_gated_codes", ROWS, [dict(X=None), dict(X=ODD), dict(ldx=39), dict(rows=-1),
                              dict(rows=H.HF_GATED_MAX_OUT + 1), dict(cols=0), dict(cols=65537),
                              dict(codes=None), dict(ldc=39), dict(scale=None),
                              dict(scale=ctypes.c_void_p(4098)), dict(codes=FAKE)]),
    ("hf_gated_product", PROD, [dict(A=None), dict(lda=39), dict(sa=None), dict(sa=ODD),
                                dict(B=None), dict(ldb=39), dict(sb=None), dict(rows=-1),
                                dict(rows=257), dict(n=0), dict(n=H.HF_GATED_MAX_OUT + 1),
                                dict(k=0), dict(k=97, lda=97, ldb=97), dict(Y=None), dict(Y=ODD),
                                dict(ldy=9), dict(Y=FAKE)]),
    ("hf_gated_forward_codes", FWDC, [b for b in MATS if ODD not in b.values()] + [
        dict(X=ODD), dict(sg=None), dict(su=None), dict(sd=None), dict(sg=ODD), dict(Y=None),
        dict(Y=ODD), dict(ldy=63), dict(Y=FAKE)]),
]


@pytest.mark.parametrize("fn,good,bads", CALLS, ids=["%s-%d" % (c[0], i)
                                                     for i, c in enumerate(CALLS)])
def test_refusals(L, fn, good, bads):
    """Each bad argument is refused with a message; the good ones get as far as
    the missing workspace, or for calls without one are not made here."""
    rc, h = create(L)
    assert rc == OK
    f = getattr(L, fn)
    for bad in bads:
        assert set(bad) <= set(good), bad
        assert f(h, *dict(good, **bad).values()) == EINVAL, bad
        assert L.hf_gated_last_error(h), bad
    if fn not in ("hf_gated_pack", "hf_gated_unpack", "hf_gated_codes"):
        assert f(h, *good.values()) == EWS
        assert b"workspace" in L.hf_gated_last_error(h)
    assert L.hf_gated_destroy(h) == OK
