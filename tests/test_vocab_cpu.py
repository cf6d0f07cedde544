"""Host-side checks of the vocabulary calls that need no GPU: limits, the
workspace's size, and the refusals, all made before any device call."""

import ctypes
import os

import pytest

from paper_1606_00511_amd import hf as H

OK, EINVAL, EWS = H.HF_OK, H.HF_EINVAL, H.HF_EWORKSPACE
FAKE = ctypes.c_void_p(1 << 20)          # never dereferenced
FAKE2 = ctypes.c_void_p(1 << 30)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(H.LIB_PATH):
        from paper_1606_00511_amd.build import build_library
        build_library()
    return H.lib()


def create(L, vocab=1000, width=64, type=H.HF_TYPE_BF16, rows=256):
    h = ctypes.c_void_p()
    return L.hf_vocab_create(vocab, width, type, rows, None, ctypes.byref(h)), h


def test_create_validates(L):
    for bad in (dict(vocab=0), dict(vocab=-5), dict(vocab=H.HF_VOCAB_MAX + 1),
                dict(width=0), dict(width=H.HF_VOCAB_MAX_WIDTH + 1), dict(type=2),
                dict(type=-1), dict(rows=0), dict(rows=H.HF_VOCAB_MAX_ROWS + 1)):
        rc, h = create(L, **bad)
        assert rc == EINVAL and not h.value, bad
    assert L.hf_vocab_create(10, 10, 0, 10, None, None) == EINVAL
    for good in (dict(vocab=1, width=1, rows=1), dict(vocab=H.HF_VOCAB_MAX),
                 dict(rows=H.HF_VOCAB_MAX_ROWS), dict(width=H.HF_VOCAB_MAX_WIDTH)):
        rc, h = create(L, **good)
        assert rc == OK and L.hf_vocab_destroy(h) == OK, good


def test_limits_are_the_headers():
    txt = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                            "include", "hf.h")).read()
    for name in ("HF_IGNORE", "HF_VOCAB_MAX", "HF_VOCAB_MAX_WIDTH", "HF_VOCAB_MAX_ROWS",
                 "HF_VOCAB_MAX_TOP"):
        line = next(l for l in txt.splitlines() if l.startswith("#define " + name + " "))
        assert eval(line.split(None, 2)[2]) == getattr(H, name), name


@pytest.mark.parametrize("type", [H.HF_TYPE_FP32, H.HF_TYPE_BF16])
@pytest.mark.parametrize("vocab,width", [(1, 1), (1973, 2048), (50257, 1021), (131072, 4096),
                                         (H.HF_VOCAB_MAX, 64)])
def test_workspace_grows_with_rows(L, type, vocab, width):
    rc, h = create(L, vocab, width, type, 262144)
    assert rc == OK
    rows = [1, 2, 64, 127, 128, 129, 256, 257, 1000, 4096, 4097, 8192, 8193, 16384, 65536,
            262143, 262144]
    got = [L.hf_vocab_workspace_bytes(h, r) for r in rows]
    assert all(0 < a <= b for a, b in zip(got, got[1:])), got
    assert L.hf_vocab_workspace_bytes(h, 0) == got[-1]
    assert L.hf_vocab_workspace_bytes(h, 262145) == 0
    assert L.hf_vocab_destroy(h) == OK


def test_workspace_does_not_hold_the_logits(L):
    """A full minibatch on a large vocabulary: 4.3 GB of fp32 logits, and of
    the workspace less than that (1.5 GiB of it for smaller calls, whose
    logits are kept)."""
    rc, h = create(L, 131072, 4096, H.HF_TYPE_BF16, 8192)
    assert rc == OK
    assert L.hf_vocab_workspace_bytes(h, 0) < 2.6e9
    assert L.hf_vocab_destroy(h) == OK


def test_null_context(L):
    assert L.hf_vocab_destroy(None) == OK
    assert L.hf_vocab_set_stream(None, None) == EINVAL
    assert L.hf_vocab_workspace_bytes(None, 1) == 0
    assert L.hf_vocab_set_workspace(None, FAKE, 1 << 30) == EINVAL
    assert L.hf_vocab_check(None) == EINVAL
    assert L.hf_vocab_last_error(None) == b"null context"
    assert L.hf_vocab_loss(None, FAKE, 64, FAKE, 64, FAKE, 4, 0.0, FAKE, FAKE) == EINVAL
    assert L.hf_vocab_distill(None, FAKE, 64, FAKE, 64, FAKE, 4, FAKE, 4, 4, 1.0, 4, 0.0, FAKE,
                              FAKE) == EINVAL
    assert L.hf_vocab_embed(None, FAKE, 64, FAKE, 4, 1.0, FAKE, 64) == EINVAL
    assert L.hf_vocab_embed_grad(None, FAKE, 4, 1.0, FAKE, 64, FAKE, 64, 0) == EINVAL


def test_workspace_refusals(L):
    rc, h = create(L)
    assert rc == OK
    assert L.hf_vocab_set_workspace(h, None, 1 << 30) == EINVAL
    assert L.hf_vocab_set_workspace(h, ctypes.c_void_p(4096 + 16), 1 << 30) == EINVAL
    assert b"256-byte" in L.hf_vocab_last_error(h)
    need = L.hf_vocab_workspace_bytes(h, 1)
    assert L.hf_vocab_set_workspace(h, ctypes.c_void_p(4096), need - 1) == EWS
    assert L.hf_vocab_check(h) == OK          # nothing has run
    assert L.hf_vocab_destroy(h) == OK


NAN, INF = float("nan"), float("inf")
LOSS = dict(X=FAKE, ldx=64, W=FAKE, ldw=64, y=FAKE, rows=4, denom=0.0, loss=FAKE,
            row_loss=FAKE)
GRAD = dict(LOSS, dX=FAKE2, lddx=64, dW=FAKE2, lddw=64, accumulate=0)
LIST = dict(X=FAKE, ldx=64, W=FAKE, ldw=64, ids=FAKE, ldi=8, t=FAKE, ldt=8, top=8, tau=1.0,
            rows=4, denom=0.0, loss=FAKE, row_loss=FAKE)
LGRAD = dict(LIST, dX=FAKE2, lddx=64, dW=FAKE2, lddw=64, accumulate=0)
EMBED = dict(E=FAKE, lde=64, tok=FAKE, rows=4, scale=1.0, out=FAKE2, ldo=64)
EGRAD = dict(tok=FAKE, rows=4, scale=1.0, dout=FAKE, ldd=64, dE=FAKE2, lde=64, accumulate=0)
ODD, ODD4 = ctypes.c_void_p((1 << 20) + 1), ctypes.c_void_p((1 << 20) + 2)
HEAD_BAD = [dict(X=None), dict(X=ODD), dict(ldx=63), dict(ldx=(1 << 31) + 1), dict(W=None),
            dict(W=ODD), dict(ldw=10), dict(rows=-1), dict(rows=257), dict(denom=-1.0),
            dict(denom=NAN), dict(denom=INF), dict(loss=None), dict(loss=ODD4),
            dict(row_loss=ODD4)]
GRAD_BAD = HEAD_BAD + [dict(dX=None, dW=None), dict(dX=ODD), dict(lddx=63), dict(dW=ODD),
                       dict(lddw=63), dict(accumulate=2), dict(accumulate=-1),
                       dict(dX=FAKE), dict(dW=FAKE)]          # over X, over W
LIST_BAD = [dict(ids=None), dict(ids=ODD4), dict(ldi=7), dict(t=None), dict(t=ODD4),
            dict(ldt=7), dict(top=0), dict(top=-1), dict(top=129, ldi=200, ldt=200),
            dict(tau=0.0), dict(tau=-1.0), dict(tau=NAN), dict(tau=INF), dict(tau=1e-5),
            dict(tau=1e5)]
CALLS = [
    ("hf_vocab_loss", LOSS, HEAD_BAD + [dict(y=None), dict(y=ODD4)]),
    ("hf_vocab_loss_grad", GRAD, GRAD_BAD + [dict(y=None), dict(y=ODD4)]),
    ("hf_vocab_distill", LIST, HEAD_BAD + LIST_BAD),
    ("hf_vocab_distill_grad", LGRAD, GRAD_BAD + LIST_BAD),
    ("hf_vocab_embed", EMBED, [dict(E=None), dict(E=ODD), dict(lde=63), dict(tok=None),
                               dict(tok=ODD4), dict(rows=-1), dict(rows=257), dict(scale=NAN),
                               dict(scale=INF), dict(out=None), dict(out=ODD), dict(ldo=63),
                               dict(out=FAKE)]),
    ("hf_vocab_embed_grad", EGRAD, [dict(tok=None), dict(rows=-1), dict(rows=257),
                                    dict(scale=NAN), dict(dout=None), dict(dout=ODD),
                                    dict(ldd=63), dict(dE=None), dict(dE=ODD), dict(lde=63),
                                    dict(accumulate=3), dict(dE=FAKE)]),
]


@pytest.mark.parametrize("fn,good,bads", CALLS, ids=[c[0] for c in CALLS])
def test_refusals(L, fn, good, bads):
    """Each bad argument is refused with a message; the good ones get as far
    as the missing workspace."""
    rc, h = create(L)
    assert rc == OK
    f = getattr(L, fn)
    for bad in bads:
        assert f(h, *dict(good, **bad).values()) == EINVAL, bad
        assert L.hf_vocab_last_error(h), bad
    assert f(h, *good.values()) == EWS
    assert b"workspace" in L.hf_vocab_last_error(h)
    assert L.hf_vocab_destroy(h) == OK


@pytest.mark.parametrize("type,rows,a_word", [
    (H.HF_TYPE_FP32, 1, 64 * 4), (H.HF_TYPE_FP32, 128, 128 * 4),
    (H.HF_TYPE_BF16, 1, 1 * 4 + 2 * 32 * 2), (H.HF_TYPE_BF16, 128, 128 * 4 + 2 * 128 * 2)])
def test_workspace_of_few_rows(L, type, rows, a_word):
    """Few rows of the largest vocabulary: their logits and delta take what the
    rows need (delta of whole blocks of 64 or 32 rows), beside a statistics
    entry of 8 bytes a row and 32 words, 256 MiB each of packed W and of
    partials, and little else."""
    rc, h = create(L, H.HF_VOCAB_MAX, 64, type, rows)
    assert rc == OK
    most = H.HF_VOCAB_MAX * (a_word + rows / 4) + (520 << 20)
    assert L.hf_vocab_workspace_bytes(h, 0) < most
    assert L.hf_vocab_destroy(h) == OK
