"""That the sizes of tests/gated_norms.py, at which results are compared with 64 bits, run
every kernel of the gated block that the library has: read from a log of a stub in the HIP
runtime's place.  No GPU."""

from tests import gated_norms as N
from tests import hip_stub
from tests.test_gated_host import GATED, stub  # noqa: F401  (a fixture)


def test_every_kernel_is_compared(stub):  # noqa: F811
    names, seen = hip_stub.run(stub, GATED.replace(
        "stream=None)", "stream=None, act=H.HF_SILU)").replace("F, H.HF_SILU,", "F, act,") + """
S.stub_names.restype = ctypes.c_char_p
seen = set()
def note():
    seen.update(l[1] for l in log() if l[0] == "launch")
def calls(type, act, T, D, F):
    h = gated(D, F, type, T, act=act)
    for keep in (0, 1, 2):
        assert forward(h, T, D, F, keep) == H.HF_OK
    assert grad(h, T, D, F) == H.HF_OK
    assert L.hf_gated_grad(h, IN, D, None, 0, IN, D, IN, D, IN, F, 1, IN, 2 * F, None, 0, IN, D, T,
                           OUT, D, OUT, D, OUT + (1 << 40), D, OUT, F, 0) == H.HF_OK
    assert codes_forward(h, T, D, F) == H.HF_OK
    note()
    assert L.hf_gated_destroy(h) == H.HF_OK
for type in (0, 1):
    for T, D, F in %r:
        for act in H.GATED_ACTS.values():
            calls(type, act, T, D, F)
    for T, D, F in %r:
        calls(type, H.HF_SILU, T, D, F)
    for T, n, k in %r:
        h = gated(k, 64, type, T)
        assert product(h, T, n, k) == H.HF_OK
        note()
    h = gated(64, 64, type, 1)
    for R, C in %r:
        nb = (C + 31) // 32
        assert L.hf_gated_pack(h, IN, C, R, C, OUT, C, OUT, nb) == H.HF_OK
        assert L.hf_gated_unpack(h, IN, C, IN, nb, R, C, OUT, C) == H.HF_OK
    for R, C in %r:
        assert L.hf_gated_codes(h, IN, C, R, C, OUT, C, OUT) == H.HF_OK
    note()
result = [[n for n in S.stub_names().decode().split() if n.startswith("hf_gated_")], sorted(seen)]
""" % (N.ACT_SIZES, N.SIZES, N.PRODUCTS, N.PACKS, N.ROW_CODES))
    assert len(names) > 150
    assert sorted(set(names) - set(seen)) == []
