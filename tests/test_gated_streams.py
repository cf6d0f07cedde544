"""Calls of the gated block that use no workspace (checkpoints, codes) take part in the
order of a context's calls, as the header has it: read from a log of a stub in the HIP
runtime's place.  No GPU."""

import pytest

from tests import hip_stub
from tests.test_gated_host import GATED, stub  # noqa: F401  (a fixture)

CALLS = GATED + """
def pack(h): return L.hf_gated_pack(h, IN, 64, 40, 64, OUT, 64, OUT + (1 << 40), 2)
def unpack(h): return L.hf_gated_unpack(h, IN, 64, IN, 2, 40, 64, OUT, 64)
def codes(h): return L.hf_gated_codes(h, IN, 64, 40, 64, OUT, 64, OUT + (1 << 40))
"""


@pytest.mark.parametrize("first", ["pack", "unpack", "codes"])
def test_first_call(stub, first):  # noqa: F811
    """The first call of a context, and a block on another stream that may read what it
    wrote."""
    lines = hip_stub.run(stub, CALLS + """
h = gated(stream=0xa00)
assert %s(h) == H.HF_OK
assert L.hf_gated_set_stream(h, 0xb00) == H.HF_OK
assert forward(h, 100) == H.HF_OK
result = log()
""" % first)
    assert sum(l[0] == "launch" for l in lines) > 1
    assert hip_stub.unordered(lines) == []


def test_without_a_workspace(stub):  # noqa: F811
    """Before a workspace is handed over, which is done with nothing at work."""
    lines = hip_stub.run(stub, CALLS + """
h = ctypes.c_void_p()
assert L.hf_gated_create(64, 128, H.HF_SILU, 1, 256, 0xa00, ctypes.byref(h)) == H.HF_OK
assert codes(h) == H.HF_OK
assert L.hf_gated_set_stream(h, 0xb00) == H.HF_OK
assert pack(h) == H.HF_OK and unpack(h) == H.HF_OK
result = log()
""")
    assert [l[0] for l in lines] == ["launch", "record", "wait", "launch", "launch"]
    assert hip_stub.unordered(lines) == []


@pytest.mark.parametrize("call", ["pack", "unpack", "codes"])
def test_after_a_captured_call(stub, call):  # noqa: F811
    """Eager calls, a captured one on another stream between, and one on a third: behind
    the eager ones before; while the stream of those is captured it is refused, and the
    captured ones record nothing."""
    lines, at, to = hip_stub.run(stub, CALLS + """
h = gated(stream=0xa00)
assert forward(h, 100) == H.HF_OK
S.stub_capture(0xb00, 1)
assert L.hf_gated_set_stream(h, 0xb00) == H.HF_OK
at = len(S.stub_log().splitlines())
assert %s(h) == H.HF_OK
to = len(S.stub_log().splitlines())
S.stub_capture(0xb00, 0)
assert L.hf_gated_set_stream(h, 0xc00) == H.HF_OK
assert %s(h) == H.HF_OK
S.stub_capture(0xc00, 1)
assert L.hf_gated_set_stream(h, 0xd00) == H.HF_OK
assert %s(h) == H.HF_EHIP and b"captured" in L.hf_gated_last_error(h)
S.stub_capture(0xc00, 0)
assert %s(h) == H.HF_OK
result = [log(), at, to]
""" % ((call,) * 4))
    assert [l[0] for l in lines[at:to]] == ["launch"]
    assert hip_stub.unordered(lines, [("0xb00", at, to)]) == []
