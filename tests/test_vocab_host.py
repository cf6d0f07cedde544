"""What the vocabulary calls ask of the HIP runtime, read from a log of a stub
that takes the runtime's place: the order of streams, launch sizes.  No GPU."""

import os

import pytest

from tests import hip_stub

A, B, C = "0xa00", "0xb00", "0xc00"


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    from paper_1606_00511_amd import hf as H
    if not os.path.exists(H.LIB_PATH):
        from paper_1606_00511_amd.build import build_library
        build_library()
    return hip_stub.build(tmp_path_factory.mktemp("stub"))


EMBED = """
def call(rows=4):
    return L.hf_vocab_embed(h, IN, 64, IN, rows, 1.0, OUT, 64)
"""


def test_streams_in_turn(stub):
    """A call on each of three streams: each one behind those before."""
    lines = hip_stub.run(stub, EMBED + """
h = vocab(stream=0xa00)
for s in (0xa00, 0xb00, 0xa00, 0xc00):
    assert L.hf_vocab_set_stream(h, s) == H.HF_OK and call() == H.HF_OK
result = log()
""")
    assert sum(l[0] == "launch" for l in lines) == 4
    assert hip_stub.unordered(lines) == []


def test_two_switches_without_a_call(stub):
    """A call on A, none or a refused one on B, a call on C: C's is behind
    A's, with whose workspace it works."""
    for between in ("", "assert call(257) == H.HF_EINVAL\n"):
        lines = hip_stub.run(stub, EMBED + """
h = vocab(stream=0xa00)
assert call() == H.HF_OK
assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_OK
""" + between + """
assert L.hf_vocab_set_stream(h, 0xc00) == H.HF_OK
assert call() == H.HF_OK
result = log()
""")
        assert [l[-1] for l in lines if l[0] == "launch"] == [A, C]
        assert hip_stub.unordered(lines) == []
