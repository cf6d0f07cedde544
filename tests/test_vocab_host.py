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


def test_a_captured_call_between(stub):
    """An eager call on A, a captured one on B, an eager one on C: C's is
    behind A's, though nothing could be made to wait on B meanwhile.  Then the
    same with B's capture ended before the switch, and with eager calls on B
    itself after its capture."""
    for ended, last in ((False, 0xc00), (True, 0xc00), (True, 0xb00)):
        lines = hip_stub.run(stub, EMBED + """
h = vocab(stream=0xa00)
assert call() == H.HF_OK
S.stub_capture(0xb00, 1)
assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_OK
at = len(S.stub_log().splitlines())
assert call() == H.HF_OK
ended, last = %r, %r
if ended:
    S.stub_capture(0xb00, 0)
to = len(S.stub_log().splitlines())
assert L.hf_vocab_set_stream(h, last) == H.HF_OK
assert call() == H.HF_OK
lines = log()
result = [lines, at, to]
""" % (ended, last))
        lines, at, to = lines
        assert [l[-1] for l in lines if l[0] == "launch"] == [A, B, hex(last)]
        assert hip_stub.unordered(lines, [(B, at, to)]) == [], (ended, last)
        # nothing of A's enters B's capture
        assert all(l[0] == "launch" for l in lines[at:to])


def test_a_switch_to_capture_records_nothing(stub):
    """Events and waits on a stream that captures would become part of the
    graph: none are made, and the eager call after it makes them."""
    lines = hip_stub.run(stub, EMBED + """
h = vocab(stream=0xa00)
assert call() == H.HF_OK
S.stub_capture(0xb00, 1)
assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_OK
assert call() == H.HF_OK
assert call() == H.HF_OK
S.stub_capture(0xb00, 0)
result = log()
""")
    assert [l[0] for l in lines] == ["launch"] * 3


def test_eager_call_behind_a_stream_that_captures(stub):
    """Calls on A, then A captures: an eager call on B could only be put behind
    A's earlier ones through the capture.  It is refused, and goes through once
    the capture has ended."""
    lines = hip_stub.run(stub, EMBED + """
h = vocab(stream=0xa00)
assert call() == H.HF_OK
S.stub_capture(0xa00, 1)
assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_OK
assert call() == H.HF_EHIP
assert b"captur" in L.hf_vocab_last_error(h)
S.stub_capture(0xa00, 0)
assert call() == H.HF_OK
result = log()
""")
    assert [l[-1] for l in lines if l[0] == "launch"] == [A, B]
    assert hip_stub.unordered(lines) == []


@pytest.mark.parametrize("fails", ["hipStreamIsCapturing", "hipEventCreateWithFlags",
                                   "hipEventRecord", "hipStreamWaitEvent"])
def test_a_switch_that_fails(stub, fails):
    """The runtime fails during a switch of streams, which says so; the switch
    made again, or the next call, is behind the earlier ones all the same."""
    for again in (True, False):
        lines = hip_stub.run(stub, EMBED + """
h = vocab(stream=0xa00)
assert call() == H.HF_OK
S.stub_fail(b%r)
assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_EHIP
if %r:
    assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_OK
assert call() == H.HF_OK
result = log()
""" % (fails, again))
        assert [l[-1] for l in lines if l[0] == "launch"] == [A, B]
        assert hip_stub.unordered(lines) == [], again


def launches(lines, name):
    return [(l[1], [int(v) for v in l[2:8]]) for l in lines
            if l[0] == "launch" and l[1].startswith(name)]


def fits(lines):
    """Work-items of a launch: below 2^32 each way, as its size is 32 bits; at
    most 65,535 workgroups in y and z."""
    for l in lines:
        if l[0] == "launch":
            g, b = [int(v) for v in l[2:5]], [int(v) for v in l[5:8]]
            assert all(0 < x * y < 2 ** 32 for x, y in zip(g, b)), l
            assert g[1] < 65536 and g[2] < 65536, l


LIMITS = """
T, D = H.HF_VOCAB_MAX_ROWS, H.HF_VOCAB_MAX_WIDTH
result = []
for type in (H.HF_TYPE_FP32, H.HF_TYPE_BF16):
    h = vocab(%s, D, type, T)
    assert %s == H.HF_OK
    result += log()
    assert L.hf_vocab_destroy(h) == H.HF_OK
"""


def test_embedding_at_both_limits(stub):
    lines = hip_stub.run(stub, LIMITS % (9, "L.hf_vocab_embed(h, IN, D, IN, T, 1.0, OUT, D)"))
    fits(lines)
    # a wave has 64 times 16 bytes of a row
    for (_, (x, y, z, b, _, _)), size in zip(launches(lines, "hf_vocab_embed"), (4, 2)):
        assert x * y * z * (b // 64) >= 262144 * 65536 * size // 1024


def test_gradients_at_both_limits(stub):
    """All rows of the widest kind, with the vocabulary in several pieces (so
    that the row gradients are finished by a kernel of their own)."""
    lines = hip_stub.run(stub, LIMITS % (5000, """L.hf_vocab_loss_grad(
        h, IN, D, IN, D, IN, T, 0.0, IN, None, OUT, D, OUT, D, 0)"""))
    fits(lines)
    assert len(launches(lines, "hf_vocab_finish")) >= 2
    fits(hip_stub.run(stub, LIMITS % (9, "L.hf_vocab_embed_grad(h, IN, T, 1.0, IN, D, OUT, D, 0)")))


@pytest.mark.parametrize("call", [
    "L.hf_vocab_loss(h, IN, 64, IN, 64, IN, 4, 0.0, IN, None)",
    "L.hf_vocab_loss_grad(h, IN, 64, IN, 64, IN, 4, 0.0, IN, None, OUT, 64, OUT, 64, 0)",
    "L.hf_vocab_distill(h, IN, 64, IN, 64, IN, 8, IN, 8, 8, 1.0, 4, 0.0, IN, None)",
    "L.hf_vocab_distill_grad(h, IN, 64, IN, 64, IN, 8, IN, 8, 8, 1.0, 4, 0.0, IN, None, OUT, 64,"
    " OUT, 64, 0)",
    "L.hf_vocab_embed(h, IN, 64, IN, 4, 1.0, OUT, 64)",
    "L.hf_vocab_embed_grad(h, IN, 4, 1.0, IN, 64, OUT, 64, 0)"])
def test_every_call_is_ordered(stub, call):
    """Eager, captured on a second stream, eager on a third: every call with
    kernels on the workspace keeps the order."""
    lines, at, to = hip_stub.run(stub, """
h = vocab(stream=0xa00)
def call():
    assert %s == H.HF_OK
call()
S.stub_capture(0xb00, 1)
assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_OK
at = len(S.stub_log().splitlines())
call()
to = len(S.stub_log().splitlines())
S.stub_capture(0xb00, 0)
assert L.hf_vocab_set_stream(h, 0xc00) == H.HF_OK
call()
result = [log(), at, to]
""" % call)
    used = [l[-1] for l in lines if l[0] == "launch"]
    assert {A, B, C} == set(used) and used.count(A) == used.count(B) == used.count(C)
    assert hip_stub.unordered(lines, [(B, at, to)]) == []


def test_check_waits_for_the_calls_before(stub):
    """hf_vocab_check on a stream that could not be made to wait yet: it waits
    for the calls on the one before too."""
    lines = hip_stub.run(stub, EMBED + """
h = vocab(stream=0xa00)
assert call() == H.HF_OK
S.stub_capture(0xa00, 1)
assert L.hf_vocab_set_stream(h, 0xb00) == H.HF_OK
S.stub_capture(0xa00, 0)
log()
assert L.hf_vocab_check(h) == H.HF_OK
result = log()
""")
    assert ["sync", A] in lines and ["sync", B] in lines
