"""What the gated block's calls ask of the HIP runtime, read from a log of a stub
that takes the runtime's place: the order of streams, launch sizes, no launch
where there is nothing to do.  No GPU."""

import os
import subprocess

import pytest

from tests import hip_stub

GATED = """
def gated(D=64, F=128, type=H.HF_TYPE_BF16, rows=256, stream=None):
    h = ctypes.c_void_p()
    assert L.hf_gated_create(D, F, H.HF_SILU, type, rows, stream, ctypes.byref(h)) == H.HF_OK
    assert L.hf_gated_set_workspace(h, 1 << 20, L.hf_gated_workspace_bytes(h, 0)) == H.HF_OK
    log()
    return h
def forward(h, T, D=64, F=128, keep=0, shift=0):
    return L.hf_gated_forward(h, IN + shift, D, IN, D, IN, D, IN, F, T, OUT, D, keep, OUT + (1 << 40),
                              2 * F, OUT + (1 << 41), 2 * ((F + 31) // 32))
def grad(h, T, D=64, F=128, acc=0):
    nb = (F + 31) // 32
    return L.hf_gated_grad(h, IN, D, IN, (D + 31) // 32, IN, D, IN, D, IN, F, 2, IN, 2 * F, IN, 2 * nb,
                           IN, D, T, OUT, D, OUT, D, OUT + (1 << 40), D, OUT, F, acc)
def codes_forward(h, T, D=64, F=128):
    return L.hf_gated_forward_codes(h, IN, D, IN, D, IN, IN, D, IN, IN, F, IN, T, OUT, D)
def product(h, T, n, k):
    return L.hf_gated_product(h, IN, k, IN, IN, k, IN, T, n, k, OUT, n)
"""


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    from paper_1606_00511_amd import hf as H
    if not os.path.exists(H.LIB_PATH):
        from paper_1606_00511_amd.build import build_library
        build_library()
    return hip_stub.build(tmp_path_factory.mktemp("stub"))


def test_streams_in_turn(stub):
    """Calls on three streams in turn, a refused one between: each behind those
    before, with whose workspace it works."""
    lines = hip_stub.run(stub, GATED + """
h = gated(stream=0xa00)
for s in (0xa00, 0xb00, 0xa00, 0xc00):
    assert L.hf_gated_set_stream(h, s) == H.HF_OK
    assert forward(h, 100) == H.HF_OK and forward(h, 1000) == H.HF_EINVAL
    assert grad(h, 30) == H.HF_OK and product(h, 5, 100, 64) == H.HF_OK
result = log()
""")
    assert sum(l[0] == "launch" for l in lines) > 12
    assert hip_stub.unordered(lines) == []


def test_captured_call_records_nothing(stub):
    """A captured call makes no event and no wait, and an eager one after it is
    behind the eager ones before."""
    lines = hip_stub.run(stub, GATED + """
h = gated(stream=0xa00)
assert forward(h, 100) == H.HF_OK
S.stub_capture(0xb00, 1)
assert L.hf_gated_set_stream(h, 0xb00) == H.HF_OK
at = len(S.stub_log().splitlines())
assert forward(h, 100) == H.HF_OK and grad(h, 100) == H.HF_OK
to = len(S.stub_log().splitlines())
S.stub_capture(0xb00, 0)
assert L.hf_gated_set_stream(h, 0xc00) == H.HF_OK
assert forward(h, 100) == H.HF_OK
result = [log(), at, to]
""")
    lines, at, to = lines
    assert all(l[0] == "launch" for l in lines[at:to])
    assert hip_stub.unordered(lines, [("0xb00", at, to)]) == []


def test_workspace_of_fewer_rows(stub):
    """A workspace serves calls of up to the rows that its bytes are for, and is
    handed over with nothing at work in the one before."""
    lines = hip_stub.run(stub, GATED + """
h = gated()
assert L.hf_gated_set_workspace(h, 1 << 20, L.hf_gated_workspace_bytes(h, 100)) == H.HF_OK
result = log()
assert forward(h, 100) == H.HF_OK and forward(h, 200) == H.HF_EWORKSPACE
assert b"200 rows above" in L.hf_gated_last_error(h)
""")
    assert lines == [["syncall"]]


def test_no_rows(stub):
    """No rows: nothing runs, but the gradients of the matrices are set to zero
    unless they are added to."""
    lines = hip_stub.run(stub, GATED + """
h = gated()
assert forward(h, 0) == H.HF_OK and codes_forward(h, 0) == H.HF_OK
assert product(h, 0, 100, 64) == H.HF_OK and grad(h, 0, acc=1) == H.HF_OK
none = log()
assert grad(h, 0) == H.HF_OK
result = [none, log()]
""")
    none, some = lines
    assert none == [] and {l[1] for l in some} == {"hf_gated_finish_bf16"}


@pytest.mark.parametrize("type", [0, 1])
def test_launches_fit(stub, type):
    """The largest sizes: fewer than 2^32 work-items and a grid that a launch
    takes, in every call."""
    lines = hip_stub.run(stub, GATED + """
out = []
for D, F, T in ((65536, 65536, 262144), (64, 65536, 262144), (65536, 64, 262144), (1, 1, 262144),
                (65535, 65535, 1000), (1021, 2731, 1), (65536, 65536, 64)):
    h = gated(D, F, %d, T)
    for keep in (0, 1, 2):
        assert forward(h, T, D, F, keep) == H.HF_OK
    assert grad(h, T, D, F) == H.HF_OK
    assert codes_forward(h, T, D, F) == H.HF_OK
    k = max(D, F)
    assert product(h, T, 4194304, k) == H.HF_OK and product(h, 1, 4194304, k) == H.HF_OK
    assert L.hf_gated_destroy(h) == H.HF_OK
    out += log()
h = gated(64, 64, %d, 1)
assert L.hf_gated_pack(h, IN, 65536, 262144, 65536, OUT, 65536, OUT, 2048) == H.HF_OK
assert L.hf_gated_unpack(h, IN, 65536, IN, 2048, 262144, 65536, OUT, 65536) == H.HF_OK
assert L.hf_gated_codes(h, IN, 65536, 4194304, 65536, OUT, 65536, OUT) == H.HF_OK
result = out + log()
""" % (type, type))
    launches = [l for l in lines if l[0] == "launch"]
    assert len(launches) > 100
    for l in launches:
        g, b = [int(v) for v in l[2:5]], [int(v) for v in l[5:8]]
        assert all(v > 0 for v in g + b), l
        assert g[0] * g[1] * g[2] * b[0] * b[1] * b[2] < 1 << 32, l
        assert g[0] * b[0] < 1 << 32 and g[1] < 65536 and g[2] < 65536, l


def test_shares(stub):
    """The sizes whose fp32 gradients units share equally, in tiles of 128 and of 256,
    and some whose do not."""
    lines = hip_stub.run(stub, GATED + """
def grads(D, F, T, type=0):
    h = gated(D, F, type, T)
    assert grad(h, T, D, F) == H.HF_OK and L.hf_gated_destroy(h) == H.HF_OK
    return [l[1] for l in log() if "shares" in l[1] or "grads" in l[1]]
result = [grads(256, 7466, 896), grads(1000, 2500, 2500), grads(1024, 2731, 4096),
          grads(768, 2050, 300), grads(1024, 2731, 4096, 1)]
""")
    assert lines[0] == ["hf_gated_shares_f32"]
    assert lines[1:3] == [["hf_gated_shares_f32_big"]] * 2
    assert all("shares" not in l[0] for l in lines[3:])


def test_ranges(tmp_path):
    """What every launch reads and writes lies in one array of the call, or in one
    part of the workspace: over sizes of all scales, whole and odd, rows apart or
    not, all of what is kept and of the gradients asked for (gated_ranges.cpp)."""
    obj = [str(tmp_path / n) for n in ("ranges.o", "stub.o")]
    hip = ["-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-fPIE", "-O1", "-w"]
    subprocess.run(["/opt/rocm/bin/hipcc", "-x", "hip", "--offload-host-only", "-std=c++17", *hip,
                    "-I" + os.path.join(hip_stub.ROOT, "include"),
                    "-I" + os.path.join(hip_stub.ROOT, "paper_1606_00511_amd", "csrc"), "-c", "-o",
                    obj[0], os.path.join(hip_stub.ROOT, "tests", "gated_ranges.cpp")], check=True)
    subprocess.run(["g++", *hip, "-c", "-o", obj[1],
                    os.path.join(hip_stub.ROOT, "tests", "hip_stub.cpp")], check=True)
    exe = str(tmp_path / "ranges")
    subprocess.run(["g++", "-pie", "-o", exe, *obj], check=True)
    p = subprocess.run([exe, "5000"], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout + p.stderr
