"""Runs a piece of Python against libhf.so with the HIP runtime stubbed
(hip_stub.cpp): nothing is launched, and the log says what would have been."""

import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PRELUDE = """
import ctypes, json
S = ctypes.CDLL({stub!r}, mode=ctypes.RTLD_GLOBAL)
S.stub_log.restype = ctypes.c_char_p
S.stub_capture.argtypes = [ctypes.c_void_p, ctypes.c_int]
from paper_1606_00511_amd import hf as H
L = H.lib()
def log():
    lines = [l.split() for l in S.stub_log().decode().splitlines()]
    S.stub_clear()
    return lines
def vocab(V=1000, D=64, type=H.HF_TYPE_BF16, rows=256, stream=None):
    h = ctypes.c_void_p()
    assert L.hf_vocab_create(V, D, type, rows, stream, ctypes.byref(h)) == H.HF_OK
    # (addresses are never read through)
    assert L.hf_vocab_set_workspace(h, 1 << 20, L.hf_vocab_workspace_bytes(h, 0)) == H.HF_OK
    log()
    return h
IN, OUT = 1 << 44, 1 << 45
"""


def build(folder):
    """The stub, compiled into `folder`."""
    out = os.path.join(str(folder), "libhipstub.so")
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-o", out,
                    os.path.join(ROOT, "tests", "hip_stub.cpp")], check=True)
    return out


def run(stub, code):
    """What `code` leaves in `result`, from a process of its own."""
    text = PRELUDE.format(stub=stub) + code + "\nprint('RESULT', json.dumps(result))\n"
    p = subprocess.run([sys.executable, "-c", text], cwd=ROOT, capture_output=True, text=True)
    assert p.returncode == 0, p.stdout + p.stderr
    line = [l for l in p.stdout.splitlines() if l.startswith("RESULT ")][-1]
    return json.loads(line[len("RESULT "):])


def unordered(lines, captured=()):
    """The launches, as (index, index) pairs, that nothing orders one after the
    other; launches on a stream at a time when it captured (`captured`: pairs
    of a stream and the log lines between) are left out."""
    seen, events, before, pairs = {}, {}, [], []
    for i, l in enumerate(lines):
        if l[0] == "record":
            events[l[1]] = set(seen.get(l[2], ()))
        elif l[0] == "wait":
            seen.setdefault(l[2], set()).update(events.get(l[1], ()))
        elif l[0] == "launch":
            s = l[-1]
            if any(s == c and a <= i < b for c, a, b in captured):
                continue
            have = seen.setdefault(s, set())
            pairs += [(j, i) for j in before if j not in have]
            have.add(i)
            before.append(i)
    return pairs
