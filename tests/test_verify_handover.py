"""How the verification's workgroups hand their sums over, checked against the compiled gfx950 code (CPU
only: hipcc compiles, nothing runs).

A workgroup puts its sum with an exchange at device scope and counts itself with an addition; the one
that counts last reads all sums.  Nothing in the language orders the two (a release would, and writes a whole
L2 back), so the source waits for the exchange's old value, which is back once the device sees the new one.
The code must have that wait between every exchange and the addition after it, and every sum
must be read at device scope (sc1), past the reader's own caches.
"""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_21135_amd", "csrc")


def check_asm(text):
    """(exchanges, additions, reads at device scope, violations)."""
    swaps = adds = reads = 0
    waiting, bad = False, []
    for lineno, raw in enumerate(text.splitlines(), 1):
        line = raw.split(";")[0].strip()
        op = line.split()[0] if line else ""
        if op.startswith("global_atomic_swap_x2"):
            swaps, waiting = swaps + 1, True
            if not re.search(r"\bsc0\b", line):
                bad.append((lineno, "the old value is not returned"))
        elif op == "s_waitcnt" and "vmcnt(0)" in line:
            waiting = False
        elif op.startswith("global_atomic_add"):
            adds += 1
            if waiting:
                bad.append((lineno, "counted before the exchange is back"))
        elif op.startswith("global_load") and re.search(r"\bsc1\b", line):
            reads += 1
            if op != "global_load_dwordx2":
                bad.append((lineno, "a sum in parts"))
    return swaps, adds, reads, bad


def test_sums_are_there_before_they_are_counted():
    from paper_2503_21135_amd import build
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    cmd = [build.HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                                         os.path.join(CSRC, "verify.hip"), "-o", "-"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    swaps, adds, reads, bad = check_asm(res.stdout)
    assert not bad
    # six kernels: a put and a count each, a put by the last workgroup alone, two places that read
    assert (swaps, adds, reads) == (12, 6, 12)


def test_checker_catches_a_missing_wait():
    ok = """
    global_atomic_swap_x2 v[4:5], v2, v[4:5], s[2:3] sc0
    s_waitcnt vmcnt(0)
    global_atomic_add v4, v2, v4, s[12:13] sc0
    global_load_dwordx2 v[8:9], v[6:7], off sc1
    """
    assert check_asm(ok) == (1, 1, 1, [])
    assert len(check_asm(ok.replace("s_waitcnt vmcnt(0)", "s_waitcnt lgkmcnt(0)"))[3]) == 1
    assert len(check_asm(ok.replace("s[2:3] sc0", "s[2:3]"))[3]) == 1
    assert check_asm(ok.replace("off sc1", "off"))[2] == 0
