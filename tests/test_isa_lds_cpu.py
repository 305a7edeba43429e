"""LDS writes that stand in asm statements, held against the generated code (the sources are cross-compiled here, no GPU needed): the compiler waits for the writes it
has issued itself in front of a barrier, and knows of no others."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

SOURCES = ["split.hip", "compress.hip", "verify.hip", "residual.hip"]


def _listing(src, tmp):
    from paper_2603_19133_amd import build as bld
    asm = str(tmp / (src + ".s"))
    out = subprocess.run([bld.HIPCC, *[f for f in bld.FLAGS if f not in ("-shared", "-fPIC")], "-S", "--cuda-device-only", "-o", asm, os.path.join(bld.CSRC, src)],
                         capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-2000:]
    return open(asm).read().splitlines()


def barriers(lines):
    """(barriers that a hand-issued LDS write may not have reached memory in front of, hand-issued LDS writes)"""
    kernel, hand, flying, bad, writes = None, False, False, [], 0
    for line in lines:
        m = re.match(r"^(_ZN8picospec\S+):", line)
        if m:
            assert not flying, kernel
            kernel = m.group(1)
        t = line.strip()
        if t.startswith((";;#ASMSTART", ";;#ASMEND")):
            hand = t.startswith(";;#ASMSTART")
            continue
        t = t.split(";")[0].strip()
        if hand and t.startswith(("ds_write", "ds_store")):
            flying, writes = True, writes + 1
        elif t.startswith("s_waitcnt") and "lgkmcnt(0)" in t:
            flying = False
        elif t.startswith("s_barrier") and flying:
            bad.append(kernel)
            flying = False
    return bad, writes


def test_the_listing_is_understood():
    hand = [";;#ASMSTART", "ds_write2st64_b32 v1, v2, v3 offset1:128", ";;#ASMEND"]
    assert barriers(["_ZN8picospec1a:", *hand, "s_barrier"]) == (["_ZN8picospec1a"], 1)
    assert barriers(["_ZN8picospec1a:", *hand, "s_waitcnt lgkmcnt(0)", "s_barrier"]) == ([], 1)
    assert barriers(["_ZN8picospec1a:", *hand, "s_waitcnt vmcnt(0)", "s_barrier"])[0]
    assert barriers(["_ZN8picospec1a:", "ds_write_b32 v1, v2", "s_barrier"]) == ([], 0)


def test_hand_issued_lds_writes_are_waited_for_in_front_of_a_barrier(tmp_path):
    from paper_2603_19133_amd import build as bld
    if not shutil.which(bld.HIPCC):
        pytest.skip("hipcc not found")
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        found = dict(zip(SOURCES, pool.map(lambda s: barriers(_listing(s, tmp_path)), SOURCES)))
    assert found["compress.hip"][1] >= 56 and found["split.hip"][1] >= 16, {s: n for s, (_, n) in found.items()}      # (every kernel that claims has some)
    assert not any(bad for bad, _ in found.values()), {s: bad for s, (bad, _) in found.items()}
