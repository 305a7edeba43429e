"""A rule of the registers that the compiler does not keep by itself, held against the generated code (the sources are cross-compiled here, no GPU needed).

A 64-bit vector shift reads its amount as a pair of registers.  Where the amount lies in the last register that a wave has, the pair's second half lies outside the
allocation and the hardware takes the amount from v0."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

SHIFT = re.compile(r"\s*(?:v_lshlrev_b64|v_lshrrev_b64|v_ashrrev_i64)(?:_e64)?\s+v\[\d+:\d+\],\s*v(\d+),")


def last_register_shifts(lines):
    """(64-bit shifts by an amount in the last register of an allocation, all that shift by a register)"""
    # (registers are given out by eights; a function that is called runs in the allocations of the file's kernels)
    ends = {(int(m.group(1)) + 7) // 8 * 8 for m in (re.search(r"\.amdhsa_next_free_vgpr (\d+)", line) for line in lines) if m}
    name, bad, seen = None, [], 0
    for line in lines:
        m = re.match(r"^(_ZN?\S+):", line)
        if m:
            name = m.group(1)
        m = SHIFT.match(line)
        if m:
            seen += 1
            if int(m.group(1)) + 1 in ends:
                bad.append((name, line.strip()))
    return bad, seen


def test_the_listing_is_understood():
    kernel = ["_ZN1a:", "\tv_lshlrev_b64 v[2:3], v119, -1"]
    assert last_register_shifts(kernel + ["\t.amdhsa_next_free_vgpr 120"])[0] == [("_ZN1a", "v_lshlrev_b64 v[2:3], v119, -1")]
    assert last_register_shifts(kernel + ["\t.amdhsa_next_free_vgpr 113"])[0]
    assert last_register_shifts(kernel + ["\t.amdhsa_next_free_vgpr 121"]) == ([], 1)
    assert last_register_shifts(["\tv_lshlrev_b64 v[2:3], 20, v[6:7]", "\t.amdhsa_next_free_vgpr 8"]) == ([], 0)


def test_no_64_bit_shift_by_the_last_register(tmp_path):
    from paper_2603_19133_amd import build as bld
    if not shutil.which(bld.HIPCC):
        pytest.skip("hipcc not found")

    def listing(src):
        asm = str(tmp_path / (src + ".s"))
        out = subprocess.run([bld.HIPCC, *[f for f in bld.FLAGS if f not in ("-shared", "-fPIC")], "-S", "--cuda-device-only", "-o", asm, os.path.join(bld.CSRC, src)],
                             capture_output=True, text=True)
        assert out.returncode == 0, out.stderr[-2000:]
        return last_register_shifts(open(asm).read().splitlines())

    with ThreadPoolExecutor(8) as pool:
        found = dict(zip(bld.SOURCES, pool.map(listing, bld.SOURCES)))
    assert sum(n for _, n in found.values()) > 20          # (the listings were read)
    assert not any(bad for bad, _ in found.values()), {s: bad for s, (bad, _) in found.items() if bad}
