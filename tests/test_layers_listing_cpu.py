"""The copies to LDS as the compiler leaves them: wait states that this part asks the program for, which the compiler keeps by itself everywhere but around assembly in the source.

Behind a scalar write of m0 a load into LDS needs one wait state, behind a vector instruction's write of a scalar register a buffer instruction that reads it needs five."""
import os
import re
import subprocess

import pytest

from paper_2605_01989_amd import build

CSRC = os.path.join(os.path.dirname(os.path.abspath(build.__file__)), "csrc")
# one kernel for each way of copying: 16-bit rows and columns, floats in large tiles, even and odd rows, halves
KERNELS = ["BF16, false, false, false, false, Waves<2, 2, 2, 2, 3>, false, PartOut", "BF16, true, true, false, false, Waves<2, 4, 8, 4, 2>, false, PartOut",
           "F32, false, true, false, false, Waves<2, 2, 4, 4, 2>, false, PartOut", "BF16, false, true, false, false, Waves<2, 2, 4, 4, 2>, false, PartOut, false, false, true",
           "F16, false, true, false, false, Waves<2, 2, 4, 4, 2>, false, PartOut, true"]


def scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    return set() if not m else {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def written(op, operands):
    """Scalar registers that a vector instruction writes; vcc counts as none that a descriptor is in."""
    if not op.startswith("v_"):
        return set()
    places = operands[:1] if re.match(r"v_(readfirstlane|readlane|cmp)", op) else operands[1:2] if "_co_" in op or "div_scale" in op else []
    return set().union(set(), *(scalars(p) for p in places))


def too_early(listing):
    """(copies to LDS, those among them that come too early, each with the reason)"""
    before, copies, bad = [], 0, []
    for line in listing.splitlines():
        text = line.split(";")[0].strip()
        if not text or text.startswith(".") and not text.startswith(".L"):
            continue
        if text.endswith(":"):
            if not text.startswith(".L"):
                before = []
            continue
        op, _, rest = text.partition("\t" if "\t" in text else " ")
        operands = [o.strip() for o in rest.split(",")]
        if op.startswith("buffer_load") and text.endswith("lds"):
            copies += 1
            reads, states = set().union(set(), *(scalars(o.split()[0]) for o in operands[1:])), 0
            for earlier, its in reversed(before):
                if its[0] == "m0" and states < 1:
                    bad.append(f"m0: {earlier} {its} | {text}")
                if written(earlier, its) & reads:
                    bad.append(f"{states} states: {earlier} {its} | {text}")
                states += 1 + (int(its[0], 0) if earlier == "s_nop" else 0)
                if states >= 5:
                    break
        before = (before + [(op, operands)])[-8:]
    return copies, bad


def test_a_planted_one_is_found():
    calm = "k:\n\tv_readfirstlane_b32 s4, v1\n\ts_mov_b32 m0, s9\n\ts_nop 3\n\tbuffer_load_dwordx4 v0, s[4:7], 0 offen lds\n"
    assert too_early(calm) == (1, [])
    assert too_early(calm.replace("\ts_nop 3\n", ""))[1] and too_early(calm.replace("s_nop 3", "s_nop 2"))[1] and not too_early(calm.replace("s4, v1", "s8, v1").replace("s_nop 3", "s_nop 0"))[1]


@pytest.mark.parametrize("kernel", KERNELS)
def test_copies_wait_for_what_they_read(kernel, tmp_path):
    source, listing = tmp_path / "one.hip", tmp_path / "one.s"
    source.write_text(f'#include "layer_tiles.h"\ntemplate __global__ void ring_products<{kernel}>(Product, PartOut);\n')
    subprocess.check_call([build.HIPCC, *build.FLAGS, "-I", CSRC, "-S", "--offload-device-only", "-o", str(listing), str(source)], stderr=subprocess.DEVNULL)
    copies, bad = too_early(listing.read_text())
    assert copies >= 8 and not bad, (copies, len(bad), bad[:4])
