"""The waits that the hardware asks software for, where the attention over pages writes instructions by hand, in its compiled form.

A memory instruction whose address is in scalar registers must come at least five wait states (an instruction, or one more than s_nop's
operand) after a vector instruction has written them, and one that loads into LDS one after m0 has been.  The compiler counts them for
its own instructions, not for those of inline assembly."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1707_06990_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def written(line):
    """Scalar registers that a vector instruction writes."""
    m = re.match(r"v_\w+ +(s\d+|s\[\d+:\d+\])(?:,|$)", line)
    if not m:
        return set()
    n = [int(v) for v in re.findall(r"\d+", m[1])]
    return set(range(n[0], n[-1] + 1))


def states(line):
    m = re.match(r"s_nop +(\d+)", line)
    return int(m[1]) + 1 if m else 1


def least_distance(lines, at, wrote, enough):
    """Wait states between line `at` and the last one before it that wrote(line), by the order of lines, up to `enough`."""
    n = 0
    for line in reversed(lines[:at]):
        if wrote(line):
            return n
        n += states(line)
        if n >= enough:
            break
    return enough


def short_waits(lines):
    """(loads into LDS, those of them that come too early)"""
    found, early = 0, []
    for i, line in enumerate(lines):
        m = re.match(r"global_load_lds_dwordx4 v\[?[\d:]+\]?, (off|s\[(\d+):(\d+)\])", line)
        if not m:
            continue
        found += 1
        base = set(range(int(m[2]), int(m[3]) + 1)) if m[2] else set()
        if least_distance(lines, i, lambda t: bool(written(t) & base), 5) < 5:
            early.append((i, line, "address"))
        if least_distance(lines, i, lambda t: re.match(r"s_\w+ +m0,", t), 1) < 1:
            early.append((i, line, "m0"))
    return found, early


def instructions(text):
    lines = (line.split(";")[0].strip() for line in text.splitlines())
    return [line for line in lines if line and not line.startswith(".") and not line.endswith(":")]


def test_the_count_itself():
    load = "global_load_lds_dwordx4 v2, s[22:23]"
    for between, early in (([], 1), (["s_nop 3"], 1), (["s_nop 4"], 0), (["s_mov_b32 m0, s1", "s_nop 0"], 1), (["s_mov_b32 m0, s1", "s_nop 3"], 0)):
        lines = instructions("\n".join(["\tv_readlane_b32 s23, v1, 0 ; x", *between, load]))
        assert len(short_waits(lines)[1]) == early, between
    assert short_waits(["v_cmp_eq_u32_e64 s[20:22], v1, v2", load])[1] and not short_waits(["v_readlane_b32 s24, v1, 0", load])[1]
    assert short_waits(["s_mov_b32 m0, s1", "global_load_lds_dwordx4 v[2:3], off"])[1]


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no compiler")
def test_loads_into_lds_wait_for_their_addresses(tmp_path):
    source, out = "dnb_paged_attn.hip", str(tmp_path / "out.s")
    cmd = [HIPCC, *build.FLAGS, *build.MORE_FLAGS.get(source, []), "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True)
    with open(out) as f:
        found, early = short_waits(instructions(f.read()))
    assert found > 0
    assert not early, early[:5]
