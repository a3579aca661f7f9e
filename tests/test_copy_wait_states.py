"""Copies from global memory into LDS written as assembly: they take the LDS address from M0, and the compiler does not look inside for
the waits that its registers need. A copy comes one wait state or more after a scalar write of M0, and five or more after the vector unit
has written a scalar register that it reads."""
import os
import re
import subprocess

import pytest

from paper_2609_34814_amd import build


def scalars(text):
    out = set()
    for lo, hi, one in re.findall(r"\bs(?:\[(\d+):(\d+)\]|(\d+))", text):
        out |= set(range(int(lo), int(hi) + 1)) if lo else {int(one)}
    return out


def faults(listing):
    """(copies, instructions of them that come too soon), in the order of the listing."""
    copies, bad, now, m0, written = 0, [], 0, -99, {}
    for line in listing.splitlines():
        line = line.split(";")[0].strip()
        if not line or line.startswith((".", "/")) or line.endswith(":"):
            continue
        op = line.split()[0]
        args = line[len(op):]
        first = args.split(",")[0].strip()
        if "_load_lds" in op:
            copies += 1
            if now - m0 < 1:
                bad.append((line, "M0 just written"))
            if any(now - written.get(r, -99) < 5 for r in scalars(args)):
                bad.append((line, "address just written by the vector unit"))
        if op.startswith("s_") and first == "m0":
            m0 = now + 1
        if op.startswith("v_"):
            written.update({r: now + 1 for r in scalars(first)})
        now += int(args.strip(), 0) + 1 if op == "s_nop" else 1
    return copies, bad


def test_the_check_sees_faults():
    copy = "global_load_lds_dwordx4 v1, s[4:5]\n"
    assert faults("s_mov_b32 m0, s3\n" + copy)[1] and not faults("s_mov_b32 m0, s3\ns_nop 0\n" + copy)[1]
    assert not faults("s_mov_b32 m0, s3\nv_add_u32_e32 v1, v2, v3\n" + copy)[1]
    assert faults("v_readfirstlane_b32 s5, v0\ns_nop 3\n" + copy)[1] and not faults("v_readfirstlane_b32 s5, v0\ns_nop 4\n" + copy)[1]
    assert faults("s_nop 0\n" + copy + copy)[0] == 2


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="no compiler")
@pytest.mark.parametrize("source", ["diff_attn.hip", "diff_bwd.hip", "attn_fwd.hip"])
def test_copies(source, tmp_path):
    out = tmp_path / "listing.s"
    flags = [x for x in build.COMMON + build.SOURCES[source] if x != "-fPIC"]
    subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)], check=True,
                   capture_output=True)
    copies, bad = faults(out.read_text())
    assert copies and not bad, (len(bad), copies, bad[:3])
