"""Matrix products written as assembly: the compiler does not know their latency, so nothing but another product may touch a
result within 12 wait states (a product of 8 passes), nor read what the vector unit wrote less than 2 states before."""
import os
import re
import subprocess

import pytest

from paper_2609_34814_amd import build

PRODUCT = "v_mfma_f32_32x32x16_bf16"


def registers(text):
    """Vector registers ('v' and 'a') that operands name."""
    out = set()
    for kind, lo, hi, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+))", text):
        out |= {(kind, n) for n in (range(int(lo), int(hi) + 1) if lo else (int(one),))}
    return out


def faults(listing):
    """(instruction, why) of every listed instruction that comes too soon, in the order of the listing."""
    bad, now, written, moved = [], 0, {}, {}
    for line in listing.splitlines():
        line = line.split(";")[0].strip()
        if not line or line.startswith((".", "/")) or line.endswith(":"):
            continue
        op, _, rest = line.partition(" ")
        op = op.split("\t")[0]
        rest = line[len(op):]
        args = registers(rest)
        first = registers(rest.split(",")[0])
        if op == PRODUCT:
            if any(now - moved.get(r, -99) < 2 for r in args):
                bad.append((line, "operand just written"))
            if any(now - written.get(r, -99) < 12 for r in registers(",".join(rest.split(",")[1:3]))):
                bad.append((line, "operand still on its way"))
            written.update({r: now + 1 for r in first})
        else:
            if any(now - written.get(r, -99) < 12 for r in args):
                bad.append((line, "result still on its way"))
            if op.startswith("v_"):
                moved.update({r: now + 1 for r in first})
        now += int(rest.strip(), 0) + 1 if op == "s_nop" else 1
    return bad


def test_the_check_sees_faults():
    product = f"{PRODUCT} v[0:15], v[16:19], v[20:23], v[0:15]\n"
    assert not faults(product + product + "s_nop 11\nv_mul_f32_e32 v1, v3, v3")
    assert faults(product + "s_nop 10\nv_mul_f32_e32 v1, v3, v40")
    assert faults(product + "ds_write_b32 v50, v15")
    assert faults(product + "s_nop 7\nv_mov_b32_e32 v0, 0")
    assert faults("v_mov_b32_e32 v17, 0\ns_nop 0\n" + product)
    assert not faults("v_mov_b32_e32 v17, 0\ns_nop 1\n" + product)


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="no compiler")
def test_gradient_kernels(tmp_path):
    out = tmp_path / "diff_bwd.s"
    flags = [x for x in build.COMMON if x != "-fPIC"]
    subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, "diff_bwd.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    text = out.read_text()
    written_out = 0
    for name, body in re.findall(r"^(_Z\S*(?:dq|dkv)_kernel\S*):(.*?)\.Lfunc_end", text, re.S | re.M):
        written_out += body.count("#ASMSTART")
        assert not faults(body), (name, faults(body)[:3])
    assert written_out
