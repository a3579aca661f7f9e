"""Which gradient kernels have matrix products written as assembly: those of d 128, one wavefront a SIMD, and each of them. The check of
their wait states says nothing about a kernel that has none."""
import os
import re
import subprocess

import pytest

from paper_2609_34814_amd import build
from tests.test_wait_states import PRODUCT, faults


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="no compiler")
def test_products_of_every_kernel(tmp_path):
    out = tmp_path / "diff_bwd.s"
    flags = [x for x in build.COMMON if x != "-fPIC"]
    subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, "diff_bwd.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    seen = {}
    for side, d, dv, waves, body in re.findall(r"^_Z\S*diff_(dq|dkv)_kernelILi(\d+)ELi(\d+)ELi(\d+)E\S*:(.*?)\.Lfunc_end", out.read_text(),
                                               re.S | re.M):
        written = sum(PRODUCT in x for x in re.findall(r"#ASMSTART(.*?)#ASMEND", body, re.S))
        seen[side, int(d), int(dv), int(waves)] = written
        assert not faults(body)
        # of 32 tokens of the other side: two maps of d / 16 products each for the scores, and value_dim / 16 for dP
        assert written % (2 * (int(d) // 16) + int(dv) // 16) == 0 and (written > 0) == (d == "128"), (side, d, dv, waves, written)
    assert set(seen) == {(s, *x, w) for s in ("dq", "dkv") for x in ((64, 64), (64, 128), (128, 128), (128, 256)) for w in (2, 4)}
