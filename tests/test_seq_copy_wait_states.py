"""The copies into LDS of the kernels for packed sequences and paged caches come late enough after what they read."""
import os
import subprocess

import pytest

from paper_2609_34814_amd import build
from tests.test_copy_wait_states import faults


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="no compiler")
@pytest.mark.parametrize("source", ["packed_attn.hip", "paged_attn.hip", "packed_bwd.hip"])
def test_copies(source, tmp_path):
    out = tmp_path / "listing.s"
    flags = [x for x in build.COMMON + build.SOURCES[source] if x != "-fPIC"]
    subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)], check=True,
                   capture_output=True)
    copies, bad = faults(out.read_text())
    assert copies and not bad, (len(bad), copies, bad[:3])
