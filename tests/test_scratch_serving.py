"""The kernels over paged caches, of rotary positions and of adjusted logits keep no register in scratch memory (no GPU; the
assembly of the sources is looked at)."""
import os
import re
import subprocess

import pytest

from paper_2502_06352_amd import build


@pytest.mark.parametrize("source", ["lpp_paged_attention.hip", "lpp_paged.hip", "lpp_rotary.hip", "lpp_logits.hip"])
def test_no_scratch(source, tmp_path):
    out = tmp_path / "a.s"
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + build.FLAGS +
                   ["-w", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, source), "-o", str(out)], stderr=subprocess.DEVNULL, check=True)
    used = re.findall(r"\.private_segment_fixed_size: (\d+)", out.read_text())
    assert used and set(used) == {"0"}
