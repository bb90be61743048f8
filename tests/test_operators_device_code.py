"""The operators' device code (no GPU): rows and images that a lane holds are arrays that must become registers."""
import os
import re
import subprocess

import pytest

from paper_1804_08378_amd import build
from test_device_code import BIN, device_code


@pytest.mark.parametrize("source", ["bs_norm.hip", "bs_norm_resident.hip", "bs_norm_resident_grad.hip", "bs_log_probs.hip"])
def test_operators_keep_nothing_in_scratch_memory(source, tmp_path):
    build.build(force=False)
    obj = os.path.join(build.HERE, "_build", source + ".o")
    if not os.path.exists(obj) or not os.path.exists(BIN):
        pytest.skip("needs the build's objects and the ROCm toolchain")
    notes = subprocess.run([f"{BIN}/llvm-readelf", "--notes", device_code(obj, str(tmp_path))], check=True, capture_output=True, text=True).stdout
    sizes = re.findall(r"\.name:\s+(_Z\w+).*?\.private_segment_fixed_size:\s+(\d+)", notes, re.S)
    assert sizes
    scratch = [(name, int(n)) for name, n in sizes if int(n)]
    assert not scratch, (len(scratch), scratch[:5])
