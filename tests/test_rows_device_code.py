"""The device code of the layer normalisation, the activations and the 8-bit form (no GPU): rows that a lane holds are arrays that must become registers."""
import os
import re
import subprocess

import pytest

from paper_1804_08378_amd import build
from test_device_code import BIN, device_code


@pytest.mark.parametrize("source", ["bs_layer_norm.hip", "bs_layer_norm_team.hip", "bs_layer_norm_team_grad.hip", "bs_activate.hip"])
def test_nothing_is_kept_in_scratch_memory(source, tmp_path):
    build.build(force=False)
    obj = os.path.join(build.HERE, "_build", source + ".o")
    if not os.path.exists(obj) or not os.path.exists(BIN):
        pytest.skip("needs the build's objects and the ROCm toolchain")
    notes = subprocess.run([f"{BIN}/llvm-readelf", "--notes", device_code(obj, str(tmp_path))], check=True, capture_output=True, text=True).stdout
    sizes = re.findall(r"\.name:\s+(_Z\w+).*?\.private_segment_fixed_size:\s+(\d+)", notes, re.S)
    assert sizes
    scratch = [(name, int(n)) for name, n in sizes if int(n)]
    assert not scratch, (len(scratch), scratch[:5])
