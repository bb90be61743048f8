"""The device code of the group normalisation's exchange (no GPU): a work-group is counted out behind its words."""
import os
import re

import pytest

from paper_1804_08378_amd import build
from test_device_code import BIN, disassemble


def unordered(lines):
    """Whether some way from the words' stores to the count does not wait for them.  The words are stored, and looked for, by agent-scope
    accesses of 64 bits (sc1); every wave passes the barrier behind the last look, and straight in front of that barrier, with no jump between,
    every wave has to wait until its stores are complete."""
    count = [i for i, l in enumerate(lines) if l.startswith("global_atomic_add")]
    words = [i for i, l in enumerate(lines) if l.startswith("global_store_dwordx2") and " sc1" in l]
    looks = [i for i, l in enumerate(lines) if l.startswith("global_load_dwordx2") and " sc1" in l]
    assert len(count) == 1 and words and looks, (len(count), len(words), len(looks))
    barrier = next(i for i in range(looks[-1], len(lines)) if lines[i].startswith("s_barrier"))
    for i in range(barrier - 1, looks[-1], -1):
        if re.match(r"s_waitcnt vmcnt\(0\)", lines[i]):
            return False
        if lines[i].startswith(("s_branch", "s_cbranch", "global_", "flat_", "scratch_", "buffer_")):
            break
    return True


@pytest.mark.parametrize("source", ["bs_norm_resident.hip", "bs_norm_resident_grad.hip"])
def test_the_count_comes_behind_the_words(source, tmp_path):
    build.build(force=False)
    obj = os.path.join(build.HERE, "_build", source + ".o")
    if not os.path.exists(obj) or not os.path.exists(BIN):
        pytest.skip("needs the build's objects and the ROCm toolchain")
    kernels = re.split(r"\n(?=(?:[0-9a-f]+ )?<_Z)", disassemble(obj, str(tmp_path)))
    seen, bad = 0, []
    for text in kernels:
        lines = [l.split("//")[0].strip() for l in text.split("\n")]
        if any(l.startswith("global_atomic_add") for l in lines):
            seen += 1
            if unordered(lines):
                bad.append(lines[0])
    assert seen and not bad, (seen, len(bad), bad[:5])
