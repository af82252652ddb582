"""How many waves of the paged attention's kernels a SIMD holds, by the registers that the
compiler takes for them: workgroups beyond the first two on a CU hide each other's loads
where they are many, and a few registers more lose a third of them unseen."""
import os
import re
import subprocess

import pytest

from paper_2504_17577_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# (dims, cache type, 16-row blocks of query heads): waves
WAVES = {(64, 0, 1): 4, (64, 0, 2): 3, (64, 1, 1): 4, (64, 1, 2): 3, (64, 2, 1): 4, (64, 2, 2): 3,
         (128, 0, 1): 2, (128, 0, 2): 2, (128, 1, 1): 3, (128, 1, 2): 2, (128, 2, 1): 3, (128, 2, 2): 2}


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_attention_keeps_its_waves(tmp_path):
    source = next(p for p in build.SOURCES if p.endswith("paged.hip"))
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    r = subprocess.run([HIPCC, *flags, "--cuda-device-only", "-c", "-Rpass-analysis=kernel-resource-usage", "-I", build.INCLUDE, "-o",
                        str(tmp_path / "paged.o"), source], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    found, name = {}, None
    for line in r.stderr.splitlines():
        m = re.search(r"Function Name: \S*attn_paged_kernelILi(\d+)ELi(\d)ELi(\d)E", line)
        name = tuple(map(int, m.groups())) if m else None if "Function Name" in line else name
        m = re.search(r"Occupancy \[waves/SIMD\]: (\d+)", line)
        if m and name:
            found[name] = int(m.group(1))
    assert found == WAVES
