"""What the compiler makes of the paged cache's kernels: no instance keeps registers in scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2512_24086_amd import build as b


def resources(source, tmp_path):
    out = subprocess.run([b.hipcc(), *b.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                          os.path.join(b.CSRC, source), "-o", str(tmp_path / "device.o")], check=True, capture_output=True, text=True)
    return re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+).*?Occupancy \[waves/SIMD\]: (\d+).*?VGPRs Spill: (\d+)", out.stderr, re.S)


@pytest.mark.parametrize("source, instances", [("rf2_paged_attn.hip", 27), ("rf2_paged_store.hip", 2), ("rf2_paged_tables.hip", 5)])
def test_no_instance_uses_scratch_memory(source, instances, tmp_path):
    found = resources(source, tmp_path)
    assert len(found) == instances
    assert not [f for f in found if f[1] != "0" or f[3] != "0"]
    for name, _, waves, _ in found:                # what the launches and the search for the parts' length count on
        if "many_attn_kernel" in name:
            assert int(waves) >= (2 if "Li64E" in name else 1), name
        if "few_attn_kernel" in name:
            assert int(waves) >= 2, name
