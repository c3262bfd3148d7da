"""The kernels around attention keep all values in registers (no GPU): bodies that branch lane by lane, where a
register that was stored to scratch memory and is loaded again can miss lanes."""
import os
import re
import subprocess

import pytest

from paper_2406_20037_amd import build


@pytest.mark.parametrize("source, kernels", [("kern_cache8.hip", 24), ("kern_attn8.hip", 3), ("kern_attn8_bf16.hip", 12),
                                             ("kern_attn8_f16.hip", 12), ("kern_attn8_f32.hip", 8)])
def test_no_kernel_spills(tmp_path, source, kernels):
    out = subprocess.run(
        [build._hipcc(), *build.HIP_FLAGS, "-Rpass-analysis=kernel-resource-usage", "-c",
         os.path.join(build.CSRC, source), "-o", str(tmp_path / "o")],
        capture_output=True, text=True, check=True).stderr
    names = re.findall(r"Function Name: (\S+)", out)
    scratch = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", out)
    assert len(names) == len(scratch) >= kernels
    assert not {n: s for n, s in zip(names, scratch) if s != "0"}
