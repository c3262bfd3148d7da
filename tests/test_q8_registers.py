"""The quantization and gated-unit kernels keep all values in registers (no GPU).  Their bodies for tiles that
are not whole branch lane by lane, and a register that is stored there and loaded again at the end of a branch
can miss the lanes that did not take it: such a build has ended in wild addresses."""
import os
import re
import subprocess

from paper_2406_20037_amd import build


def test_no_kernel_spills(tmp_path):
    out = subprocess.run(
        [build._hipcc(), *build.HIP_FLAGS, "-Rpass-analysis=kernel-resource-usage", "-c",
         os.path.join(build.CSRC, "kern_q8.hip"), "-o", str(tmp_path / "o")],
        capture_output=True, text=True, check=True).stderr
    names = re.findall(r"Function Name: (\S+)", out)
    scratch = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", out)
    assert len(names) == len(scratch) >= 21
    assert not {n: s for n, s in zip(names, scratch) if s != "0"}
