"""The serving step's kernels keep what they work on in registers: none uses scratch memory (checked on the CPU, from the
compiler's own figures)."""
import os
import re
import subprocess

import pytest

from paper_2606_30391_amd.build import HIPCC_FLAGS, HERE

CSRC = os.path.join(HERE, "csrc")


@pytest.mark.parametrize("name", ["blocks", "cache", "attend"])
def test_no_kernel_uses_scratch_memory(name, tmp_path):
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    cmd = ["hipcc", *flags, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S",
           os.path.join(CSRC, name + ".hip"), "-o", str(tmp_path / "out.s")]
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    text = proc.stdout.decode()
    assert proc.returncode == 0, text[-2000:]
    used = {}
    for block in re.split(r"Function Name: ", text)[1:]:
        used[block.split()[0]] = int(re.search(r"ScratchSize \[bytes/lane\]: (\d+)", block).group(1))
    assert used, "no kernels found"
    assert not any(used.values()), {k: v for k, v in used.items() if v}
