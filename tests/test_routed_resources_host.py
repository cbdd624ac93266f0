"""What the compiler says of the routed layers' kernels that choose their own shapes (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_1907_01729_amd import build


@pytest.mark.parametrize("source", ["sk_route.hip", "sk_dropout.hip"])
def test_registers_are_enough(source, tmp_path):
    """No kernel keeps registers in memory."""
    run = subprocess.run([build.hipcc(), *build.HIP_FLAGS, "--cuda-device-only", "-c",
                          "-Rpass-analysis=kernel-resource-usage", "-o", str(tmp_path / "out.o"),
                          os.path.join(build.CSRC, source)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr
    kernels = re.split(r"Function Name: ", run.stderr)[1:]
    assert kernels
    for k in kernels:
        scratch, = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", k)
        assert scratch == "0", k.split()[0]
