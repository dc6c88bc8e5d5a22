"""The compiler's resource report of the kernels around the 4-bit cache: no vector register may spill, and scalar ones only into lanes of a vector
register, where attention keeps sizes and pointers for its end (its loops over whole tiles touch them once a step at most)."""
import re
import shutil
import subprocess

import pytest

from paper_2401_06706_amd import build as B
from tests.test_kernel_resources import HIPCC


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
@pytest.mark.parametrize("source,scalars", [("fourbit_attn.hip", 64), ("fourbit_rows.hip", 0), ("pages.hip", 0), ("logits_rules.hip", 0)])
def test_no_register_spills(source, scalars, tmp_path):
    flags = [f for f in B.HIPCC_FLAGS if f != "-shared"]
    res = subprocess.run([HIPCC] + flags + ["-c", "-Rpass-analysis=kernel-resource-usage", f"{B.CSRC}/{source}", "-o", str(tmp_path / "x.o")],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-2000:]
    kernels = res.stdout.split("Function Name: ")[1:]
    assert kernels
    for k in kernels:
        vector, scalar = re.findall(r"VGPRs Spill: (\d+)", k), re.findall(r"SGPRs Spill: (\d+)", k)
        scratch = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", k)
        assert [int(n) for n in vector + scratch] == [0, 0] and int(scalar[0]) <= scalars, k[:2000]
