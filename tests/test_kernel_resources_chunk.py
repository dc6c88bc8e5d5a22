"""The compiler's resource report of chunk attention, weight sums, eviction and log probabilities.  Vector registers: none may spill but a few of the
two instances that fill 256 (they are kept for the end of an item); none of the kernel for many rows, which has all 512."""
import re
import shutil
import subprocess

import pytest

from paper_2401_06706_amd import build as B
from tests.test_kernel_resources import HIPCC


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
@pytest.mark.parametrize("source,vectors,scalars", [("chunk_attn.hip", 4, 32), ("chunk_wide.hip", 0, 128), ("weight_sums.hip", 0, 0), ("kv_evict.hip", 0, 0),
                                                    ("token_logprobs.hip", 0, 8)])
def test_register_spills(source, vectors, scalars, tmp_path):
    flags = [f for f in B.HIPCC_FLAGS if f != "-shared"] + B.SOURCE_FLAGS.get(source, [])
    res = subprocess.run([HIPCC] + flags + ["-c", "-Rpass-analysis=kernel-resource-usage", f"{B.CSRC}/{source}", "-o", str(tmp_path / "x.o")],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-2000:]
    kernels = res.stdout.split("Function Name: ")[1:]
    assert kernels
    for k in kernels:
        vector, scalar = int(re.findall(r"VGPRs Spill: (\d+)", k)[0]), int(re.findall(r"SGPRs Spill: (\d+)", k)[0])
        assert vector <= vectors and scalar <= scalars, k[:2000]
