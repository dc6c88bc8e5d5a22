"""Builds libmcsd.so (HIP, gfx950 only) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmcsd.so")
SOURCES = ["api.hip", "tree_attn.hip", "tree_attn_shared.hip", "tree_attn_any.hip", "verify_sample.hip", "draft_sample.hip", "tree_commit.hip",
           "fourbit_rows.hip", "fourbit_attn.hip", "pages.hip", "logits_rules.hip",
           "chunk_attn.hip", "chunk_wide.hip", "weight_sums.hip", "kv_evict.hip", "token_logprobs.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]
# chunk_wide_kernel holds more than 256 registers: scores and accumulators that vector instructions read stay in the half of the
# register file that these can address, instead of being copied there
SOURCE_FLAGS = {"chunk_wide.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def _run(cmd: list) -> str:
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    # hipcc's host pass does not know the packed-fp32 feature and says so once per file: harmless.
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    return out


def build(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        cmds = [[hipcc] + compile_flags + SOURCE_FLAGS.get(s, []) + ["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objects)]
        cmds.append([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared"] + objects + ["-o", LIB])
        if verbose:
            for c in cmds:
                print(" ".join(c), flush=True)
        with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
            outs = list(pool.map(_run, cmds[:-1]))
        outs.append(_run(cmds[-1]))
    out = "\n".join(o for o in outs if o.strip())
    if out and verbose:
        print(out, flush=True)
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
