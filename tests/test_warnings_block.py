"""CPU check: the kernels of the feed-forward half of a block compile for gfx950 without a warning, and so does the host's
side of their sources.  Their loops are unrolled through lambdas that make lambdas, where a reference to a parameter of one
that has ended, or an index beyond an array, is only ever a warning."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36662_amd", "csrc")


@pytest.mark.parametrize("side", ["device", "host"])
@pytest.mark.parametrize("source", ["gated_ff_inst.hip", "residual_inst.hip", "muon_inst.hip", "block_api.hip"])
def test_no_warnings(source, side):
    hipcc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not available")
    cmd = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Wall", "-Werror", "-Wno-unused-command-line-argument",
           *(("-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops") if side == "device" else ()), f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
           f"--cuda-{side}-only", "-fsyntax-only", os.path.join(CSRC, source)]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[:3000]
