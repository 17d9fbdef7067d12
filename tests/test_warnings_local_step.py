"""CPU check: the kernels of a local step compile for gfx950 without a warning.  Their launch loops are built from
nested lambdas, where a reference to a variable of an outer one that has ended is only ever a warning."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36662_amd", "csrc")


@pytest.mark.parametrize("source", ["mxfp4_inst.hip", "preference_inst.hip", "clip_inst.hip", "local_api.hip"])
def test_no_warnings(source):
    hipcc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not available")
    cmd = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Wall", "-Werror", "-Wno-unused-command-line-argument",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
           "--cuda-device-only", "-fsyntax-only", os.path.join(CSRC, source)]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[:3000]
