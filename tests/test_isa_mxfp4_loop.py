"""CPU check of the 4-bit product's main loop in the gfx950 assembly.

Operands stream into LDS through direct loads, several stages ahead, and a step of the
loop waits at its barrier with a count: at most (stages - 2) times the loads of a stage may
still be on their way.  That count is only right if a step issues exactly one stage's
loads and no other vector memory instruction is left out of or put between them; and the
loop is only fast if it has no spill and waits nowhere else for memory.  This test
compiles the kernels for gfx950 and checks the loop the compiler actually emitted."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36662_amd", "csrc")
INCLUDE = os.path.join(ROOT, "include")
KERNELS = [(4, 2), (2, 2), (2, 4), (1, 2)]      # tile (in 64 rows) and stages


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    hipcc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("isa") / "mxfp4.s")
    cmd = [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           f"-I{INCLUDE}", f"-I{CSRC}", "--cuda-device-only", "-S", os.path.join(CSRC, "mxfp4_inst.hip"), "-o", out]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout[-3000:]
    with open(out) as f:
        return f.read()


def _ops(text, tile, stages, bf16):
    """The kernel's labels, direct loads, other memory accesses, products, barriers, waits and branches, in order."""
    m = re.search(rf"^_ZN8autoloco14mx_tile_kernelILi{tile}ELi{stages}ELb{bf16}E\w*:(.*?)s_endpgm", text, re.S | re.M)
    ops = []
    for line in m.group(1).split("\n"):
        line = line.split(";")[0].strip()
        if re.match(r"\.LBB\w+:", line):
            ops.append(("label", line[:-1]))
        elif "global_load_lds" in line:
            ops.append(("direct", line))
        elif re.match(r"(global|buffer|flat|scratch)_", line):
            ops.append(("memory", line))
        elif line.startswith("v_mfma"):
            ops.append(("product", line))
        elif line.startswith("s_barrier"):
            ops.append(("barrier", line))
        elif line.startswith("s_waitcnt") and "vmcnt" in line:
            ops.append(("wait", int(re.search(r"vmcnt\((\d+)\)", line).group(1))))
        elif line.startswith(("s_cbranch", "s_branch")):
            ops.append(("branch", line.split()[1]))
    return ops


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("tile,stages", KERNELS)
def test_a_step_waits_for_the_next_stage_only(asm, tile, stages, bf16):
    ops = _ops(asm, tile, stages, bf16)
    loads = 5 * tile                                   # of a wave for a stage: 4 T of codes and T of scales
    where = {v: i for i, (k, v) in enumerate(ops) if k == "label"}
    loops = [ops[where[v] + 1:i] for i, (k, v) in enumerate(ops) if k == "branch" and v in where and where[v] < i]
    main = [b for b in loops if any(k == "direct" for k, _ in b) and not any(k in ("label", "branch") for k, _ in b)]
    assert len(main) == 1, "one loop that issues loads, without a branch inside"
    kinds = [k for k, _ in main[0]]
    assert kinds.count("direct") == loads and kinds.count("memory") == 0
    assert kinds.count("product") == 4 * tile * tile
    assert kinds.count("barrier") == 1 and [v for k, v in main[0] if k == "wait"] == [(stages - 2) * loads]
    assert kinds.index("barrier") == kinds.index("wait") + 1
    # the loads of the stage that the barrier frees come after it; only with one phase of
    # reading ahead does half of them wait for the next step
    after = kinds[kinds.index("barrier"):].count("direct")
    assert after == (loads // 2 if tile == 4 else loads)
    # before the loop: the stages issued but the first may be on their way
    first = next(i for i, (k, v) in enumerate(ops) if k == "wait" and v > 0)
    ahead = (stages - 2) * loads + loads // 2 if tile == 4 else (stages - 1) * loads
    assert ops[first][1] == ahead and ops[first + 1][0] == "barrier"
    assert sum(k == "direct" for k, _ in ops[:first]) == loads + ahead


def test_no_spills(asm):
    spills = [int(n) for n in re.findall(r"\.vgpr_spill_count:\s*(\d+)", asm)]
    private = [int(n) for n in re.findall(r"\.private_segment_fixed_size:\s*(\d+)", asm)]
    assert spills and not any(spills) and not any(private)
