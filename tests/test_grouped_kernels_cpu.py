"""The kernels of the grouped layers as the compiler takes them, without a GPU."""
import os
import re
import subprocess

import pytest

from paper_2503_21364_amd import build as hip_build

UNITS = sorted(u for u in hip_build.UNITS if u.startswith(("grouped", "checkpoint8")))


def _orders_memory(line):
    return 'asm sideeffect ""' in line and "~{memory}" in line or line.startswith("fence ")


def unordered_barriers(ir):
    """Barriers of workgroups without something in front of them, and behind them, that keeps memory accesses on their side: a
    wait for what is on its way may stand between, nothing else.  `ir`: the translation unit as it is before any optimisation."""
    lines, bad, ours = [line.strip() for line in ir.splitlines()], [], True
    for i, line in enumerate(lines):
        if line.startswith("define "):
            ours = "@_Z" not in line or "3lmk" in line         # __syncthreads() has its own fences
        if not ours or not line.startswith(("call void @llvm.amdgcn.s.barrier(", "tail call void @llvm.amdgcn.s.barrier(")):
            continue
        before = i - 1
        while "@llvm.amdgcn.s.waitcnt(" in lines[before]:
            before -= 1
        if not _orders_memory(lines[before]) or not _orders_memory(lines[i + 1]):
            bad.append((i, lines[before], lines[i + 1]))
    return bad


@pytest.mark.parametrize("unit", UNITS)
def test_no_memory_access_may_pass_a_barrier(unit, tmp_path):
    out = str(tmp_path / "unit.ll")
    subprocess.run([hip_build.hipcc(), *hip_build.COMMON, *hip_build.UNITS[unit], "--cuda-device-only", "-emit-llvm", "-S",
                    "-Xclang", "-disable-llvm-passes", os.path.join(hip_build.CSRC, unit), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        ir = f.read()
    assert re.search(r"define .*_kernel", ir)
    bad = unordered_barriers(ir)
    assert not bad, (len(bad), bad[0])


def test_a_barrier_alone_is_found():
    fence = 'call void asm sideeffect "", "~{memory}"() #1'
    wait, barrier = "call void @llvm.amdgcn.s.waitcnt(i32 112)", "call void @llvm.amdgcn.s.barrier()"
    for lines, count in (([fence, wait, barrier, fence], 0), (["fence release", barrier, "fence acquire"], 0),
                         (["store i32 0, ptr %1", wait, barrier, fence], 1), ([fence, barrier, "%2 = load i32, ptr %1"], 1)):
        assert len(unordered_barriers("\n".join(lines))) == count
