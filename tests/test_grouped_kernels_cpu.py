"""The kernels of the grouped layers as the compiler takes them, without a GPU."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2503_21364_amd import binding as B
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


# ---- what a compute unit holds of the kernels over small matrices, against what the calls plan with
def _report(unit, tmp_path_factory):
    """Template arguments -> the compiler's report, of the kernels of a unit."""
    cmd = [hip_build.hipcc(), *hip_build.COMMON, *hip_build.UNITS[unit], "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage",
           "-c", os.path.join(hip_build.CSRC, unit), "-o", str(tmp_path_factory.mktemp("obj") / "unit.o")]
    text = subprocess.run(cmd, capture_output=True, text=True, check=True).stderr
    kernels = {}
    for part in text.split("Function Name: ")[1:]:
        numbers = tuple(int(v) for v in re.findall(r"L[jb](\d+)E", part.split()[0]))
        kernels[numbers] = {k: int(v) for k, v in re.findall(r" ([A-Z][A-Za-z]+(?: Spill| \[[^\]]*\])?): (\d+)", part)}
    return kernels


@pytest.fixture(scope="module")
def backward_report(tmp_path_factory):
    return _report("grouped_narrow_bwd.hip", tmp_path_factory)


def _workgroups(lds_bytes):
    return (160 << 10) // ((lds_bytes + 1279) // 1280 * 1280)            # LDS is given out in pieces of 1280 bytes


def _pitch(width):
    return ((width + 3) // 4 | 1) * 4


@pytest.mark.parametrize("k", [16, 32, 48, 64])
@pytest.mark.parametrize("n", [32, 64, 80, 96])
def test_all_runs_of_a_gradient_of_small_matrices_are_held_at_once(backward_report, n, k):
    cn, ck = n // 16, k // 16
    # weights and four wavefronts' tiles of 16 rows; then four copies of the sums, rows of which are 4 floats apart
    floats = max(n * k + 4 * 16 * (_pitch(n) + _pitch(k)), 4 * (n * (k + 4) + n))
    kernels = [backward_report[cn, ck, codes] for codes in (0, 1)]
    held = min(_workgroups(4 * floats), *(r["Occupancy [waves/SIMD]"] for r in kernels))
    rows, blocks = 1 << 30, 1
    runs = B.grouped_linear_backward_bytes(rows, blocks, n, k) // (4 * (n * k + n)) - blocks
    assert 1 <= runs <= 256 * held, (runs / 256, held)
    assert all(r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0 for r in kernels), kernels


@pytest.fixture(scope="module")
def narrow_rows(tmp_path_factory):
    """(columns, sums) -> whether the kernels over small matrices take the product, and its runs."""
    B.lib()
    exe = str(tmp_path_factory.mktemp("host") / "narrow_rows")
    lib = os.path.dirname(hip_build.LIB)
    subprocess.run([hip_build.hipcc(), "-std=c++17", "-O1", f"--offload-arch={hip_build.ARCH}", "--offload-host-only", "-x", "hip",
                    os.path.join(os.path.dirname(__file__), "host", "narrow_rows_driver.cpp"), "-I", hip_build.INCLUDE, "-I", hip_build.CSRC,
                    "-L", lib, "-l:" + os.path.basename(hip_build.LIB), "-Wl,-rpath," + lib, "-o", exe], check=True, capture_output=True)
    lines = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines()
    return {(int(c), int(s)): (f == "1", int(r)) for c, s, f, r in (line.split() for line in lines)}


def _narrow_lds(cols, sums):
    """Weights in steps of four sum indices and tiles of 16 columns (1 .. 6 and 8 of them), the bias, four tiles of 16 rows."""
    tiles = (cols + 15) // 16
    tiles = 8 if tiles == 7 else tiles
    return 4 * ((sums + 3) // 4 * tiles * 64 + tiles * 16 + 4 * 16 * _pitch(sums))


def test_small_matrices_are_those_of_which_a_compute_unit_holds_two(narrow_rows):
    for (cols, sums), (fits, _) in narrow_rows.items():
        small = cols <= 128 and 4 <= sums <= 128 and _narrow_lds(cols, sums) <= 80 << 10
        assert fits == small, (cols, sums, _narrow_lds(cols, sums))


def test_all_runs_of_a_product_of_small_matrices_are_held_at_once(narrow_rows, tmp_path_factory):
    """By LDS; and the registers of every kernel leave four wavefronts a SIMD, or as many as LDS in its smallest size."""
    for (cols, sums), (fits, runs) in narrow_rows.items():
        if fits:
            assert 1 <= runs <= 256 * min(4, _workgroups(_narrow_lds(cols, sums))), (cols, sums, runs / 256)
    for (tiles, pieces, _, gate), r in _report("grouped_narrow.hip", tmp_path_factory).items():
        least = {3: 4, 4: 37, 8: 65}[pieces]                              # sums of the kernel's smallest size
        assert r["Occupancy [waves/SIMD]"] >= min(4, _workgroups(_narrow_lds(16 * tiles, least))), (tiles, pieces, gate)
        assert r["VGPRs Spill"] == 0 and r["ScratchSize [bytes/lane]"] == 0


# ---- the counted wait of kernels whose workgroups take tiles one after the other: no more than N accesses to memory may be left, where N stores stand
# behind the loads that are waited for
def stores_between_marks(assembly):
    """(kernel, N, stores between the marks that no branch can pass by), of every place where a whole tile is stored."""
    found, lines, kernel, i = [], assembly.splitlines(), None, 0
    while i < len(lines):
        label = re.match(r"(_Z\S+):", lines[i])
        kernel = label.group(1) if label else kernel
        mark = re.search(r"; (\d+) stores begin", lines[i])
        i += 1
        if not mark:
            continue
        count, past = 0, None                   # past: the label up to which a branch leads
        while "stores end" not in lines[i]:
            line = lines[i].split(";")[0].strip()
            assert not line.startswith(("s_endpgm", "flat_", "s_branch", "s_setpc")) and "stores begin" not in lines[i], (kernel, line)
            if line == f"{past}:":
                past = None
            elif line.startswith("s_cbranch"):
                past = past or line.split()[-1]
            elif past is None and line.startswith(("global_store_dwordx4", "buffer_store_dwordx4")):
                count += 1
            i += 1
        assert past is None, (kernel, past)
        found.append((kernel, int(mark.group(1)), count))
    return found


@pytest.mark.parametrize("unit,places", [("grouped_linear4.hip", 6), ("grouped_gated_wide.hip", 24)])
def test_as_many_stores_as_the_next_tile_counts(unit, places, tmp_path):
    # places: the tiles' sizes by the types, past the caches or not; by both layouts, both directions and three activations
    out = str(tmp_path / "unit.s")
    subprocess.run([hip_build.hipcc(), *hip_build.COMMON, *hip_build.UNITS[unit], "--cuda-device-only", "-S", os.path.join(hip_build.CSRC, unit), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        found = stores_between_marks(f.read())
    assert len(found) == places
    assert all(count >= n for _, n, count in found), found


def test_a_store_that_a_branch_passes_by_is_not_counted():
    store = "\tglobal_store_dwordx4 v[0:1], v[2:5], off nt"
    skipped = ["\ts_cbranch_execz .LBB0_2", store, ".LBB0_2:    ; %x"]
    for lines, count in (([store, store], 2), ([store, *skipped, store], 2), (skipped, 0), (["\tglobal_load_dwordx4 v[0:3], v[4:5], off"], 0)):
        text = "\n".join(["_ZN3lmk1kE:", "\t; 2 stores begin", *lines, "\t; stores end"])
        assert stores_between_marks(text) == [("_ZN3lmk1kE", 2, count)]
