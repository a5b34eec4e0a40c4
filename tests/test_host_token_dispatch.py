"""What the launchers of a decoding tenant's operators say of their kernels (profiles turn it into shares of the chip, which plans are searched with) against
what the compiler gave them: registers and LDS from the metadata of the built library's code objects.  No GPU is needed."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2304_11745_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
LLVM = "/opt/rocm/llvm/bin"
TOOLS = [shutil.which(t) or os.path.join(LLVM, t) for t in ("llvm-objdump", "llvm-readelf")]


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """{mangled name: (registers of a wave, LDS bytes, threads)}"""
    where = tmp_path_factory.mktemp("objects")
    lib = shutil.copy(build.LIB, where)                           # the code objects are unpacked beside it
    subprocess.run([TOOLS[0], "--offloading", lib], check=True, capture_output=True, timeout=120)
    out = {}
    for obj in glob.glob(str(where / "*gfx950")):
        notes = subprocess.run([TOOLS[1], "--notes", obj], check=True, capture_output=True, text=True, timeout=120).stdout
        for kernel in notes.split("  - .agpr_count:")[1:]:
            field = {k: re.search(r"^    \.%s: +(\S+)$" % k, kernel, re.M).group(1) for k in ("name", "vgpr_count", "group_segment_fixed_size", "max_flat_workgroup_size")}
            out[field["name"]] = int(field["vgpr_count"]), int(field["group_segment_fixed_size"]), int(field["max_flat_workgroup_size"])
    return out


def held(registers, lds, threads):
    """Workgroups that a unit of four SIMDs, each with 512 registers a lane and room for 8 waves, and 160 KB of LDS holds."""
    waves = min(8, 512 // -(-registers // 8 * 8)) if registers else 8
    by_registers = waves // -(-threads // 256)
    return max(1, min(by_registers, 160 * 1024 // lds if lds else by_registers))


@pytest.mark.skipif(shutil.which("hipcc") is None or not all(map(os.path.exists, TOOLS)), reason="no compiler or no LLVM tools")
def test_launchers_know_their_kernels(tmp_path, compiled):
    exe = str(tmp_path / "token_dispatch_driver")
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-x", "hip", os.path.join(HERE, "token_dispatch_driver.cpp"), "-x", "none", build.LIB, "-Wl,-rpath," + os.path.dirname(build.LIB), "-o", exe]
    built = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert built.returncode == 0, built.stderr[-4000:]
    told = [line.split() for line in subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout.splitlines()]
    wrong, seen = [], set()
    for name, per_unit, lds, threads in told:
        match = [k for k in compiled if name in k]
        assert len(match) == 1, (name, match)
        registers, bytes_, most = compiled[match[0]]
        seen.add(match[0])
        if (int(per_unit), int(lds), int(threads)) != (held(registers, bytes_, most), bytes_, most):
            wrong.append((name, (per_unit, lds, threads), registers, (held(registers, bytes_, most), bytes_, most)))
    assert not wrong, wrong
    ours = {k for k in compiled if re.search("cache_attention|cache_write|cache_read|sample_kernel|qknorm_rope", k)}
    assert seen == ours, ours - seen
