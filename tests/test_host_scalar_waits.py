"""Wait states between a vector instruction that writes scalar registers (a lane read into one, a comparison) and a memory instruction that reads them:
five at least, whatever way leads there.  The compiler puts them in for its own loads; those written as assembly (fp8_gemm.hip) it does not see.  The machine
code of the built library is read, so no GPU is needed."""
import glob
import re
import shutil
import subprocess

import pytest

from paper_2304_11745_amd import build
from test_host_matrix_waits import OBJDUMP, functions

NEEDED = 5
SCALAR = re.compile(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)")
MEMORY = ("buffer_", "global_", "flat_", "scratch_")


def scalars(text):
    out = set()
    for lo, hi, one in SCALAR.findall(text):
        out.update(range(int(lo), int(hi) + 1) if lo else [int(one)])
    return out


def shortest(code, start):
    """Fewest wait states between the write at `start` and a memory instruction that reads what it wrote; NEEDED if there are as many on every way."""
    best, seen, todo = NEEDED, {}, [(start + 1, 0, frozenset(scalars(code[start][1].split(", ")[0])))]
    while todo:
        i, waits, written = todo.pop()
        while i < len(code) and waits < best and written and waits < seen.get((i, written), NEEDED):
            seen[i, written] = waits
            op, args, to = code[i]
            if op.startswith(MEMORY) and scalars(args) & written:
                best = waits
                break
            if op in ("s_endpgm", "s_setpc_b64", "s_swappc_b64"):
                break
            if op.startswith("s_") and not op.startswith(("s_cmp", "s_bitcmp", "s_nop", "s_waitcnt", "s_barrier", "s_branch", "s_cbranch")):
                written = written - scalars(args.split(", ")[0])          # a scalar instruction's result needs no wait
            waits += int(args, 0) + 1 if op == "s_nop" else 1
            if op == "s_branch":
                i = to
                continue
            if op.startswith("s_cbranch"):
                todo.append((to, waits, written))
            i += 1
    return best


CODE = """
0000000000001000 <k>:
	v_readfirstlane_b32 s4, v0                                 // 000000001000: 7E080500
	s_cbranch_scc1 2                                           // 000000001004: BF850002 <k+0x10>
	s_nop 7                                                    // 000000001008: BF800007
	s_mov_b32 {1}, 0                                             // 00000000100C: BE840080
	s_nop {0}                                                    // 000000001010: BF800000
	buffer_load_dwordx4 v1, s[4:7], s9 offen lds               // 000000001014: E05D1000 09010001
	s_endpgm                                                   // 00000000101C: BF810000
"""


@pytest.mark.parametrize("nops,other,waits", [(0, "s8", 2), (2, "s8", 4), (3, "s8", 5), (0, "s4", 2), (9, "s4", 5)])
def test_the_distance_is_that_of_the_shortest_way(nops, other, waits):
    code = functions(CODE.format(nops, other))["k"]
    assert len(code) == 7 and shortest(code, 0) == waits


@pytest.mark.skipif(OBJDUMP is None, reason="llvm-objdump not found")
def test_scalar_registers_written_by_vector_instructions_are_waited_for(tmp_path):
    lib = shutil.copy(build.LIB, tmp_path)                        # the code objects are unpacked beside it
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, timeout=120)
    checked, kernels, short = 0, set(), []
    for obj in sorted(glob.glob(str(tmp_path / "*gfx950"))):
        listing = subprocess.run([OBJDUMP, "-d", obj], check=True, capture_output=True, text=True, timeout=120).stdout
        for name, code in functions(listing).items():
            for i, (op, args, _) in enumerate(code):
                if not op.startswith("v_") or not args.startswith("s"):
                    continue
                checked += 1
                kernels.add(name)
                got = shortest(code, i)
                if got < NEEDED:
                    short.append((name, i, op, args, got))
    assert not short, short[:10]
    assert checked > 1000 and any("fp8_tile_kernel" in k for k in kernels)
