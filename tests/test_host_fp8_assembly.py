"""What the assembly within the products of 8-bit rows takes for granted, read from the machine code of the built library (no GPU needed): the register m0, which its
loads set without the compiler's knowledge, holds nothing else; and masks of lanes that comparisons leave are not read by the vector unit within two wait states."""
import glob
import shutil
import subprocess

import pytest

from paper_2304_11745_amd import build
from test_host_matrix_waits import OBJDUMP, functions
from test_host_scalar_waits import scalars

IMPLICIT = ("s_movrel", "v_movrel", "v_interp", "s_sendmsg", "ds_gws", "s_ttracedata")


def uses_of_m0(code):
    """Instructions that use m0, but for a plain move into it with a load into LDS behind it, one instruction between them at most; and loads without such a move."""
    wrong, set_for = [], set()
    for i, (op, args, _) in enumerate(code):
        if op == "s_mov_b32" and args.startswith("m0, s"):
            load = next((k for k in (i + 1, i + 2) if k < len(code) and code[k][0].startswith("buffer_load") and code[k][1].endswith(" lds")), None)
            if load is not None:
                set_for.add(load)
                continue
            wrong.append(i)
        elif "m0" in args.replace(",", " ").split() or op.startswith(IMPLICIT) or op.endswith("_addtid_b32"):
            wrong.append(i)
    return wrong + [i for i, (op, args, _) in enumerate(code) if op.startswith(("buffer_load", "global_load")) and (args.endswith(" lds") or "_lds_" in op) and i not in set_for]


def early_masks(code):
    """Lane masks of class comparisons that a vector instruction reads as one of the next two."""
    out = []
    for i, (op, args, _) in enumerate(code):
        if op == "v_cmp_class_f32_e64":
            mask = scalars(args.split(", ")[0])
            out += [i for o, a, _ in code[i + 1:i + 3] if o.startswith("v_") and scalars(a) & mask]
    return out


CODE = """
0000000000001000 <k>:
	s_mov_b32 m0, s4                                           // 000000001000: BEFC0004
	{0}                                                        // 000000001004: BF800000
	buffer_load_dword v1, s[4:7], s9 offen lds                 // 000000001008: E0511000 09010001
	v_cmp_class_f32_e64 s[10:11], v2, s12                      // 000000001010: D010000A 00001902
	{1}                                                        // 000000001018: BF800000
	v_cndmask_b32_e64 v3, 0, 1, s[10:11]                       // 00000000101C: D1000003 00290280
	s_endpgm                                                   // 000000001024: BF810000
"""


@pytest.mark.parametrize("one,other,m0,masks", [("s_nop 0", "s_nop 0", 0, 1), ("s_nop 0", "v_mov_b32_e32 v4, v5", 0, 1), ("s_add_i32 m0, s5, s6", "s_nop 0", 1, 1), ("s_mov_b32 s8, m0", "s_nop 0", 1, 1),
                                                ("s_sendmsg sendmsg(MSG_INTERRUPT)", "s_nop 0", 1, 1), ("buffer_load_dword v1, s[4:7], s9 offen lds", "s_nop 0", 1, 1),
                                                ("s_nop 0", "v_mov_b32_e32 v4, s10", 0, 2)])
def test_the_reader_sees_what_it_is_for(one, other, m0, masks):
    code = functions(CODE.format(one, other))["k"]
    assert len(uses_of_m0(code)) == m0 and len(early_masks(code)) == masks
    far = functions(CODE.format(one, "s_nop 0").replace("s_endpgm", "v_cndmask_b32_e64 v3, 0, 1, s[10:11]").replace("	v_cndmask_b32_e64 v3, 0, 1, s[10:11]                       // 00000000101C", "	s_nop 1  // 00000000101C"))["k"]
    assert not early_masks(far)


@pytest.mark.skipif(OBJDUMP is None, reason="llvm-objdump not found")
def test_nothing_else_uses_m0_and_masks_are_left_time(tmp_path):
    lib = shutil.copy(build.LIB, tmp_path)                        # the code objects are unpacked beside it
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, timeout=120)
    tiles, compared = 0, 0
    for obj in sorted(glob.glob(str(tmp_path / "*gfx950"))):
        listing = subprocess.run([OBJDUMP, "-d", obj], check=True, capture_output=True, text=True, timeout=120).stdout
        for name, code in functions(listing).items():
            if "fp8_" not in name:
                continue
            assert not early_masks(code), name
            compared += sum(op == "v_cmp_class_f32_e64" for op, _, _ in code)
            if "fp8_tile_kernel" in name:
                assert not uses_of_m0(code), (name, [code[i] for i in uses_of_m0(code)][:5])
                assert any(args.endswith(" lds") for _, args, _ in code)
                tiles += 1
    assert tiles == 14 and compared > 100
