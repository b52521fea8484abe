"""64-bit selections of values that a wavefront has in common, in the library as it is built.

For `a < b ? a : b` of such numbers the compiler compares on the vector unit (the scalar one has no 64-bit order) and selects on the scalar one.  Between the two an instruction has
to carry the comparison's result into the scalar condition; it has been seen to be missing, and the selection went by whatever an earlier instruction had left there.
"""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2605_29727_amd", "libbastion_tv.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
SETS_SCC = re.compile(r"s_(add|sub|addc|subb|cmp|bitcmp|and|or|xor|andn2|orn2|nand|nor|xnor|not|lshl|lshr|ashr|bfe|abs|absdiff|min|max|wqm|quadmask|bcnt\d)")


def unconnected(listing):
    """(comparison, selection) pairs with nothing between them that sets the scalar condition, where no scalar comparison ahead of them has set it for that selection."""
    found, compared, meant = [], None, False
    for line in listing.splitlines():
        text = line.split("//")[0].strip()
        if not text or text.endswith(":"):
            compared, meant = None, False
            continue
        op = text.split()[0]
        if re.match(r"v_cmp_\w+_[iu]64", op):
            compared = text
        elif op.startswith("s_cselect"):
            if compared and not meant:
                found.append((compared, text))
            elif not compared:
                meant = False
        elif SETS_SCC.match(op):
            compared, meant = None, op.startswith(("s_cmp", "s_bitcmp"))
        elif op.startswith(("s_branch", "s_cbranch", "s_endpgm")):
            compared, meant = None, False
    return found


def test_the_check_sees_a_selection_without_its_comparison():
    bad = """0000000000000100 <k>:
	s_ashr_i32 s19, s18, 31                                    // 000000000100: 90139F12
	v_cmp_gt_i64_e32 vcc, s[4:5], v[2:3]                       // 000000000104: 7CC80404
	s_cselect_b32 s1, s5, s19                                  // 000000000108: 85011305
"""
    assert len(unconnected(bad)) == 1
    assert unconnected(bad.replace("	s_cselect", "	s_cmp_lg_u64 vcc, 0\n	s_cselect")) == []
    assert unconnected(bad.replace("s_ashr_i32 s19, s18, 31", "s_cmp_lt_i32 s14, 7")) == []          # (a selection by that comparison)


def test_no_selection_is_without_its_comparison(tmp_path):
    if not os.path.exists(LIB):
        from paper_2605_29727_amd import build
        build.build()
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.check_call([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, stdout=subprocess.DEVNULL)
    files = sorted(tmp_path.glob("*gfx950"))
    assert files
    for f in files:
        assert unconnected(subprocess.check_output([OBJDUMP, "-d", "--no-show-raw-insn", str(f)], text=True)) == []
