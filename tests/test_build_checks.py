"""What the build reads in the assembly of the cache's kernels (no GPU)."""
import os

from paper_2510_08055_amd import build

MARKS = """
_ZN3moe20compact_tiles_kernelILi8ELi8EEE:
\tglobal_atomic_add v8, v[4:5], v8, off sc0
\ts_waitcnt vmcnt(0)
\ts_cbranch_scc1 .LBB0_2
\tglobal_store_dword v[0:1], v22, off offset:8 sc1
\ts_cbranch_vccnz .LBB0_2
.LBB0_1:
\tglobal_load_dword v38, v[22:23], off offset:8 sc1
\ts_waitcnt vmcnt(0)
\ts_cbranch_execnz .LBB0_1
\tglobal_store_dwordx4 v[6:7], v[98:101], off nt
.LBB0_2:
\t;;#ASMSTART
\ts_waitcnt vmcnt(0)
\t;;#ASMEND
\ts_barrier
\tglobal_atomic_add v1, v[4:5], v1, off offset:4 sc0
\ts_waitcnt vmcnt(0)
.LBB0_3:
\tglobal_store_dword v[4:5], v1, off sc1
\ts_cbranch_execnz .LBB0_3
\ts_endpgm
"""


def test_build_rejects_counts_before_marks_have_arrived():
    """A block that ends without waiting for its mark, on any path, could have it land on a word that the last block has cleared."""
    kernel = "compact_tiles_kernel"
    assert build._marks_behind_counts(MARKS, kernel) == []
    for waits_for in ("vmcnt(1)", "lgkmcnt(0)"):
        bad = MARKS.replace(";;#ASMSTART\n\ts_waitcnt vmcnt(0)", f";;#ASMSTART\n\ts_waitcnt {waits_for}")
        found = build._marks_behind_counts(bad, kernel)
        assert len(found) == 1 and "offset:4" in found[0]
        assert build._marks_behind_counts(bad, "another_kernel") == []
    assert len(build._marks_behind_counts(MARKS.replace(" sc1", ""), kernel)) == 1      # (nothing to check is a fault of the check)


def test_marks_of_the_built_kernels():
    """The same of what the present sources compile to."""
    src, kernel = next(iter(build.MARKS_BEFORE_COUNTS.items()))
    asm = os.path.join(build.OBJ, src.replace(".hip", "-hip-amdgcn-amd-amdhsa-gfx950.s"))
    if not os.path.exists(asm) or os.path.getmtime(asm) < os.path.getmtime(os.path.join(build.CSRC, src)):
        os.makedirs(build.OBJ, exist_ok=True)
        build._compile(src, False)
    with open(asm) as f:
        text = f.read()
    assert len(list(build._listings(text, kernel))) == 5
    assert build._marks_behind_counts(text, kernel) == []
