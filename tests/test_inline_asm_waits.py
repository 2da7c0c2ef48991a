"""The kernels whose inner loops are inline assembly on pinned registers: no load is in flight into one of these (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

from _asm_waits import conflicts, kernels

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def test_the_check_itself():
    text = """
_Zkernel:
	scratch_load_dword v7, off, off offset:12
	scratch_load_dwordx2 v[10:11], off, off offset:16
	s_cbranch_scc1 .Lother
	;;#ASMSTART
	v_mfma_f32_32x32x16_f16 v[%s], v[20:23], v[24:27], 0
	;;#ASMEND
.Lother:                                ; comment
	s_waitcnt vmcnt(%d)
	;;#ASMSTART
	s_cbranch_vccnz .Lcold
.Lback:
	v_add_f32 v30, v31, v32
	.subsection 1
.Lcold:
	v_add_f32 v7, v%d, v7
	s_branch .Lback
	.subsection 0
	;;#ASMEND
	s_endpgm
.Lfunc_end0:
"""

    def found(*args):
        (name, lines), = kernels(text % args)
        assert name == "_Zkernel"
        c, reached = conflicts(lines)
        assert reached == 1.0
        return sorted({r for _, r in c})

    assert found("40:55", 0, 8) == []
    assert found("0:15", 0, 8) == [7, 10, 11]  # written before the wait
    assert found("40:55", 1, 8) == []  # the older load has ended
    assert found("40:55", 1, 10) == [10]  # in the other subsection
    assert found("40:55", 2, 8) == [7]


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
def test_no_load_is_in_flight_into_a_register_of_a_statement(tmp_path):
    from paper_2604_12219_amd.build import CSRC, FLAGS
    sources = ("pasa_attn", "pasa_cache_tile")
    jobs = []
    for name in sources:
        with open(tmp_path / (name + ".log"), "w") as log:
            cmd = [HIPCC, *FLAGS, "-S", "--cuda-device-only", os.path.join(CSRC, name + ".hip"), "-o", str(tmp_path / (name + ".s"))]
            jobs.append((name, subprocess.Popen(cmd, stdout=log, stderr=subprocess.STDOUT)))
    for name, job in jobs:
        assert job.wait(timeout=600) == 0, (tmp_path / (name + ".log")).read_text()[-2000:]
    checked = 0
    for s in sources:
        for name, lines in kernels((tmp_path / (s + ".s")).read_text()):
            if not any("v_mfma" in line for line in lines):
                continue
            bad, reached = conflicts(lines)
            assert not bad, (name, bad[:4])
            assert reached > 0.99, (name, reached)
            checked += 1
    assert checked > 30
