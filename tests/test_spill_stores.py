"""Vector registers in scratch memory: the reading of assembly, what the build refuses, and the operators' kernels as they are; CPU-only."""
import os
import subprocess

import pytest

from paper_2206_08888_amd import build, spills

SPILL = "\tscratch_store_dword off, v1, off ; 4-byte Folded Spill\n"


def _listing(body):
    return "_Z1kv:\n" + body + "\ts_endpgm\n.Lfunc_end0:\n"


IF = "\ts_and_saveexec_b64 s[0:1], vcc\n\ts_cbranch_execz .LBB0_2\n; %%bb.1:\n\tv_mov_b32_e32 v0, 0\n%s.LBB0_2:\n%s\ts_or_b64 exec, exec, s[0:1]\n%s"
ELSE = ("\ts_and_saveexec_b64 s[0:1], vcc\n\ts_xor_b64 s[0:1], exec, s[0:1]\n\ts_cbranch_execz .LBB0_2\n; %%bb.1:\n\tv_mov_b32_e32 v0, 0\n.LBB0_2:\n"
        "\ts_andn2_saveexec_b64 s[0:1], s[0:1]\n\ts_cbranch_execz .LBB0_4\n%s; %%bb.3:\n.LBB0_4:\n\ts_or_b64 exec, exec, s[0:1]\n%s")
ASIDE = ("\tv_mov_b32_e32 v9, 0\n\ts_and_saveexec_b64 s[0:1], vcc\n\tv_writelane_b32 v9, s0, 3\n\tv_writelane_b32 v9, s1, 4\n\ts_mov_b64 s[0:1], 0\n%s"
         "\tv_readlane_b32 s4, v9, 3\n\tv_readlane_b32 s5, v9, %d\n\ts_or_b64 exec, exec, s[4:5]\n" + SPILL)
LOOP = ("\ts_mov_b64 s[2:3], exec\n.LBB0_1:\n\tv_cmp_gt_i32_e32 vcc, 0, v1\n\ts_and_b64 s[4:5], vcc, exec\n%s\ts_andn2_b64 exec, exec, vcc\n\ts_cbranch_execnz .LBB0_1\n"
        "; %%bb.2:\n%s\ts_mov_b64 exec, s[2:3]\n%s")


@pytest.mark.parametrize("body, partial", [
    (SPILL, 0),
    (IF % ("", "", SPILL), 0), (IF % (SPILL, "", ""), 1), (IF % ("", SPILL, ""), 1),     # behind the if, in it, in front of the instruction that ends it
    (IF % ("", "\ts_mov_b32 s1, 0\n", SPILL), 1),                                       # the mask is lost
    (ELSE % ("", SPILL), 0), (ELSE % (SPILL, ""), 1),
    (ASIDE % ("", 4), 0), (ASIDE % ("", 5), 1), (ASIDE % ("\tv_mov_b32_e32 v9, 1\n", 4), 1),
    (LOOP % ("", "", SPILL), 0), (LOOP % ("", SPILL, ""), 1), (LOOP % (SPILL, "", ""), 1),
    ("\tv_cmpx_gt_i32_e32 0, v1\n" + SPILL, 1), ("\ts_mov_b64 exec, s[2:3]\n" + SPILL, 1), ("\ts_mov_b64 exec, s[2:3]\n\ts_mov_b64 exec, -1\n" + SPILL, 0),
    ("\ts_mov_b64 s[2:3], exec\n\ts_and_b64 exec, exec, vcc\n\tv_mad_u64_u32 v[2:3], s[2:3], v0, v1, v[4:5]\n\ts_or_b64 exec, exec, s[2:3]\n" + SPILL, 1),
    ("\ts_cbranch_scc0 .LBB0_9\n\ts_mov_b64 exec, vcc\n.LBB0_9:\n" + SPILL, 1)])         # narrowed on one of two ways there
def test_partial_stores(body, partial):
    assert len(spills.partial_stores(_listing(body))) == partial
    assert spills.partial_stores(_listing(body.replace(" ; 4-byte Folded Spill", ""))) == []


def test_what_the_build_refuses():
    log = "k.hip:9:1: remark: Function Name: %s [x]\nk.hip:9:1: remark:     VGPRs Spill: %d [x]\n"
    listing = lambda body: _listing(body) + "\t.amdhsa_kernel k\n"
    engine, operator = "_ZN3pop6k_stepINS_1xEEEvv", "_ZN3pop12_GLOBAL__N_15recur10k_backwardIfEEvv"
    build.refuse_spills("k.hip", log % (operator, 0), listing(""))
    build.refuse_spills("k.hip", log % (engine, 7), listing(SPILL))
    with pytest.raises(RuntimeError, match="recur"):
        build.refuse_spills("k.hip", log % (operator, 3), listing(SPILL))
    with pytest.raises(RuntimeError, match="some lanes"):
        build.refuse_spills("k.hip", log % (engine, 7), listing(IF % ("", SPILL, "")))
    with pytest.raises(RuntimeError, match="0 kernels"):
        build.refuse_spills("k.hip", "", listing(""))


@pytest.mark.parametrize("source, kernels", [("k_recurrence.hip", 57), ("k_clip.hip", 7), ("k_orthogonalize.hip", 42)])
def test_kernels_of_operators_do_not_spill(tmp_path, source, kernels):
    asm = tmp_path / "k.s"
    out = subprocess.run([build._hipcc(), *build.FLAGS, "-Rpass-analysis=kernel-resource-usage", "--cuda-device-only", "-S", os.path.join(build.CSRC, source),
                          "-o", str(asm)], check=True, capture_output=True, text=True)
    build.refuse_spills(source, out.stderr, asm.read_text())
    assert len(build.vector_spills(out.stderr)) >= kernels
