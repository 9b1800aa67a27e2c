"""The build's check of the 6-bit conversions, whose results must not lie in their operands' registers: on small assembly texts with one
planted mistake each (on the CPU), and over the assembly of the library that is actually built."""
import os
import re

import pytest

from paper_2605_20104_amd import build as b

KERNEL = "_ZN5graft19tree_attn_mx_kernelILi128ELi1ELb0ELb0EEEvPKiS2_S2_NS_12AttnMxParamsE"
GOOD = ["v_cvt_scalef32_2xpk16_fp6_f32 v[66:71], v[2:17], v[18:33], v34", "v_cvt_scalef32_pk32_f32_fp6 v[2:33], v[66:71], v34",
        "v_cvt_scalef32_2xpk16_fp6_f32 v[66:71], v[2:17], v[18:33], s3", "v_cvt_scalef32_pk_fp4_f32 v4, v4, v5, v6"]
BAD = ["v_cvt_scalef32_2xpk16_fp6_f32 v[66:71], v[2:17], v[18:33], v71", "v_cvt_scalef32_2xpk16_fp6_f32 v[12:17], v[2:17], v[18:33], v34",
       "v_cvt_scalef32_2xpk16_fp6_f32 v[28:33], v[2:17], v[18:33], v34", "v_cvt_scalef32_pk32_f32_fp6 v[2:33], v[66:71], v2",
       "v_cvt_scalef32_pk32_f32_fp6 v[2:33], v[28:33], v34"]


def _asm(line):
    return "\n".join(["\t.text", KERNEL + ":", "\ts_nop 0", "\t" + line, "\ts_endpgm", ".Lfunc_end0:"])


@pytest.mark.parametrize("line", GOOD)
def test_results_apart_from_operands(line):
    assert b.check_attention_asm(_asm(line)) == []


@pytest.mark.parametrize("line", BAD)
def test_a_result_in_an_operand(line):
    bad = b.check_attention_asm(_asm(line))
    assert len(bad) == 1 and "operand" in bad[0] and line in bad[0] and "line 4" in bad[0]


def test_the_built_library():
    path = b._asm_of("tree_attn_mx.hip")
    if not os.path.exists(path):
        pytest.skip("no assembly kept from a build in this tree")
    with open(path) as f:
        text = f.read()
    assert len(re.findall(r"v_cvt_scalef32_2xpk16_fp6", text)) >= 20       # every attention kernel has some
    assert b.check_attention_asm(text) == []


def test_the_build_keeps_that_assembly():
    assert "tree_attn_mx.hip" in b.CHECKED and set(b.HAND_SCHEDULED) < set(b.CHECKED)
