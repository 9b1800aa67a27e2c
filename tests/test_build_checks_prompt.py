"""The build's check of hand-placed registers covers the prompt attention kernels, and the library that is built passes it."""
import os

import pytest

from paper_2605_20104_amd import build as b

KERNEL = "_ZN5graft18prompt_attn_kernelILi%dELi2ELb0EEEvPKiS2_NS_12PromptParamsE"


def _asm(d, *lines):
    asm = lambda x: [";;#ASMSTART", "\t" + x, ";;#ASMEND"] if x.startswith("v_mfma") else ["\t" + x]                # noqa: E731
    return "\n".join(["\t.text", KERNEL % d + ":", *[y for x in lines for y in asm(x)], "\ts_endpgm", ".Lfunc_end0:"])


@pytest.mark.parametrize("d,managed", [(128, 192), (64, 96)])
def test_managed_registers(d, managed):
    assert b._managed_accvgprs(KERNEL % d) == managed
    assert b.check_attention_asm(_asm(d, "v_accvgpr_read_b32 v1, a%d" % managed)) == []
    bad = b.check_attention_asm(_asm(d, "v_accvgpr_read_b32 v1, a%d" % (managed - 1)))
    assert len(bad) == 1 and "hand-managed" in bad[0]


def test_distances():
    mfma = "v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], a[128:131], 0"
    assert b.check_attention_asm(_asm(128, "s_nop 1", mfma, "s_nop 15", "v_add_f32_e32 v40, v0, v1")) == []
    early = b.check_attention_asm(_asm(128, "s_nop 1", mfma, "v_add_f32_e32 v40, v0, v1"))
    assert len(early) == 1 and "read of an MFMA result" in early[0]
    late = b.check_attention_asm(_asm(128, "s_nop 1", "v_mov_b32_e32 v20, 0", mfma))
    assert len(late) == 1 and "write of an MFMA source" in late[0]


def test_the_built_library():
    path = b._asm_of("prompt_attn_bf16.hip")
    if not os.path.exists(path):
        pytest.skip("no assembly kept from a build in this tree")
    with open(path) as f:
        text = f.read()
    assert text.count("prompt_attn_kernelI") >= 4 and "prompt_attn_bf16.hip" in b.CHECKED
    assert b.check_attention_asm(text) == []
