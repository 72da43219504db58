"""Build-time guards of the cross attention kernels, as for the self attention's: no vector register spills, no early touch of
an asm MFMA's result, copies' scalars in time, and stores of whole rows outside loops over descriptors."""
import re

import pytest

from test_build_guards import device_asm, early_reads_of_asm_mfma_results, kernel_instructions, kernel_metadata
from test_build_guards_eight_waves import late_scalars_of_copies


def moves_in_loops(text, name):
    body = text[text.index("\n" + name + ":"):]
    lines = body[:body.index(".end_amdhsa_kernel")].splitlines()
    labels = {m.group(1): i for i, m in enumerate(re.match(r"(\.LBB\w+):", l) for l in lines) if m}
    inside = set()
    for i, l in enumerate(lines):
        m = re.search(r"\ts_c?branch\w*\s+(\.LBB\w+)", l)
        if m and labels.get(m.group(1), i) < i:
            inside |= set(range(labels[m.group(1)], i))
    return sum("v_accvgpr_mov" in lines[i] for i in inside)


@pytest.mark.parametrize("source,kernel,n,asm_form", [
    ("fwd.hip", "cross_forward_kernel", 5, False), ("bwd.hip", "cross_dq_kernel", 3, True),
    ("bwd.hip", "cross_dkdv_eight_kernel", 2, True), ("bwd.hip", "cross_dkdv_four_kernel", 1, True),
    ("bwd.hip", "cross_both_eight_kernel", 2, True), ("bwd.hip", "cross_both_four_kernel", 1, True)])
def test_cross_attention_kernels(source, kernel, n, asm_form):
    text = device_asm(source)
    spills = {k: v for k, v in kernel_metadata(text).items() if kernel in k}
    assert len(spills) == n and not any(spills.values()), spills
    for name in spills:
        ins = kernel_instructions(text, name)
        assert any(l.startswith("v_mfma_f32_32x32x16_bf16") for l in ins), name
        assert any(re.match(r"v_mfma_f32_32x32x16_bf16 v\[", l) for l in ins) or not asm_form, name
        if asm_form:
            assert early_reads_of_asm_mfma_results(ins) == [], name
            assert moves_in_loops(text, name) == 0, name     # nor copies between sets of accumulator registers in a loop
        assert late_scalars_of_copies(ins) == [], name
        assert not any(l.startswith("scratch_") for l in ins), name
        for i, l in enumerate(ins):
            if l.startswith("buffer_store"):
                assert not any(x.startswith("s_cbranch_execnz") for x in ins[i + 1:i + 5]), (name, ins[i:i + 5])
