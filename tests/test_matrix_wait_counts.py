"""The least number of instructions between a matrix instruction and the first use of its result, as a number of the hardware's and not of this library's: gfx950
asks for 8 behind one of four passes on bf16 and for 10 behind one of eight passes on fp32.  On every path of the built delta rule's kernels, with a branch
between or without (no GPU needed)."""
import os

import pytest

from tests.test_matrix_waits import FAR, LLVM, TOOLS, distances, kernels, library

ASKED = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}


def short_of(found):
    """{(instruction, use): (straight, across a branch)} of what comes too early or is of an instruction whose number is not known"""
    return {key: tuple(least) for key, least in found.items() if min(least) < ASKED.get(key[0], FAR + 1)}


@pytest.mark.skipif(not all(os.path.exists(f"{LLVM}/{t}") for t in TOOLS), reason="no LLVM tools")
def test_no_kernel_asks_too_early(tmp_path):
    seen, short = set(), {}
    for text in library(str(tmp_path)):
        for name, code in kernels(text).items():
            found = distances(code)
            seen |= {key[0] for key in found}
            if short_of(found):
                short[name] = short_of(found)
    assert seen == set(ASKED) and not short


def test_a_kernel_that_is_short_everywhere_is_found():
    """Where no use of an instruction keeps its distance there is no longer one to compare with."""
    lines = ["v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]", "s_nop 5", "v_accvgpr_read_b32 v9, a3", "s_endpgm"]
    code = [(4 * i, line, None) for i, line in enumerate(lines)]
    assert short_of(distances(code)) == {("v_mfma_f32_16x16x32_bf16", "other"): (6, FAR)}
    code[1] = (4, "s_nop 7", None)
    assert not short_of(distances(code))
    assert short_of(distances([(0, "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]", None), *code[1:]]))
