"""Every kernel of the e4m3 product is compared with the oracle in each of its forms: the choice between them, evaluated with the
constants in its source, sends each case of test_gpu_fp8_kernels.py where that says (no GPU needed)."""
import os
import re

import test_gpu_fp8_kernels as cases

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1901_10997_amd", "csrc", "matmul_fp8.hip")


def _constant(name):
    with open(SOURCE) as f:
        return int(re.search(r"constexpr int %s = (\d+);" % name, f.read()).group(1))


def _kernel(M, N):
    few, large = _constant("kFewTiles"), _constant("kLargeTiles")
    tiles = lambda rows: -(-N // 128) * -(-M // rows)  # noqa: E731
    if M > 64 and tiles(64) > few:
        return "tile4" if tiles(128) >= large else "tile2"
    return "rows1" if M <= 16 else "rows4"


def test_the_choice_is_the_one_evaluated_here():
    """The rule itself, as it stands in the source."""
    with open(SOURCE) as f:
        text = f.read()
    assert "if (a.M > 64 && tiles_in(a, 64) > kFewTiles && " in text
    assert "return tiles_in(a, 128) >= kLargeTiles ? tiles_of<4>(a, s) : tiles_of<2>(a, s);" in text
    assert "if (a.M <= 16) hipLaunchKernelGGL(matmul_fp8_rows_kernel<1>" in text


def test_every_form_of_every_kernel_has_a_case():
    reached = set()
    for kernel, M, N, K, out, w_rows, bias, _, _ in cases.CASES:
        assert _kernel(M, N) == kernel, (M, N)
        reached.add((kernel, out, w_rows))
        reached.add((kernel, out, "bias") if bias else (kernel, "no bias"))
    for kernel in ("rows1", "rows4", "tile2", "tile4"):
        assert (kernel, "no bias") in reached
        for out in ("f32", "bf16"):
            assert {(kernel, out, 1), (kernel, out, 128), (kernel, out, "bias")} <= reached, (kernel, out)
    no_columns = cases.test_no_columns_gives_the_bias.pytestmark
    for mark in no_columns:
        if mark.args[0] == "kernel,M,N":
            assert [_kernel(M, N) for _, M, N in mark.args[1]] == [k for k, _, _ in mark.args[1]]
