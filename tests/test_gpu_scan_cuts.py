"""Gated linear recurrence where the choice to cut time into segments changes: numbers of workgroups and of tiles on both sides,
with lengths and without, forward and gradient."""
import pytest

from test_gpu_scan import test_forward_and_gradient as check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,Bn,H,dtype,ragged", [
    (130, 16, 700, "f32", False), (130, 15, 700, "f32", False), (200, 12, 700, "f32", False), (200, 11, 700, "bf16", False),
    (200, 24, 700, "f32", True), (200, 17, 700, "f32", True), (200, 15, 701, "bf16", True), (140, 32, 700, "bf16", False),
    (480, 12, 900, "f32", False), (481, 12, 900, "f32", False), (96, 2, 70, "f32", False), (97, 2, 70, "f32", False), (128, 2, 70, "bf16", True), (129, 2, 70, "bf16", True),
])
@pytest.mark.parametrize("reverse", [False, True])
def test_both_sides_of_the_cut(T, Bn, H, dtype, ragged, reverse):
    check(T, Bn, H, dtype, reverse, ragged, "tb", 0, 0, True)
