"""Gated linear recurrence of many steps and about as many workgroups as compute units, where the choice to cut time depends on the
type: results on both sides of it."""
import pytest

from test_gpu_scan import test_forward_and_gradient as check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,Bn,H,dtype", [
    (520, 11, 1080, "f32"), (520, 12, 1000, "f32"), (520, 12, 1001, "bf16"), (520, 13, 1001, "bf16"), (520, 26, 990, "bf16"), (520, 25, 990, "bf16"),
])
@pytest.mark.parametrize("ragged", [False, True])
def test_both_sides_of_the_cut(T, Bn, H, dtype, ragged):
    check(T, Bn, H, dtype, not ragged, ragged, "tb", 0, 0, True)
