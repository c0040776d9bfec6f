"""Host-side checks of the layer norm's entry points (no GPU needed)."""
import pytest

import paper_1708_04728_b200 as dr

P, Q = 4096, 8192               # addresses that are aligned for every argument; nothing is launched


@pytest.mark.parametrize("npix", [0, 4])
def test_one_buffer_for_both_weight_gradients_is_refused(npix):
    """Two sums into one buffer: whichever block comes last would win."""
    n0 = dr.dr_launch_count()
    with pytest.raises(dr.DrError) as e:
        dr.dr_layernorm_bwd(npix, 16, P, 0, P, 0, P, P, P, P, 0, Q, Q, P, 1 << 40, 0, 0)
    assert e.value.status == dr.DR_ERR_INVALID_ARG and dr.dr_launch_count() == n0
