"""Host-side checks of how the orthogonalised update is run (no GPU needed)."""
import pytest

import paper_1708_04728_b200 as dr


@pytest.mark.parametrize("kind", [-1, 3])
def test_the_self_test_knows_three_kernels(kind):
    n0 = dr.dr_launch_count()
    with pytest.raises(dr.DrError) as e:
        dr.dr_selftest_lost_cluster(kind, 0)
    assert e.value.status == dr.DR_ERR_INVALID_ARG and dr.dr_launch_count() == n0
