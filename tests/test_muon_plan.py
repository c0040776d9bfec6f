"""Host-side checks of how the orthogonalised update is run (no GPU needed)."""
import pytest

import paper_1708_04728_b200 as dr


@pytest.mark.parametrize("kind", [-1, 3])
def test_the_self_test_knows_three_kernels(kind):
    n0 = dr.dr_launch_count()
    with pytest.raises(dr.DrError) as e:
        dr.dr_selftest_lost_cluster(kind, 0)
    assert e.value.status == dr.DR_ERR_INVALID_ARG and dr.dr_launch_count() == n0


def test_pairs_only_where_the_device_holds_them():
    """The plan asks the device for its capacity of CTA pairs and of clusters; without a device to ask there is none."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("asks the device that is there")
    for shape in ((1, 2048, 2048), (1, 4096, 9216), (1, 2000, 16000)):
        plan = dr.dr_orthogonalise_plan(*shape)
        assert plan["kernel"] == "alone" and plan["cluster"] == 0 and plan["share"] == 1


def test_plan_of_small_and_odd_matrices():
    small = dr.dr_orthogonalise_plan(1, 64, 147)
    assert small["kernel"] == "small" and small["ctas"] == 1 and small["terms"] == 3 and small["two_steps"] == 0
    assert dr.dr_orthogonalise_plan(1, 147, 64) == small
    alone = dr.dr_orthogonalise_plan(200, 100, 4200)
    assert alone["kernel"] == "alone" and alone["ctas"] == 1 and 1 < alone["groups"] < 200
    assert dr.dr_orthogonalise_plan(0, 300, 300)["groups"] >= 1
    for bad, status in (((1, 0, 4), -1), ((-1, 4, 4), -1), ((1, 70000, 4), -2)):
        with pytest.raises(dr.DrError) as e:
            dr.dr_orthogonalise_plan(*bad)
        assert e.value.status == status
    assert dr._lib.dr_orthogonalise_plan(1, 4, 4, None) == -1
