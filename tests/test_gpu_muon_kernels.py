"""The orthogonalised update in float32, as the weights see it (w = 0, momentum 0, rate -1), against the definition in float64 on the
GPU: the bounds that the header states, at the sizes that reach each of its kernels."""
import math

import pytest

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
# What include/dr.h states for the relative error of O (Frobenius): random matrices, wide spectra or low rank, at most 64 rows.
RANDOM, SPREAD, FEW_ROWS = 1e-3, 4e-3, 1e-4


@pytest.fixture(scope="module")
def dr():
    import paper_1708_04728_b200 as dr
    return dr


def gaussian(seed, *shape):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


def polynomial(u, steps=5, coef=None, eps=1e-7):
    """O of one matrix in float64, with the coefficients as the library holds them."""
    import torch
    coef = torch.tensor(coef or COEF * steps).double().tolist()
    x = u.double().T if u.shape[0] > u.shape[1] else u.double()
    x = x / (x.norm() + eps)
    for k in range(steps):
        a, b, c = coef[3 * k:3 * k + 3]
        gram = x @ x.T
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def update(dr, u, steps=5, coef=None, eps=1e-7):
    import torch
    b, r, c = u.shape
    w, v = torch.zeros_like(u), torch.zeros_like(u)
    ws = torch.full((dr.dr_orthogonalise_workspace_bytes(b, r, c),), 0xFF, dtype=torch.uint8, device="cuda")
    dr.dr_muon_update(b, r, c, w, v, u, -1.0, 0.0, 0.0, False, steps, coef, eps, None, ws, ws.numel())
    st, info = dr.dr_device_status()
    assert st == 0, info
    return w / math.sqrt(max(1.0, r / c))


def error(o, u, *args):
    ref = polynomial(u, *args)
    return float((o.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("b,r,c,steps", [(200, 100, 4200, 1), (200, 100, 4200, 3), (200, 100, 4200, 5), (150, 4200, 100, 4), (160, 60, 8200, 5)])
def test_operands_from_memory(dr, b, r, c, steps):
    """Matrices of one processor each whose X does not fit the L2 cache together: operand slices come from memory and from the cache,
    and land out of order."""
    import torch
    u = gaussian(b + r + steps, b, r, c)
    o = update(dr, u, steps)
    for i in (0, 1, b // 2, b - 1):
        assert error(o[i], u[i], steps) <= (FEW_ROWS if min(r, c) <= 64 else RANDOM)
    for _ in range(3):
        assert torch.equal(update(dr, u, steps), o), "not the same on a second run"


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_a_launch_without_its_cluster_returns(dr, kind):
    """The kernels compare the cluster they find with the one their arguments name before the first instruction that needs it."""
    assert dr.dr_device_status()[0] == 0
    dr.dr_selftest_lost_cluster(kind)
    st, info = dr.dr_device_status()
    assert st == dr.DR_ERR_DEVICE_TIMEOUT and info[1] == 77
    assert dr.dr_device_status()[0] == 0
    u = gaussian(kind, 1, 40, 72)
    assert error(update(dr, u)[0], u[0]) <= FEW_ROWS


@pytest.mark.parametrize("shape,kernel,two_steps", [
    ((1, 2048, 2048), "pair", 0), ((1, 2049, 2300), "pair", 0), ((1, 2000, 16000), "pair", 1), ((1, 13200, 512), "alone", 1),
    ((40, 130, 4200), "alone", 1), ((200, 100, 4200), "alone", 1), ((1, 512, 2048), "share", 0), ((1, 1000, 2048), "alone", 0)])
def test_every_kernel_has_its_shapes(dr, shape, kernel, two_steps):
    """The shapes by which the tests below reach each kernel: a change of the plan's rules must not leave one untested."""
    plan = dr.dr_orthogonalise_plan(*shape)
    assert plan["kernel"] == kernel and plan["two_steps"] == two_steps, plan
