"""The re-learning step of a layer-normalised slim layer (examples/refit_layernorm.py): the new operators in the chain
they are made for, every gradient checked against its formula on what the kernel in front of it wrote."""
import importlib.util
import os

import numpy as np
import pytest

import dr_synth as S
from util import err_norms, to_dev_bf16, to_host

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("refit_layernorm", os.path.join(ROOT, "examples", "refit_layernorm.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("B,H,cin,cout", [(2, 14, 64, 64), (3, 9, 72, 200), (2, 12, 64, 136)])
def test_gradients_of_the_chain(ex, B, H, cin, cout):
    import oracle.finetune as F
    x, target = ex.teacher(B, H, cin, cout)
    layer = ex.Refit(B, H, cin, cout)
    layer.gamma += 0.1 * __import__("torch").randn(cout, device="cuda")
    layer.gradients(x, target)
    z, y, du, dz = (to_host(t).reshape(-1, cout) for t in (layer.z, layer.y, layer.du, layer.dz))
    t = to_host(target).reshape(-1, cout)
    gamma, beta = to_host(layer.gamma), to_host(layer.beta)
    mean = z.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((z - mean) ** 2).mean(1, keepdims=True) + ex.EPS_LN)
    h = (z - mean) * rstd
    # bfloat16 results: half a unit in the last place is 2^-8 of the value at most, a third of that in the mean square
    mx, l2 = err_norms(y, np.maximum(h * gamma + beta, 0))
    assert mx <= 2.0 ** -8 and l2 <= 2.0 ** -8
    assert abs(float(layer.loss) - 0.5 / B * ((y - t) ** 2).sum()) <= 1e-5 * 0.5 / B * ((y - t) ** 2).sum()
    mx, l2 = err_norms(du, np.where(y > 0, (y - t) / B, 0))
    assert mx <= 2.0 ** -8 and l2 <= 2.0 ** -8
    s = du * gamma
    ref = rstd * (s - s.mean(1, keepdims=True) - h * (s * h).mean(1, keepdims=True))
    mx, l2 = err_norms(dz, ref)
    assert mx <= 2.0 ** -7 and l2 <= 2.0 ** -8
    for got, want in ((layer.dgamma, (du * h).sum(0)), (layer.dbeta, du.sum(0))):
        mx, l2 = err_norms(to_host(got), want)
        assert mx <= 1e-4 and l2 <= 1e-4            # float32 sums; xhat from float32 statistics
    mx, l2 = err_norms(to_host(layer.dw), F.conv2d_wgrad(to_host(x), to_host(layer.dz), 3, 1, 1))
    assert mx <= 2e-5 and l2 <= 1e-5


def test_the_step_updates_every_parameter(ex):
    """The filters move by the orthogonalised momentum: lr * sqrt(max(1, rows / cols)) times a matrix whose singular values lie near one."""
    import torch
    layer = ex.Refit(2, 14, 64, 64, lr=0.01, momentum=0.0)
    x, target = ex.teacher(2, 14, 64, 64)
    w0, g0, b0 = layer.w.clone(), layer.gamma.clone(), layer.beta.clone()
    layer.step(x, target)
    move = (w0 - layer.w).reshape(64, -1).double() / 0.01
    s = torch.linalg.svdvals(move)
    # five steps of the quintic take singular values of 0.01 .. 1 (of the norm) to between 0.68 and 1.14.  One direction has no part in the
    # gradient: the layer norm's dz sums to zero over the channels, so the rows of dW do too (up to the rounding of dz to bfloat16).
    assert 0.3 <= float(s[-2]) and float(s.max()) <= 1.25
    ones = torch.ones(64, dtype=torch.float64, device="cuda") / 8
    assert float((ones @ layer.dw.reshape(64, -1).double()).norm()) <= 0.02 * float(layer.dw.norm())
    assert bool((layer.gamma != g0).all()) and bool((layer.beta != b0).any())
    assert torch.equal(layer.shadow, layer.w.to(torch.bfloat16))


@pytest.mark.parametrize("update", ["muon", "sgd"])
def test_the_loss_falls(ex, update):
    x, target = ex.teacher(4, 14, 64, 96)
    layer = ex.Refit(4, 14, 64, 96, update=update, lr=0.02 if update == "muon" else 0.0005)
    losses = []
    for _ in range(40):
        layer.step(x, target)
        losses.append(float(layer.loss))
    assert all(np.isfinite(losses)) and losses[-1] < 0.7 * losses[0], (losses[0], losses[-1])
    import paper_1708_04728_b200 as dr
    assert dr.dr_device_status()[0] == 0
