"""The step that re-learns a layer for several tasks (examples/refit_adapters.py): dropout, adapters, their gradients and the updates in the chain they are
made for, every gradient checked against its formula on what the kernel in front of it wrote."""
import importlib.util
import os

import numpy as np
import pytest

import oracle.adapter as A
from util import err_norms, to_host

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("refit_adapters", os.path.join(ROOT, "examples", "refit_adapters.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def chain(ex, layer, x, target, step):
    """The chain's outputs against their formulas at the step counter's value `step`."""
    M, K, N = layer.M, layer.cin, layer.cout
    x64 = to_host(x).reshape(M, K)
    fi = A.factors(M, K, layer.p_input, layer.seed + 1, step) if layer.p_input else None
    f = A.factors(M, K, layer.desc.drop_p, layer.seed, step) if layer.desc.drop_p else None
    if fi is not None:
        mx, l2 = err_norms(to_host(layer.xd), x64 * fi)
        assert mx <= 2.0 ** -8 and l2 <= 2.0 ** -8                              # bfloat16 results: half a unit in the last place
        x64 = to_host(layer.xd)
    w, a, b, s = to_host(layer.w), to_host(layer.a16), to_host(layer.b16), to_host(layer.scale)
    rs, ids = layer.row_start.cpu().numpy(), layer.task.cpu().numpy()
    y, t = A.forward(x64, w, to_host(layer.bias), a, b, s, rs, ids, True, f)
    mx, l2 = err_norms(to_host(layer.y).reshape(M, N), y)
    assert mx <= 2.0 ** -8 and l2 <= 2.0 ** -8
    mx, l2 = err_norms(to_host(layer.t), t)
    assert l2 <= (K + 64) * 2.0 ** -24                                          # float32 sums
    yy, tt = to_host(layer.y).reshape(M, N), to_host(target).reshape(M, N)
    mx, l2 = err_norms(to_host(layer.dz).reshape(M, N), np.where(yy > 0, (yy - tt) / layer.B, 0))
    assert mx <= 2.0 ** -8 and l2 <= 2.0 ** -8
    dz, t32 = to_host(layer.dz).reshape(M, N), to_host(layer.t)
    dx, da, db = A.backward(dz, x64, w, a, b, s, rs, ids, t32, f)
    if fi is not None:
        dx = dx * fi
    # with dropout at the input dx' is rounded before it is scaled, and rounded again
    mx, l2 = err_norms(to_host(layer.dx), dx)
    assert mx <= 2.0 ** -7 and l2 <= 2.0 ** -7
    for got, want in ((layer.da, da), (layer.db, db)):
        mx, l2 = err_norms(to_host(got), want)
        assert mx <= 1e-4 and l2 <= 1e-5                                        # float32 sums of up to M products


@pytest.mark.parametrize("images,size,cin,cout,rank,tasks,p,p_input", [(6, 7, 64, 48, 8, 3, 0.1, 0.0), (5, 14, 136, 200, 12, 2, 0.25, 0.4), (9, 5, 57, 72, 5, 4, 0.0, 0.5)])
def test_gradients_of_the_chain(ex, images, size, cin, cout, rank, tasks, p, p_input):
    import torch
    x, target = ex.teacher(images, size, cin, cout, rank, tasks)
    layer = ex.Tasks(images, size, cin, cout, rank, tasks, p=p, p_input=p_input)
    layer.b16 = (0.2 * torch.randn(layer.b.shape, device="cuda")).to(torch.bfloat16)        # away from the zero it begins with
    layer.step_count.fill_(41)
    layer.gradients(x, target)
    chain(ex, layer, x, target, 41)


@pytest.mark.parametrize("update", ["sgd", "muon"])
def test_a_captured_step_is_the_step(ex, update):
    """Three replays of a captured step: masks move with the counter, gradients are those of the formulas, every parameter moves as its update says."""
    import torch
    x, target = ex.teacher(8, 7, 64, 72, 8, 3)
    layer, plain = (ex.Tasks(8, 7, 64, 72, 8, 3, p=0.2, p_input=0.1, update=update) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(x, target)                    # the first step allocates nothing, but loads kernels
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, target)
    plain.step(x, target)
    for i in range(1, 4):
        graph.replay()
        plain.step(x, target)
        torch.cuda.synchronize()
        assert int(layer.step_count) == i + 1
        for a, b in ((layer.y, plain.y), (layer.dx, plain.dx), (layer.da, plain.da), (layer.db, plain.db), (layer.a, plain.a), (layer.b, plain.b)):
            assert torch.equal(a, b)             # the same kernels in the same order: the same bits
    assert bool((layer.b != 0).any()) and torch.equal(layer.a16, layer.a.to(torch.bfloat16)) and torch.equal(layer.b16, layer.b.to(torch.bfloat16))
    import paper_1708_04728_b200 as dr
    assert dr.dr_device_status()[0] == 0


def test_the_example_runs(ex, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["refit_adapters.py", "--steps", "3", "--images", "4", "--size", "7", "--cin", "64", "--cout", "48", "--drop-input", "0.2"])
    ex.main()
    assert "step   2" in capsys.readouterr().out
