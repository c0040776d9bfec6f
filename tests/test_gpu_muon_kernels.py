"""The orthogonalised update in float32, as the weights see it (w = 0, momentum 0, rate -1), against the definition in float64 on the
GPU: the bounds that the header states, at the sizes that reach each of its kernels."""
import math

import pytest

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
# What include/dr.h states for the relative error of O (Frobenius): normal values, wide spectra or low rank, one direction, at most 64 rows.
RANDOM, SPREAD, SINGLE, FEW_ROWS = 1e-3, 4e-3, 1e-2, 1e-4


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


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("own_coef", [False, True])
@pytest.mark.parametrize("b,r,c", [(1, 2048, 2048), (1, 2049, 2300), (1, 2000, 16000), (1, 13200, 512), (1, 520, 13207), (40, 130, 4200), (1, 512, 2048)])
def test_steps_of_the_large_kernels(dr, b, r, c, own_coef, steps):
    """CTA pairs, two steps at a time (with a single one behind them where the number is odd), both, shared tiles; coefficients per step."""
    import torch
    u = gaussian(r + c + steps, b, r, c)
    coef = [x for k in range(steps) for x in (3.0 - 0.2 * k, -3.2 + 0.1 * k, 1.2 - 0.05 * k)] if own_coef else None
    o = update(dr, u, steps, coef)
    for i in {0, b - 1}:
        assert error(o[i], u[i], steps, coef) <= RANDOM
    assert torch.equal(update(dr, u, steps, coef), o), "not the same on a second run"


@pytest.mark.parametrize("b,r,c", [(1, 1, 300), (1, 300, 1), (2, 2, 50), (1, 64, 147), (3, 33, 200), (150, 16, 24), (1, 576, 64), (1, 60, 4200), (1, 65, 70), (27, 96, 800),
                                   (1, 100, 4096), (1, 128, 864), (1, 100, 4200), (1, 129, 130), (160, 129, 130), (9, 144, 816), (1, 192, 576), (6, 256, 2304), (1, 2304, 250),
                                   (1, 512, 2049), (1, 1000, 2048), (1, 4100, 1040)])
def test_every_kernel_in_float32(dr, b, r, c):
    u = gaussian(b + r + c, b, r, c)
    o = update(dr, u)
    for i in {0, b // 2, b - 1}:
        assert error(o[i], u[i]) <= (FEW_ROWS if min(r, c) <= 64 else RANDOM)


@pytest.mark.parametrize("r,c", [(40, 72), (64, 576), (60, 4200), (65, 300), (96, 800), (100, 4200), (130, 1000), (200, 1000), (512, 2048), (512, 13200), (2048, 2048), (2000, 16000)])
def test_spectra_and_ranks(dr, r, c):
    """Singular values over two, four and six decades; ranks 16, 4 and 1."""
    import torch
    k = min(r, c)
    p, q = (torch.linalg.qr(gaussian(s + k, s, k).double())[0] for s in (r, c))
    for decades in (2, 4, 6):
        u = (p * torch.logspace(0, -decades, k, device="cuda", dtype=torch.float64) @ q.T).float()[None]
        assert error(update(dr, u)[0], u[0]) <= (FEW_ROWS if k <= 64 else SPREAD), f"{decades} decades"
    for rank in (16, 4, 1):
        u = (gaussian(rank, 1, r, rank) @ gaussian(rank + 1, 1, rank, c))
        assert error(update(dr, u)[0], u[0]) <= (FEW_ROWS if k <= 64 else SINGLE if rank == 1 else SPREAD), f"rank {rank}"


@pytest.mark.parametrize("b,r,c", [(160, 129, 130), (300, 40, 72), (300, 72, 41), (200, 100, 300), (40, 128, 1021), (30, 256, 200), (3, 300, 520), (2, 2048, 2048)])
def test_nan_and_infinity_stay_in_their_matrix(dr, b, r, c):
    """Groups of processors that take matrices in turns, on the buffers of the one before, and matrices side by side: what is clean comes out
    with the same bits, whatever its neighbours held."""
    import torch
    u = gaussian(b + r, b, r, c)
    clean = update(dr, u)
    spoilt = {0: float("nan"), 1: float("inf"), b // 2: float("-inf")} if b > 3 else {0: float("nan")}
    for i, x in spoilt.items():
        u[i, (7 * i) % r, (11 * i + c - 1) % c] = x
    o = update(dr, u)
    for i in range(b):
        if i in spoilt:
            assert bool(torch.isnan(o[i]).all()), f"matrix {i}"
        else:
            assert torch.equal(o[i], clean[i]), f"matrix {i}"


@pytest.mark.parametrize("b,r,c", [(1, 1000, 2048), (1, 512, 2048), (1, 2048, 2048), (1, 512, 13200), (9, 144, 816), (200, 100, 300)])
def test_captured_graph_and_late_input(dr, b, r, c):
    """Launches with and without the kernel in front, replayed from a graph; and on a stream whose input comes late."""
    import torch
    u = gaussian(b + c, b, r, c)
    ref, o = (torch.zeros((b, r, c), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(dr.dr_orthogonalise_workspace_bytes(b, r, c), dtype=torch.uint8, device="cuda")
    call = lambda x, out, stream=None: dr.dr_orthogonalise(b, r, c, x, 5, None, 1e-7, out, ws, ws.numel(), dr.DR_NS_G_F32, stream)
    call(u, ref)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(u, o)
    for _ in range(3):
        o.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, ref)
    side, late, big = torch.cuda.Stream(), torch.zeros_like(u), torch.randn(4096, 4096, device="cuda")
    o.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-4
        late.copy_(u)
    call(late, o, side)
    side.synchronize()
    assert torch.equal(o, ref)
    assert dr.dr_device_status()[0] == 0


@pytest.mark.parametrize("r,c", [(40, 72), (96, 224), (33, 65), (160, 352), (300, 171), (4200, 60)])
def test_any_size_of_the_gradient(dr, r, c):
    """Norms from the smallest numbers float32 holds to the largest, without eps; all zeros with the smallest eps."""
    import torch
    for scale in (1e-43, 1e-39, 1e-36, 1e-20, 1e20, 1e37):
        u = (gaussian(r, 1, r, c).double() * scale).float()
        assert bool(torch.isfinite(u).all()) and float(u.abs().max()) > 0
        assert error(update(dr, u, 5, None, 0.0)[0], u[0], 5, None, 0.0) <= (FEW_ROWS if min(r, c) <= 64 else RANDOM), scale
    for eps in (1e-30, 1e-36, 1e-40, 1e-45):
        assert bool((update(dr, torch.zeros((1, r, c), device="cuda"), 5, None, eps) == 0).all()), eps


@pytest.mark.parametrize("b,r,c", [(150, 4, 4096), (150, 4, 65536), (150, 65536, 3), (75, 7, 40000), (1, 4, 65536), (1, 60, 65536), (3, 65536, 66)])
def test_the_longest_rows(dr, b, r, c):
    """Float32 sums along the longest side the calls take, by one processor and by many."""
    u = gaussian(b + r + c, b, r, c)
    o = update(dr, u)
    few = min(r, c) <= 64 and (b == 1 or max(r, c) <= 4096)
    for i in {0, b - 1}:
        assert error(o[i], u[i]) <= (FEW_ROWS if few else RANDOM)


@pytest.mark.parametrize("shapes", [[(1, 2048, 2048), (1, 64, 147)], [(1, 1000, 2048), (9, 144, 816)], [(1, 512, 2048), (200, 100, 300)], [(1, 512, 13200), (27, 96, 800)]])
def test_beside_convolutions(dr, shapes):
    """Updates on two streams while a third runs convolutions: all of them want tensor memory, and some have to run on all processors at a time."""
    import torch
    us = [gaussian(sum(s), *s) for s in shapes]
    wss = [torch.empty(dr.dr_orthogonalise_workspace_bytes(*s), dtype=torch.uint8, device="cuda") for s in shapes]
    d = dr.dr_conv_desc(k=3, stride=1, pad=1, Cin=192, Cout=256, flags=dr.DR_BIAS | dr.DR_RELU)
    x, w, b = gaussian(1, 64, 28, 28, 192).to(torch.bfloat16), gaussian(2, 256, 3, 3, 192).to(torch.bfloat16) * 0.02, gaussian(3, 256)
    outs = lambda n: [[torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes] for _ in range(n)]
    ys = [torch.zeros((64, 28, 28, 256), dtype=torch.bfloat16, device="cuda") for _ in range(7)]

    def updates(i, o, stream=None):
        dr.dr_orthogonalise(*shapes[i], us[i], 5, None, 1e-7, o[i], wss[i], wss[i].numel(), dr.DR_NS_G_F32, stream)

    def conv(y, stream=None):
        dr.dr_conv_slim_ws(d, 64, 28, 28, x, w, b, None, y, None, None, 0, stream)

    ref, = outs(1)
    for i in range(2):
        updates(i, ref)
    conv(ys[-1])
    got, streams = outs(6), [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for k in range(6):
        for _ in range(4):
            conv(ys[k], streams[2])
        for i in range(2):
            updates(i, got[k], streams[i])
        for _ in range(4):
            conv(ys[k], streams[2])
    st, info = dr.dr_device_status()
    assert st == 0, info
    for o in got:
        assert all(torch.equal(a, e) for a, e in zip(o, ref))
    assert all(torch.equal(y, ys[-1]) for y in ys)
