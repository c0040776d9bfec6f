"""GPU parity of the orthogonalised update (Newton-Schulz products) and of the optimiser step on it, against the
definitions in float64."""
import math

import numpy as np
import pytest

import dr_synth as S

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8
COEF = (3.4445, -4.7750, 2.0315)
# Operands of 11 bits: a rounding error of 2^-12 of each operand's size, averaged over the elements of a product and
# carried through the products that follow (factors up to |b| + |c| = 7 per step).  In float64 emulation of that scheme the
# relative error of O is 2e-4 .. 1e-3 for matrices of 16 and more rows.
PRODUCTS = 1.5e-3


@pytest.fixture(scope="module")
def dr():
    import paper_1708_04728_b200 as dr
    return dr


def polynomial(u, steps=5, coef=None, eps=1e-7):
    u = np.asarray(u, np.float64)
    coef = coef or COEF * steps
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (np.sqrt((x * x).sum()) + eps)
    for k in range(steps):
        a, b, c = coef[3 * k:3 * k + 3]
        gram = x @ x.T
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def gradient(name, shape):
    b, r, c = shape
    k = min(16, r, c)
    return (S.normal(0, name + "l", (b, r, k)).astype(np.float64) @ S.normal(0, name + "r", (b, k, c)) * (0.3 / math.sqrt(k))
            + S.normal(0, name, shape)).astype(np.float32)


def scratch(dr, b, r, c):
    import torch
    return torch.full((dr.dr_orthogonalise_workspace_bytes(b, r, c),), 0xFF, dtype=torch.uint8, device="cuda")


def close(got, ref, what=""):
    assert np.all(np.isfinite(got)), what
    rms = np.sqrt((ref ** 2).mean())
    rel = np.sqrt(((got - ref) ** 2).mean()) / rms
    big = np.max(np.abs(got - ref) / (np.abs(ref) + rms))
    assert rel <= U16 + PRODUCTS and big <= 2 * U16 + 20 * PRODUCTS, f"{what}: rel {rel:.2e}, largest {big:.2e}"


def orthogonalise(dr, g, f32, steps=5, coef=None, eps=1e-7):
    import torch
    b, r, c = g.shape
    t = torch.from_numpy(g).cuda()
    t = t if f32 else t.to(torch.bfloat16)
    o = torch.full((b, r, c), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = scratch(dr, b, r, c)
    dr.dr_orthogonalise(b, r, c, t, steps, coef, eps, o, ws, ws.numel(), dr.DR_NS_G_F32 if f32 else 0)
    st, info = dr.dr_device_status()
    assert st == 0, info
    return o, t.double().cpu().numpy()


SHAPES = [(1, 1, 1), (1, 1, 7), (1, 9, 1), (2, 1, 300), (1, 16, 16), (1, 24, 17), (1, 64, 147), (3, 33, 200), (1, 128, 128), (1, 127, 129),
          (1, 130, 70), (1, 64, 576), (1, 192, 576), (1, 256, 256), (1, 257, 255), (2, 200, 1000), (1, 300, 300), (1, 1000, 264), (1, 384, 1500),
          (5, 96, 96), (9, 128, 1024), (40, 64, 640), (1, 100, 4096), (1, 128, 3000), (1, 60, 4096), (1, 2000, 128), (12, 300, 65), (1, 512, 2049), (1, 1030, 515), (20, 40, 72), (150, 16, 24), (1, 48, 5000), (1, 7000, 33), (3, 320, 640)]


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("b,r,c", SHAPES)
def test_orthogonalise(dr, b, r, c, f32):
    import torch
    g = gradient(f"ns{b}.{r}.{c}", (b, r, c))
    o, gd = orthogonalise(dr, g, f32)
    got = o.double().cpu().numpy()
    for i in range(b):
        close(got[i], polynomial(gd[i]), f"matrix {i}")
    again, _ = orthogonalise(dr, g, f32)
    assert torch.equal(o, again), "not the same on a second run"


@pytest.mark.parametrize("r,c", [(1000, 2048), (2048, 1500), (1536, 1536), (1100, 2305), (4100, 1040)])
def test_orthogonalise_large(dr, r, c):
    """Sizes at which every processor has several tiles."""
    g = gradient(f"nsl{r}.{c}", (1, r, c))
    o, gd = orthogonalise(dr, g, True)
    close(o.double().cpu().numpy()[0], polynomial(gd[0]))


@pytest.mark.parametrize("b,r,c", [(1, 256, 2304), (6, 256, 2304), (1, 2304, 250), (2, 200, 6000), (1, 130, 9000), (1, 512, 2048), (1, 320, 4200), (14, 256, 1152), (1, 136, 5001)])
def test_few_long_rows(dr, b, r, c):
    """Sizes at which several processors share a tile of X X^T along the long axis."""
    import torch
    g = gradient(f"fl{b}.{r}.{c}", (b, r, c))
    o, gd = orthogonalise(dr, g, True)
    got = o.double().cpu().numpy()
    for i in range(b):
        close(got[i], polynomial(gd[i]), f"matrix {i}")
    again, _ = orthogonalise(dr, g, True)
    assert torch.equal(o, again), "not the same on a second run"


@pytest.mark.parametrize("b,r,c", [(9, 144, 816), (20, 144, 300), (12, 160, 160), (37, 144, 270), (40, 260, 131), (160, 129, 130)])
def test_many_matrices(dr, b, r, c):
    """Batches whose matrices get groups of processors of every kind, side by side and in turns."""
    g = gradient(f"mm{b}.{r}.{c}", (b, r, c))
    o, gd = orthogonalise(dr, g, True)
    got = o.double().cpu().numpy()
    for i in range(b):
        close(got[i], polynomial(gd[i]), f"matrix {i}")


@pytest.mark.parametrize("r,c", [(80, 208), (160, 200), (400, 140), (136, 1000)])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 7])
def test_steps_and_coefficients(dr, steps, r, c):
    g = gradient(f"st{steps}", (1, r, c))
    coef = []
    for k in range(steps):
        coef += [3.0 - 0.2 * k, -3.2 + 0.1 * k, 1.2 - 0.05 * k]
    for cf in (None, coef):
        o, gd = orthogonalise(dr, g, True, steps, cf)
        close(o.double().cpu().numpy()[0], polynomial(gd[0], steps, cf), f"coef {cf}")


@pytest.mark.parametrize("scale", [1e-18, 1e-6, 1.0, 1e15])
def test_scale_does_not_matter(dr, scale):
    g = (gradient("sc", (1, 96, 224)).astype(np.float64) * scale).astype(np.float32)
    o, gd = orthogonalise(dr, g, True, eps=0.0)
    close(o.double().cpu().numpy()[0], polynomial(gd[0], eps=0.0))


def test_eps_damps_a_small_gradient(dr):
    g = gradient("ep", (1, 40, 72)) * np.float32(1e-9)
    o, gd = orthogonalise(dr, g, True, eps=1e-7)
    close(o.double().cpu().numpy()[0], polynomial(gd[0], eps=1e-7))


@pytest.mark.parametrize("r,c", [(40, 72), (160, 300), (600, 300)])
def test_zero_rank_one_and_repeated_rows(dr, r, c):
    """No row at all, one direction alone, and equal rows: every direction without a part in U stays without one."""
    import torch
    z = np.zeros((1, r, c), np.float32)
    o, _ = orthogonalise(dr, z, True)
    assert bool((o == 0).all())
    one = np.zeros((1, r, c), np.float32)
    one[0, 3, 5] = -2.5
    o, gd = orthogonalise(dr, one, True)
    got = o.double().cpu().numpy()[0]
    ref = polynomial(gd[0])
    assert abs(got[3, 5] - ref[3, 5]) <= (U16 + 4 * PRODUCTS) * abs(ref[3, 5])       # one element: nothing averages
    got[3, 5] = 0
    assert np.all(got == 0)
    rep = np.repeat(gradient("rp", (1, 1, c)), r, axis=1)
    rep[:, r // 2:] = 0
    o, gd = orthogonalise(dr, rep, True)
    got, ref = o.double().cpu().numpy()[0], polynomial(gd[0])
    assert np.all(got[r // 2:] == 0)
    assert np.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum()) <= U16 + 4 * PRODUCTS   # a single direction: nothing averages


def test_nan_and_infinity_stay_in_their_matrix(dr):
    g = gradient("nn", (5, 70, 150))
    g[1, 3, 4] = np.nan
    g[3, 69, 149] = np.inf
    o, gd = orthogonalise(dr, g, True)
    got = o.double().cpu().numpy()
    for i in (0, 2, 4):
        close(got[i], polynomial(gd[i]), f"matrix {i}")
    assert np.all(np.isnan(got[1])) and np.all(np.isnan(got[3]))


def muon(dr, w, v, g, lr, mu, decay, nesterov, shadow=True, steps=5):
    import torch
    b, r, c = w.shape
    wd, vd, gd = (torch.from_numpy(a.copy()).cuda() for a in (w, v, g))
    s = torch.full((b, r, c), float("nan"), dtype=torch.bfloat16, device="cuda") if shadow else None
    ws = scratch(dr, b, r, c)
    dr.dr_muon_update(b, r, c, wd, vd, gd, lr, mu, decay, nesterov, steps, None, 1e-7, s, ws, ws.numel())
    st, info = dr.dr_device_status()
    assert st == 0, info
    return wd, vd, s


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("b,r,c", [(1, 64, 147), (1, 192, 576), (2, 300, 130), (6, 96, 400), (1, 512, 1200), (1, 17, 4099), (1, 1, 33), (1, 900, 64)])
def test_muon_update(dr, b, r, c, nesterov):
    import torch
    g, v = gradient(f"mg{r}.{c}", (b, r, c)), 3 * gradient(f"mv{r}.{c}", (b, r, c))
    w = (S.normal(0, f"mw{r}.{c}", (b, r, c)) * math.sqrt(2 / c)).astype(np.float32)
    lr, mu, decay = 0.02, np.float32(0.95), np.float32(0.1)
    wd, vd, s = muon(dr, w, v, g, lr, float(mu), float(decay), nesterov)
    v64 = float(mu) * v.astype(np.float64) + g
    assert np.all(np.abs(vd.double().cpu().numpy() - v64) <= 2 * U32 * (np.abs(v) + np.abs(g)))
    wn, scale = wd.double().cpu().numpy(), math.sqrt(max(1.0, r / c))
    for i in range(b):
        o = polynomial(g[i] + float(mu) * v64[i] if nesterov else v64[i])
        ref = w[i] - lr * (scale * o + float(decay) * w[i].astype(np.float64))
        step = lr * scale * np.sqrt((o ** 2).mean())
        d = wn[i] - ref
        # rounding of w itself, and the error of O times the size of the step; a single row has one direction, where nothing averages
        assert np.sqrt((d ** 2).mean()) <= 4 * U32 * np.sqrt((w[i] ** 2).mean()) + (4 if min(r, c) == 1 else 1) * PRODUCTS * step
        assert np.abs(d).max() <= 4 * U32 * np.abs(w[i]).max() + 20 * PRODUCTS * step
    assert torch.equal(s, wd.to(torch.bfloat16))
    w2, v2, _ = muon(dr, w, v, g, lr, float(mu), float(decay), nesterov, shadow=False)
    assert torch.equal(wd, w2) and torch.equal(vd, v2)


def test_update_is_along_the_orthogonalised_momentum(dr):
    """momentum 0, no decay, w = 0: the new weights are -lr * O of the gradient, by both entry points."""
    g = gradient("al", (1, 160, 352))
    z = np.zeros_like(g)
    wd, _, _ = muon(dr, z, z, g, 1.0, 0.0, 0.0, False)
    o, _ = orthogonalise(dr, g, True)
    import torch
    assert torch.equal((-wd).to(torch.bfloat16), o)


def test_empty_batch_graph_and_other_stream(dr):
    import torch
    r, c = 96, 288
    n0 = dr.dr_launch_count()
    t = torch.zeros(8, device="cuda")
    ws = scratch(dr, 1, r, c)
    dr.dr_orthogonalise(0, r, c, t, 5, None, 1e-7, t, ws, ws.numel())
    dr.dr_muon_update(0, r, c, t, t, t, 0.1, 0.9, 0.0, True, 5, None, 1e-7, None, ws, ws.numel())
    assert dr.dr_launch_count() == n0
    g = torch.from_numpy(gradient("gr", (1, r, c))).cuda()
    o, ref = torch.zeros((1, r, c), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, r, c), dtype=torch.bfloat16, device="cuda")
    dr.dr_orthogonalise(1, r, c, g, 5, None, 1e-7, ref, ws, ws.numel(), dr.DR_NS_G_F32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dr.dr_orthogonalise(1, r, c, g, 5, None, 1e-7, o, ws, ws.numel(), dr.DR_NS_G_F32)
    for _ in range(3):
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, ref)
    side, late = torch.cuda.Stream(), torch.zeros_like(g)
    ws2 = scratch(dr, 1, r, c)
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    o.zero_()
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-4
        late.copy_(g)
    dr.dr_orthogonalise(1, r, c, late, 5, None, 1e-7, o, ws2, ws2.numel(), dr.DR_NS_G_F32, stream=side)
    side.synchronize()
    assert torch.equal(o, ref)


def test_two_streams_at_once(dr):
    """Calls on two streams with a workspace each, overlapping on the device."""
    import torch
    shapes = [(1, 256, 1152), (2, 192, 640)]
    gs = [torch.from_numpy(gradient(f"two{r}", (b, r, c))).cuda() for b, r, c in shapes]
    wss = [scratch(dr, *s) for s in shapes]
    refs = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    for s, g, ws, o in zip(shapes, gs, wss, refs):
        dr.dr_orthogonalise(*s, g, 5, None, 1e-7, o, ws, ws.numel(), dr.DR_NS_G_F32)
    torch.cuda.synchronize()
    outs = [[torch.zeros(s, dtype=torch.bfloat16, device="cuda") for _ in range(10)] for s in shapes]
    streams = [torch.cuda.Stream() for _ in shapes]
    torch.cuda.synchronize()
    for k in range(10):
        for s, g, ws, o, st in zip(shapes, gs, wss, outs, streams):
            dr.dr_orthogonalise(*s, g, 5, None, 1e-7, o[k], ws, ws.numel(), dr.DR_NS_G_F32, stream=st)
    torch.cuda.synchronize()
    assert dr.dr_device_status()[0] == 0
    for ref, o in zip(refs, outs):
        assert all(torch.equal(ref, t) for t in o)
