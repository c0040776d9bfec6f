"""The layer norm takes its vector kernels wherever rows lie alike in vectors of 16 bytes: the same bits as rows that lie densely."""
import pytest

import dr_synth as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dr():
    import paper_1708_04728_b200 as dr
    return dr


def dev(a, f32):
    import torch
    t = torch.from_numpy(a).float().cuda()
    return t if f32 else t.to(torch.bfloat16)


def at(dense, off, ld):
    """A copy of `dense`, its rows `ld` apart from element `off` on."""
    import torch
    t = torch.full((off + dense.shape[0] * ld,), 5.0, dtype=dense.dtype, device="cuda")
    v = t[off:].view(dense.shape[0], ld)[:, :dense.shape[1]]
    v.copy_(dense)
    return v


@pytest.mark.parametrize("xf32,yf32", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("M,C,whole", [(700, 200, True), (9001, 36, True), (300, 1004, True), (61, 4100, True), (33, 8192, True), (700, 333, False), (9001, 61, False), (40, 6001, False)])
def test_float32_rows_four_elements_apart(dr, M, C, whole, xf32, yf32):
    """Vectors are 4 elements where a tensor is float32: tensors 4 elements apart, in place or in pitch, lie alike.  `whole`: rows of whole
    vectors against dense ones; otherwise rows one element off a boundary against the same with all tensors at one place."""
    import torch
    x, dy = (dev(S.normal(0, f"{n}{M}.{C}", (M, C)), f) for n, f in (("ax", xf32), ("ady", yf32)))
    g, b = dev(1 + 0.2 * S.normal(0, f"ag{C}", (C,)), True), dev(S.normal(0, f"ab{C}", (C,)), True)
    flags = dr.DR_LN_X_F32 * xf32 | dr.DR_LN_Y_F32 * yf32
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
    ld, off = (C, 0) if whole else (C + 2, 1)
    results = []
    for ox, px, oy, py in ((0, 0, 0, 0), (4, 4, 0, 0), (0, 0, 4, 4), (4, 0, 8, 4)):
        xv, dyv = at(x, off + ox, ld + px), at(dy, off + oy, ld + py)
        y, dx = at(torch.zeros_like(dy), off + oy, ld + py), at(torch.zeros_like(x), off + ox, ld + px)
        mean, rstd, dg, db = (torch.empty(n, device="cuda") for n in (M, M, C, C))
        dr.dr_layernorm(M, C, xv, ld + px, g, b, 1e-5, y, ld + py, mean, rstd, flags)
        dr.dr_layernorm_bwd(M, C, dyv, ld + py, xv, ld + px, g, mean, rstd, dx, ld + px, dg, db, ws, ws.numel(), flags)
        results.append([t.clone() for t in (y, mean, rstd, dx, dg, db)])
    for r in results[1:]:
        for name, a, e in zip(("y", "mean", "rstd", "dx", "dgamma", "dbeta"), r, results[0]):
            assert torch.equal(a, e), name


@pytest.mark.parametrize("yf32", [True, False])
@pytest.mark.parametrize("C,pad", [(3, 0), (20, 0), (100, 0), (333, 0), (333, 1), (513, 0), (1000, 0), (1030, 3), (3001, 2), (6000, 0), (8191, 0), (9000, 0)])
def test_backward_of_a_constant_row_far_from_zero(dr, C, pad, yf32):
    """x = mean throughout and 1/sqrt(eps) = 1e6: xhat is zero, though mean / sqrt(eps) passes float32's range; dx is that of the centred gradient."""
    import torch
    M, eps = 5, 1e-12
    x = S.normal(0, f"cr{C}", (M, C)).astype("float32")
    x[1], x[3] = 1e33, -2e33
    dyt = dev(S.normal(0, f"crd{C}", (M, C)), yf32)
    g = dev(1 + 0.2 * S.normal(0, f"crg{C}", (C,)), True)
    x64 = torch.from_numpy(x).cuda().double()
    mean = x64.mean(1).float()
    mean[1], mean[3] = 1e33, -2e33
    rstd = (1 / (((x64 - mean.double()[:, None]) ** 2).mean(1) + eps).sqrt()).float()
    xv, dx = at(dev(x, True), 0, C + pad), torch.empty((M, C), device="cuda")
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
    dr.dr_layernorm_bwd(M, C, dyt, 0, xv, C + pad, g, mean, rstd, dx, 0, dg, db, ws, ws.numel(), dr.DR_LN_X_F32 | dr.DR_LN_Y_F32 * yf32)
    h = (xv.double() - mean.double()[:, None]) * rstd.double()[:, None]
    t = dyt.double() * g.double()
    ref = rstd.double()[:, None] * (t - t.mean(1, keepdim=True) - h * (t * h).mean(1, keepdim=True))
    # 64 rounding errors of 2^-24 on the sizes of the summands, as everywhere for these sums
    tol = 64 * 2.0 ** -24 * rstd.double()[:, None] * (t.abs() + t.abs().mean(1, keepdim=True) + h.abs() * (t * h).abs().mean(1, keepdim=True))
    assert bool(((dx.double() - ref).abs() <= tol).all())
    assert bool(((dg.double() - (dyt.double() * h).sum(0)).abs() <= 64 * 2.0 ** -24 * (dyt.double() * h).abs().sum(0)).all())
    assert bool(((db.double() - dyt.double().sum(0)).abs() <= 64 * 2.0 ** -24 * dyt.double().abs().sum(0)).all())


def test_one_row_of_the_most_channels(dr):
    """Two to the 31st less one: positions in the row and the stride behind them pass 31 bits."""
    import torch
    C = 2 ** 31 - 1
    x = torch.tensor([1.0, -1.0], dtype=torch.bfloat16, device="cuda").repeat(2 ** 30)[:C]
    y, mean, rstd = torch.empty_like(x), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    dr.dr_layernorm(1, C, x, 0, None, None, 0.0, y, 0, mean, rstd)
    # mean 1 / C, variance 1; a thread's sums are whole numbers below 2^24, their join is rounded as every mean here: 64 errors of 2^-24 of mean |x|
    assert torch.equal(y, x)
    assert abs(float(mean) - 1 / C) <= 64 * 2.0 ** -24 and abs(float(rstd) - 1) <= 64 * 2.0 ** -24


def test_weight_gradients_of_a_row_of_2_to_the_30_channels(dr):
    import torch
    C = 2 ** 30
    pattern = lambda *v: torch.tensor(v, dtype=torch.bfloat16, device="cuda").repeat(C // 4)
    x, dy = pattern(1.0, -1.0, 1.0, -1.0), pattern(1.0, 2.0, 3.0, 4.0)
    dx, dg, db = torch.empty_like(x), torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(1, C), dtype=torch.uint8, device="cuda")
    dr.dr_layernorm_bwd(1, C, dy, 0, x, 0, None, torch.zeros(1, device="cuda"), torch.ones(1, device="cuda"), dx, 0, dg, db, ws, ws.numel())
    # mean of dy 2.5, of dy xhat -0.5: dx = dy - 2.5 + 0.5 x
    assert torch.equal(dx, pattern(-1.0, -1.0, 1.0, 1.0))
    assert torch.equal(db, dy.float()) and torch.equal(dg, dy.float() * x.float())
