"""GPU parity of layer normalisation, forward and backward, against its formulas in float64, at the sizes, types,
strides and values where it can go wrong."""
import numpy as np
import pytest

import dr_synth as S

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8          # half a unit in the last place, relative: 24 and 8 significant bits
# Sums of C float32 terms: a lane adds at most 32 in a row and lanes are joined pairwise or in a few steps; 64 rounding
# errors bound both, the statistics' own and those of the element-wise chain behind them.
SUM = 64 * U32


@pytest.fixture(scope="module")
def dr():
    import paper_1708_04728_b200 as dr
    return dr


def dev(a, f32):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
    return t if f32 else t.to(torch.bfloat16)


def host(t):
    return t.double().cpu().numpy()


def empty(shape, f32):
    import torch
    return torch.full(shape, float("nan"), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")


def rows(name, M, C, offset=1.0):
    x = S.normal(0, name, (M, C)) * (0.2 + 3 * S.uniform(0, name + "s", (C,), 0.0, 1.0)) + offset * S.normal(0, name + "o", (C,))
    return S.round_bf16(x.astype(np.float32))


def forward(x, g, b, eps):
    x = x.astype(np.float64)
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    return (x - mean) * rstd * g + b, mean[:, 0], rstd[:, 0]


def backward(dy, x, g, mean, rstd):
    h = (x - mean[:, None]) * rstd[:, None]
    t = dy * g
    dx = rstd[:, None] * (t - t.mean(1, keepdims=True) - h * (t * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def check_forward(got, x, g, b, eps, yf32):
    y, mean, rstd = forward(x, g, b, eps)
    spread = (np.abs(x).mean(1) * rstd)[:, None]                 # how many deviations the row lies from zero
    tol = SUM * (1 + spread) * (np.abs(g) * (1 + np.abs((y - b) / np.where(g == 0, 1, g))) + np.abs(b)) + (U32 if yf32 else U16) * np.abs(y)
    assert np.all(np.abs(got[0] - y) <= tol), np.max(np.abs(got[0] - y) / tol)
    assert np.all(np.abs(got[1] - mean) <= SUM * np.abs(x).mean(1) + 1e-30)
    assert np.all(np.abs(got[2] - rstd) <= SUM * (1 + spread[:, 0]) * rstd)


SIZES = [(1, 1), (3, 1), (1, 8), (5, 7), (2, 8), (33, 24), (9, 64), (17, 65), (300, 96), (64, 128), (50, 147), (129, 192), (1000, 256),
         (31, 257), (40, 333), (25, 512), (11, 513), (13, 520), (49, 1024), (20, 1031), (7, 2048), (6, 4096), (5, 5000), (3, 8192), (4, 8193),
         (2, 16384), (2, 16400), (2, 20001), (2, 33000), (4097, 40)]


@pytest.mark.parametrize("xf32,yf32", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("M,C", SIZES)
def test_forward(dr, M, C, xf32, yf32):
    x = rows(f"ln{M}.{C}", M, C)
    g, b = 1 + 0.2 * S.normal(0, f"g{C}", (C,)), 0.3 * S.normal(0, f"b{C}", (C,))
    y, mean, rstd = empty((M, C), yf32), empty((M,), True), empty((M,), True)
    flags = dr.DR_LN_X_F32 * xf32 | dr.DR_LN_Y_F32 * yf32
    dr.dr_layernorm(M, C, dev(x, xf32), 0, dev(g, True), dev(b, True), 1e-5, y, 0, mean, rstd, flags)
    check_forward((host(y), host(mean), host(rstd)), x, g.astype(np.float64), b.astype(np.float64), 1e-5, yf32)


@pytest.mark.parametrize("xf32,yf32", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("M,C", SIZES)
def test_backward(dr, M, C, xf32, yf32):
    import torch
    x, dy = rows(f"lnb{M}.{C}", M, C), S.round_bf16(S.normal(0, f"dy{M}.{C}", (M, C)))
    g = 1 + 0.2 * S.normal(0, f"g{C}", (C,))
    _, mean, rstd = forward(x, 1, 0, 1e-5)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    dx, dg, db = empty((M, C), xf32), empty((C,), True), empty((C,), True)
    ws = torch.full((dr.dr_layernorm_bwd_workspace_bytes(M, C),), 0xFF, dtype=torch.uint8, device="cuda")
    flags = dr.DR_LN_X_F32 * xf32 | dr.DR_LN_Y_F32 * yf32
    args = (M, C, dev(dy, yf32), 0, dev(x, xf32), 0, dev(g, True), dev(mean, True), dev(rstd, True))
    dr.dr_layernorm_bwd(*args, dx, 0, dg, db, ws, ws.numel(), flags)
    m64, r64 = mean.astype(np.float64), rstd.astype(np.float64)
    rdx, rdg, rdb = backward(dy.astype(np.float64), x.astype(np.float64), g.astype(np.float64), m64, r64)
    h = np.abs((x - m64[:, None]) * r64[:, None])
    t = np.abs(dy * g)
    parts = r64[:, None] * (t + t.mean(1, keepdims=True) + h * (t * h).mean(1, keepdims=True))     # sizes of the summands
    tol = SUM * parts + (U32 if xf32 else U16) * np.abs(rdx)
    assert np.all(np.abs(host(dx) - rdx) <= tol), np.max(np.abs(host(dx) - rdx) / (tol + 1e-300))
    # a sum over M rows: at most M rounding errors, and far fewer as rows are summed in ranges
    rsum = (32 + min(M, 512)) * U32
    assert np.all(np.abs(host(dg) - rdg) <= rsum * (np.abs(dy) * h).sum(0) + 1e-30)
    assert np.all(np.abs(host(db) - rdb) <= rsum * np.abs(dy).sum(0) + 1e-30)
    dx2, dg2, db2 = empty((M, C), xf32), empty((C,), True), empty((C,), True)
    ws.fill_(0x55)
    dr.dr_layernorm_bwd(*args, dx2, 0, dg2, db2, ws, ws.numel(), flags)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2) and torch.equal(db, db2), "not the same on a second run"


def test_many_rows(dr):
    """More rows than one round of the grid holds, forward and backward; a sample of rows against the formula, the sums in full."""
    import torch
    M, C = 60001, 72
    x, dy = rows("many", M, C), S.round_bf16(S.normal(0, "many.dy", (M, C)))
    g, b = 1 + 0.2 * S.normal(0, "many.g", (C,)), 0.3 * S.normal(0, "many.b", (C,))
    y, mean, rstd = empty((M, C), False), empty((M,), True), empty((M,), True)
    xd, gd = dev(x, False), dev(g, True)
    dr.dr_layernorm(M, C, xd, 0, gd, dev(b, True), 1e-5, y, 0, mean, rstd)
    check_forward((host(y), host(mean), host(rstd)), x, g.astype(np.float64), b.astype(np.float64), 1e-5, False)
    dx, dg, db = empty((M, C), False), empty((C,), True), empty((C,), True)
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
    dr.dr_layernorm_bwd(M, C, dev(dy, False), 0, xd, 0, gd, mean, rstd, dx, 0, dg, db, ws, ws.numel())
    rdx, rdg, rdb = backward(dy.astype(np.float64), x.astype(np.float64), g.astype(np.float64), host(mean), host(rstd))
    h = np.abs((x - host(mean)[:, None]) * host(rstd)[:, None])
    t = np.abs(dy * g)
    parts = host(rstd)[:, None] * (t + t.mean(1, keepdims=True) + h * (t * h).mean(1, keepdims=True))
    assert np.all(np.abs(host(dx) - rdx) <= SUM * parts + U16 * np.abs(rdx))
    assert np.all(np.abs(host(dg) - rdg) <= 544 * U32 * (np.abs(dy) * h).sum(0))
    assert np.all(np.abs(host(db) - rdb) <= 544 * U32 * np.abs(dy).sum(0))


@pytest.mark.parametrize("M,C,pad,off", [(37, 96, 32, 8), (37, 96, 31, 3), (21, 333, 5, 1), (9, 2048, 64, 16), (9, 2050, 3, 2), (130, 64, 64, 64)])
def test_channel_slices_are_kept_apart(dr, M, C, pad, off):
    """Rows of a wider tensor, at offsets that are 16-byte aligned and not: the slice is written, its neighbours stay."""
    import torch
    wide = S.round_bf16(S.normal(0, f"sl{C}.{off}", (M, C + pad)))
    dyw = S.round_bf16(S.normal(0, f"sld{C}.{off}", (M, C + pad)))
    g, b = 1 + 0.2 * S.normal(0, f"g{C}", (C,)), 0.3 * S.normal(0, f"b{C}", (C,))
    off = min(off, pad)
    ld = C + pad
    xw, yw, dxw, dyd = dev(wide, False), empty((M, ld), False), empty((M, ld), False), dev(dyw, False)
    yw.fill_(7.0)
    dxw.fill_(7.0)
    mean, rstd = empty((M,), True), empty((M,), True)
    dr.dr_layernorm(M, C, xw[:, off:], ld, dev(g, True), dev(b, True), 1e-5, yw[:, off:], ld, mean, rstd)
    x = wide[:, off:off + C]
    check_forward((host(yw[:, off:off + C]), host(mean), host(rstd)), x, g.astype(np.float64), b.astype(np.float64), 1e-5, False)
    dg, db = empty((C,), True), empty((C,), True)
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
    dr.dr_layernorm_bwd(M, C, dyd[:, off:], ld, xw[:, off:], ld, dev(g, True), mean, rstd, dxw[:, off:], ld, dg, db, ws, ws.numel())
    rdx, rdg, _ = backward(dyw[:, off:off + C].astype(np.float64), x.astype(np.float64), g.astype(np.float64), host(mean), host(rstd))
    got = host(dxw[:, off:off + C])
    assert np.all(np.abs(got - rdx) <= 8 * SUM * np.abs(rdx).max() + U16 * np.abs(rdx))
    assert np.abs(host(dg) - rdg).max() <= 600 * U32 * np.abs(dyw).sum(0).max()
    for t in (yw, dxw):
        assert bool((t[:, :off] == 7).all()) and bool((t[:, off + C:] == 7).all()), "written outside the slice"


@pytest.mark.parametrize("xf32,yf32", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("M,C,ldx,ldy,offx,offy", [(50, 40, 41, 40, 0, 0), (9000, 65, 72, 67, 3, 2), (700, 200, 203, 201, 1, 0), (300, 600, 601, 603, 0, 2),
                                                   (500, 2000, 2003, 2000, 1, 0), (40, 4096, 4096, 4096, 0, 1), (20, 5001, 5003, 5001, 0, 0),
                                                   (9001, 61, 61, 61, 5, 5), (6000, 333, 341, 349, 2, 10), (2500, 1030, 1033, 1033, 7, 7)])
def test_rows_at_any_offset(dr, M, C, ldx, ldy, offx, offy, xf32, yf32):
    """Rows whose offset from a 16-byte boundary differs between the tensors, or changes from row to row, over several rounds."""
    import torch
    flags = dr.DR_LN_X_F32 * xf32 | dr.DR_LN_Y_F32 * yf32
    xa, dya = rows(f"ao{C}", M, C), S.round_bf16(S.normal(0, f"aod{C}", (M, C)))
    g, b = 1 + 0.2 * S.normal(0, f"g{C}", (C,)), 0.3 * S.normal(0, f"b{C}", (C,))

    def strided(a, ld, off, f32):
        t = torch.full((off + M * ld,), 9.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        v = t[off:].view(M, ld)[:, :C]
        if a is not None:
            v.copy_(dev(a, f32))
        return t, v

    (_, x), (_, dy), (yt, y), (dxt, dx) = strided(xa, ldx, offx, xf32), strided(dya, ldy, offy, yf32), strided(None, ldy, offy, yf32), strided(None, ldx, offx, xf32)
    mean, rstd = empty((M,), True), empty((M,), True)
    dr.dr_layernorm(M, C, x, ldx, dev(g, True), dev(b, True), 1e-5, y, ldy, mean, rstd, flags)
    check_forward((host(y), host(mean), host(rstd)), xa, g.astype(np.float64), b.astype(np.float64), 1e-5, yf32)
    dg, db = empty((C,), True), empty((C,), True)
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
    dr.dr_layernorm_bwd(M, C, dy, ldy, x, ldx, dev(g, True), mean, rstd, dx, ldx, dg, db, ws, ws.numel(), flags)
    m64, r64 = host(mean), host(rstd)
    rdx, rdg, rdb = backward(dya.astype(np.float64), xa.astype(np.float64), g.astype(np.float64), m64, r64)
    h = np.abs((xa - m64[:, None]) * r64[:, None])
    t = np.abs(dya * g)
    parts = r64[:, None] * (t + t.mean(1, keepdims=True) + h * (t * h).mean(1, keepdims=True))
    assert np.all(np.abs(host(dx) - rdx) <= SUM * parts + (U32 if xf32 else U16) * np.abs(rdx))
    assert np.all(np.abs(host(dg) - rdg) <= 544 * U32 * (np.abs(dya) * h).sum(0) + 1e-30)
    assert np.all(np.abs(host(db) - rdb) <= 544 * U32 * np.abs(dya).sum(0) + 1e-30)
    for whole, view, off, ld in ((yt, y, offy, ldy), (dxt, dx, offx, ldx)):
        view.fill_(9.0)
        assert bool((whole == 9).all()), "written outside the rows"


@pytest.mark.parametrize("xf32,yf32", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("C", [257, 264, 341, 384, 385, 520, 683, 768, 1030, 1365, 1536, 2056, 2730, 3001, 3080, 4104, 5461, 6144, 6150])
def test_rows_a_little_longer_than_a_team(dr, C, xf32, yf32):
    """Channel counts on both sides of every change of a thread's share, of dense rows and of rows inside wider ones."""
    import torch
    M = 203
    x = rows(f"t{C}", M, C)
    g, b = 1 + 0.2 * S.normal(0, f"g{C}", (C,)), 0.3 * S.normal(0, f"b{C}", (C,))
    for pad in (0, 16):
        xt, yt = empty((M, C + pad), xf32), empty((M, C + pad), yf32)
        xt[:, pad // 2:pad // 2 + C] = dev(x, xf32)
        yt.fill_(7.0)
        mean, rstd = empty((M,), True), empty((M,), True)
        dr.dr_layernorm(M, C, xt[:, pad // 2:], C + pad, dev(g, True), dev(b, True), 1e-5, yt[:, pad // 2:], C + pad, mean, rstd,
                        dr.DR_LN_X_F32 * xf32 | dr.DR_LN_Y_F32 * yf32)
        check_forward((host(yt[:, pad // 2:pad // 2 + C]), host(mean), host(rstd)), x, g.astype(np.float64), b.astype(np.float64), 1e-5, yf32)
        assert bool((yt[:, :pad // 2] == 7).all()) and bool((yt[:, pad // 2 + C:] == 7).all())


@pytest.mark.parametrize("C", [64, 100, 777, 1024, 4096])
def test_no_weights_no_statistics_in_place(dr, C):
    import torch
    M = 19
    x = rows(f"ip{C}", M, C)
    xd = dev(x, False)
    y = empty((M, C), False)
    dr.dr_layernorm(M, C, xd, 0, None, None, 1e-5, y, 0)
    ref = forward(x, 1, 0, 1e-5)[0]
    spread = (np.abs(x).mean(1) * forward(x, 1, 0, 1e-5)[2])[:, None]
    assert np.all(np.abs(host(y) - ref) <= SUM * (1 + spread) * (1 + np.abs(ref)) + U16 * np.abs(ref))
    only_g, only_b = empty((M, C), False), empty((M, C), False)
    g, b = 1 + 0.2 * S.normal(0, f"g{C}", (C,)), 0.3 * S.normal(0, f"b{C}", (C,))
    dr.dr_layernorm(M, C, xd, 0, dev(g, True), None, 1e-5, only_g, 0)
    dr.dr_layernorm(M, C, xd, 0, None, dev(b, True), 1e-5, only_b, 0)
    assert np.all(np.abs(host(only_g) - ref * g) <= SUM * (1 + spread) * (1 + np.abs(ref)) * np.abs(g) + U16 * np.abs(ref * g))
    assert np.all(np.abs(host(only_b) - ref - b) <= SUM * (1 + spread) * (1 + np.abs(ref) + np.abs(b)) + U16 * np.abs(ref + b))
    dr.dr_layernorm(M, C, xd, 0, None, None, 1e-5, xd, 0)                       # y is x
    assert torch.equal(xd, y)
    # backward: no weight gradients, no workspace; dx is dy, then dx is x
    mean, rstd = (dev(t, True) for t in forward(x, 1, 0, 1e-5)[1:])
    dyd = dev(S.round_bf16(S.normal(0, f"ipd{C}", (M, C))), False)
    out = empty((M, C), False)
    dr.dr_layernorm_bwd(M, C, dyd, 0, dev(x, False), 0, dev(g, True), mean, rstd, out, 0, None, None, None, 0)
    a, b2 = dyd.clone(), dev(x, False)
    dr.dr_layernorm_bwd(M, C, a, 0, dev(x, False), 0, dev(g, True), mean, rstd, a, 0, None, None, None, 0)
    dr.dr_layernorm_bwd(M, C, dyd, 0, b2, 0, dev(g, True), mean, rstd, b2, 0, None, None, None, 0)
    assert torch.equal(a, out) and torch.equal(b2, out)
    # one of the two gradients alone is the one of the pair
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
    both, alone = (empty((C,), True), empty((C,), True)), (empty((C,), True), empty((C,), True))
    for dg, db in (both, (alone[0], None), (None, alone[1])):
        dr.dr_layernorm_bwd(M, C, dyd, 0, dev(x, False), 0, dev(g, True), mean, rstd, out, 0, dg, db, ws, ws.numel())
    assert torch.equal(both[0], alone[0]) and torch.equal(both[1], alone[1])


@pytest.mark.parametrize("C", [8, 33, 256, 1024, 3000])
def test_constant_infinite_and_nan_rows(dr, C):
    """A constant row has variance zero: y = beta, rstd = 1/sqrt(eps).  NaN and infinities stay in their row."""
    x = rows(f"sp{C}", 6, C)
    x[1] = 3.0
    x[2, C // 2] = np.nan
    x[3, C - 1] = np.inf
    x[4, 0] = -np.inf
    g, b = 1 + 0.2 * S.normal(0, f"g{C}", (C,)), 0.3 * S.normal(0, f"b{C}", (C,))
    y, mean, rstd = empty((6, C), True), empty((6,), True), empty((6,), True)
    dr.dr_layernorm(6, C, dev(x, True), 0, dev(g, True), dev(b, True), 1e-5, y, 0, mean, rstd, dr.DR_LN_X_F32 | dr.DR_LN_Y_F32)
    ok = [0, 1, 5]
    got = host(y), host(mean), host(rstd)
    assert np.all(np.isnan(got[0][2:5])) and np.all(np.isfinite(got[0][ok]))
    ref = forward(x[ok], g.astype(np.float64), b.astype(np.float64), 1e-5)
    # the mean of equal values may be off by a rounding error, which 1/sqrt(eps) = 316 magnifies
    assert np.all(np.abs(got[0][1] - b) <= 317 * SUM * 3 * np.abs(g) + U32 * np.abs(b))
    assert abs(got[2][1] * np.sqrt(1e-5) - 1) <= 1e-3
    assert np.abs(got[0][0] - ref[0][0]).max() <= 1e-4 and np.abs(got[0][5] - ref[0][2]).max() <= 1e-4


@pytest.mark.parametrize("C", [24, 520])
def test_gradients_against_differences(dr, C):
    """L = sum(y * r): dL/dx, dL/dgamma, dL/dbeta of the backward kernel against central differences of the forward kernel."""
    import torch
    M, f = 5, dr.DR_LN_X_F32 | dr.DR_LN_Y_F32
    x, r = rows(f"df{C}", M, C), S.normal(0, f"dr{C}", (M, C))
    g, b = 1 + 0.2 * S.normal(0, f"g{C}", (C,)), 0.3 * S.normal(0, f"b{C}", (C,))

    def loss(x, g, b):
        y = empty((M, C), True)
        dr.dr_layernorm(M, C, dev(x, True), 0, dev(g, True), dev(b, True), 1e-5, y, 0, None, None, f)
        return (host(y) * r).sum()

    y, mean, rstd = empty((M, C), True), empty((M,), True), empty((M,), True)
    dr.dr_layernorm(M, C, dev(x, True), 0, dev(g, True), dev(b, True), 1e-5, y, 0, mean, rstd, f)
    dx, dg, db = empty((M, C), True), empty((C,), True), empty((C,), True)
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
    dr.dr_layernorm_bwd(M, C, dev(r, True), 0, dev(x, True), 0, dev(g, True), mean, rstd, dx, 0, dg, db, ws, ws.numel(), f)
    dx, dg, db = host(dx), host(dg), host(db)
    h = 2.0 ** -6
    # truncation: h^2 rstd^2 times the size of a gradient (third derivative / 6); rounding: the sum's 64 U32 per unit of y, over h
    scale = np.abs(dx).max()
    tol = 4 * (h * host(rstd).max()) ** 2 * scale + SUM * np.abs(host(y) * r).sum() / h / np.sqrt(M * C)
    for i, c in ((0, 0), (1, C // 2), (4, C - 1), (2, 7)):
        e = np.zeros_like(x)
        e[i, c] = h
        assert abs((loss(x + e, g, b) - loss(x - e, g, b)) / (2 * h) - dx[i, c]) <= tol
    for c in (0, C // 3, C - 1):
        e = np.zeros_like(g)
        e[c] = h
        for d, ref in (((loss(x, g + e, b) - loss(x, g - e, b)), dg), ((loss(x, g, b + e) - loss(x, g, b - e)), db)):
            assert abs(d / (2 * h) - ref[c]) <= SUM * np.abs(host(y) * r).sum() / h / np.sqrt(M * C) + 1e-5 * np.abs(ref).max()


def test_empty_and_other_stream(dr):
    import torch
    C = 40
    g = torch.ones(C, device="cuda")
    x = dev(rows("st", 5, C), False)
    y, dg, db = empty((5, C), False), empty((C,), True), empty((C,), True)
    n0 = dr.dr_launch_count()
    dr.dr_layernorm(0, C, x, 0, g, g, 1e-5, y, 0)
    assert dr.dr_launch_count() == n0 and bool(torch.isnan(y).all())
    ws = torch.empty(max(256, dr.dr_layernorm_bwd_workspace_bytes(0, C)), dtype=torch.uint8, device="cuda")
    dr.dr_layernorm_bwd(0, C, x, 0, x, 0, g, dg, db, y, 0, dg, db, ws, ws.numel())
    assert bool((dg == 0).all()) and bool((db == 0).all()) and bool(torch.isnan(y).all())
    # a stream that has to wait for its input: the call is ordered on the stream it is given
    big = torch.randn(4096, 4096, device="cuda")
    ref = empty((5, C), False)
    dr.dr_layernorm(5, C, x, 0, g, g, 1e-5, ref, 0)
    torch.cuda.synchronize()
    side, late = torch.cuda.Stream(), torch.zeros_like(x)
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-4
        late.copy_(x)
    dr.dr_layernorm(5, C, late, 0, g, g, 1e-5, y, 0, stream=side)
    side.synchronize()
    assert torch.equal(y, ref)


def test_graph_capture(dr):
    import torch
    M, C = 300, 256
    x = dev(rows("gc", M, C), False)
    g, b = torch.rand(C, device="cuda") + 0.5, torch.rand(C, device="cuda")
    y, mean, rstd = empty((M, C), False), empty((M,), True), empty((M,), True)
    dx, dg, db = empty((M, C), False), empty((C,), True), empty((C,), True)
    ws = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")

    def step():
        dr.dr_layernorm(M, C, x, 0, g, b, 1e-5, y, 0, mean, rstd)
        dr.dr_layernorm_bwd(M, C, y, 0, x, 0, g, mean, rstd, dx, 0, dg, db, ws, ws.numel())

    step()
    ref = [t.clone() for t in (y, dx, dg, db)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, dx, dg, db):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, t) for a, t in zip(ref, (y, dx, dg, db)))
