"""GPU parity of the dropout against its definition: masks equal bit for bit, values within their rounding, at the sizes,
types, strides and values where it can go wrong."""
import numpy as np
import pytest

import dr_synth as S
import oracle.adapter as A

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8
SIZES = [(1, 1), (1, 7), (1, 8), (3, 5), (2, 9), (5, 16), (7, 24), (3, 33), (64, 31), (33, 40), (32, 1024), (9, 1000), (17, 333), (130, 257), (1000, 3), (4099, 1),
         (700, 520), (2, 9216), (3, 9217), (2049, 264)]


@pytest.fixture(scope="module")
def dr():
    import paper_1708_04728_b200 as dr
    return dr


def dev(a, f32, ld=0, shift=0):
    """A device tensor holding `a` in rows `ld` elements apart, its first element `shift` elements behind an aligned address."""
    import torch
    rows, C = a.shape
    ld = ld or C
    buf = torch.full((shift + rows * ld + 64,), 1e4, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    v = torch.as_strided(buf, (rows, C), (ld, 1), shift)
    v.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)))
    return buf, v


def run(dr, x, res, p, seed, offset, xf, yf, ldx=0, ldr=0, ldy=0, sx=0, sr=0, sy=0, step=None):
    rows, C = x.shape
    _, xt = dev(x, xf, ldx, sx)
    rt = dev(res, yf, ldr, sr)[1] if res is not None else None
    ybuf, yt = dev(np.full((rows, C), -77.0), yf, ldy, sy)
    dr.dr_dropout(rows, C, xt, ldx, rt, ldr, yt, ldy, p, seed, offset, step, dr.DR_DROP_X_F32 * xf | dr.DR_DROP_Y_F32 * yf)
    got = yt.double().cpu().numpy()
    # what lies between and around the rows is as it was
    yt.fill_(1e4)
    assert bool((ybuf == (1e4 if yf else ybuf.new_tensor(1e4))).all())
    return got


def check(got, x, res, p, seed, offset, yf):
    x = x.astype(np.float64)
    ref = A.dropout(x, None if res is None else res.astype(np.float64), p, seed, offset)
    kept = A.keep_mask(*x.shape, p, seed, offset)
    if res is None:
        assert np.array_equal(got != 0, kept & (x != 0)), "another mask"
    # 1 / (1 - p) in float32, the product, the sum with the residual: a rounding each, then that of the output
    part = np.abs(x) * kept / max(1 - A.threshold(p) / 65536, 2.0 ** -17)
    tol = 3 * U32 * (part + (0 if res is None else np.abs(res))) + (0 if yf else U16 * np.abs(ref))
    assert np.all(np.abs(got - ref) <= tol), np.max(np.abs(got - ref) - tol)


def values(name, M, C):
    return S.round_bf16(S.normal(0, name, (M, C)).astype(np.float32))


@pytest.mark.parametrize("xf,yf", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("M,C", SIZES)
def test_dense(dr, M, C, xf, yf):
    x, res = values(f"d{M}.{C}", M, C), values(f"r{M}.{C}", M, C)
    for p, r in ((0.4, None), (0.1, res)):
        check(run(dr, x, r, p, 1234567890123, 5, xf, yf), x, r, p, 1234567890123, 5, yf)


@pytest.mark.parametrize("xf,yf", [(False, False), (True, True), (True, False)])
@pytest.mark.parametrize("M,C,ldx,ldr,ldy,sx,sr,sy", [
    (37, 40, 48, 56, 64, 0, 0, 0), (37, 40, 48, 40, 64, 8, 16, 24), (37, 40, 41, 43, 47, 0, 0, 0), (37, 40, 40, 40, 40, 1, 0, 0), (37, 40, 40, 40, 40, 0, 1, 3),
    (21, 333, 501, 333, 340, 168, 0, 0), (21, 333, 333, 333, 333, 3, 5, 7), (50, 7, 9, 7, 8, 0, 2, 1), (300, 264, 300, 264, 264, 4, 4, 4), (5, 1030, 1032, 1031, 1030, 0, 0, 0)])
def test_strides_and_alignment(dr, M, C, ldx, ldr, ldy, sx, sr, sy, xf, yf):
    x, res = values(f"s{M}.{C}", M, C), values(f"t{M}.{C}", M, C)
    for r in (None, res):
        check(run(dr, x, r, 0.25, 99, 1 << 40, xf, yf, ldx, ldr, ldy, sx, sr, sy), x, r, 0.25, 99, 1 << 40, yf)


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.5, 0.999, 0.999999, 1.0])
def test_probabilities(dr, p):
    x = values("p", 40, 104)
    check(run(dr, x, None, p, 7, 0, False, True), x, None, p, 7, 0, True)
    check(run(dr, x, x, p, 7, 0, True, False), x, x, p, 7, 0, False)


def test_dropped_elements_are_zero_whatever_they_hold(dr):
    x = values("nan", 16, 64)
    x[::2, ::3] = np.nan
    x[1::2, ::5] = np.inf
    got = run(dr, x, None, 0.5, 3, 3, False, False)
    kept = A.keep_mask(16, 64, 0.5, 3, 3)
    assert np.all(got[~kept] == 0)
    assert np.array_equal(np.isnan(got), np.isnan(x) & kept) and np.array_equal(np.isinf(got), np.isinf(x) & kept)


@pytest.mark.parametrize("xf", [False, True])
@pytest.mark.parametrize("C", [64, 51])
def test_in_place_and_backward_draw_the_same_mask(dr, xf, C):
    import torch
    t = torch.float32 if xf else torch.bfloat16
    flags = (dr.DR_DROP_X_F32 | dr.DR_DROP_Y_F32) if xf else 0
    x = torch.randn(300, C, device="cuda").to(t)
    y = torch.empty_like(x)
    dr.dr_dropout(300, C, x, 0, None, 0, y, 0, 0.3, 11, 12, None, flags)
    z = x.clone()
    dr.dr_dropout(300, C, z, 0, None, 0, z, 0, 0.3, 11, 12, None, flags)
    assert torch.equal(y, z)
    r = torch.randn(300, C, device="cuda").to(t)
    s, w = r.clone(), torch.empty_like(r)
    dr.dr_dropout(300, C, x, 0, r, 0, w, 0, 0.3, 11, 12, None, flags)
    dr.dr_dropout(300, C, x, 0, s, 0, s, 0, 0.3, 11, 12, None, flags)       # y is the residual itself
    assert torch.equal(s, w)
    # the gradient of sum(dy * y) by x is dy where x was kept: a difference in one element moves it by 1 / (1 - p) or nothing
    dy = torch.ones_like(x)
    dx = torch.empty_like(x)
    dr.dr_dropout(300, C, dy, 0, None, 0, dx, 0, 0.3, 11, 12, None, flags)
    assert torch.equal(dx != 0, (y != 0) | ((x == 0) & (dx != 0)))


def test_far_rows(dr):
    """Elements, and element numbers, beyond 2^32: the last rows of a tensor of 4.4e9 elements against the definition."""
    import torch
    M, C = 539000, 8200
    x = torch.empty((M, C), dtype=torch.bfloat16, device="cuda")
    x[:2].fill_(1.0)
    x[-3:].fill_(1.0)
    dr.dr_dropout(M, C, x, 0, None, 0, x, 0, 0.5, 21, 22, None, 0)
    for first, rows in ((0, 2), (M - 3, 3)):
        kept = A.keep_mask(rows, C, 0.5, 21, 22, first=first * C)
        assert np.array_equal(x[first:first + rows].double().cpu().numpy(), 2.0 * kept)


def test_captured_call_follows_the_counter(dr):
    import torch
    x = torch.ones((64, 200), dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        dr.dr_dropout(64, 200, x, 0, None, 0, y, 0, 0.5, 1, 10, step)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dr.dr_dropout(64, 200, x, 0, None, 0, y, 0, 0.5, 1, 10, step)
        step += 1
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(y.double().cpu().numpy(), 2.0 * A.keep_mask(64, 200, 0.5, 1, 10 + i))
    step.fill_(-4)                       # the sum of both is taken modulo 2^64
    g.replay()
    torch.cuda.synchronize()
    assert np.array_equal(y.double().cpu().numpy(), 2.0 * A.keep_mask(64, 200, 0.5, 1, 6))
