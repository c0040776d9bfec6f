"""GPU parity of the low-rank adapters beside a shared layer, forward and backward, against their formulas in float64."""
import numpy as np
import pytest

import dr_synth as S
import oracle.adapter as A

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8          # half a unit in the last place, relative
SPLIT = 2.0 ** -16                        # t and u as two bfloat16 values: 2^-8 of 2^-9 is left out


def SUM(n):
    """A float32 sum of n products of bfloat16 values, relative to the sum of their sizes: n roundings at most, a few for the factors."""
    return (n + 64) * U32


@pytest.fixture(scope="module")
def dr():
    import paper_1708_04728_b200 as dr
    return dr


def requests(kind, M, adapters, seed=0):
    """Row offsets and variants of the requests."""
    rng = np.random.default_rng(seed + 31 * M + adapters)
    if kind == "one":
        return [0, M], [adapters - 1]
    if kind == "rows":                                      # single tokens, each of its own request
        return list(range(M + 1)), rng.integers(0, adapters, M).tolist()
    if kind == "none":
        return [0, M // 2, M], [-1, adapters]               # no variant; a number behind the last one
    if kind == "even":
        n = max(1, min(M, 2 * adapters))
        return [M * i // n for i in range(n + 1)], (np.arange(n) % adapters).tolist()
    if kind == "inner":                                     # rows in front of the first and behind the last request
        return [M // 5, M // 2, M // 2, M - M // 4], [0, adapters - 1, adapters // 2]
    n = max(2, min(M, 23))                                  # "ragged": empty requests, some without a variant, variants that come back
    cuts = np.sort(np.concatenate([[0, M - M // 9], rng.integers(0, M - M // 9 + 1, n - 1)]))
    ids = rng.integers(0, adapters, n)
    ids[rng.random(n) < 0.2] = -1
    return cuts.tolist(), ids.tolist()


class Case:
    def __init__(self, M, K, N, R, adapters, kind="ragged", seed=0):
        name = f"{M}.{K}.{N}.{R}.{adapters}.{kind}.{seed}"
        bf = lambda tag, shape, s=1.0: S.round_bf16((s * S.normal(0, name + tag, shape)).astype(np.float32)).astype(np.float64)
        self.M, self.K, self.N, self.R, self.adapters = M, K, N, R, adapters
        self.x, self.w = np.maximum(bf("x", (M, K)), 0) + bf("xo", (1, K), 0.25), bf("w", (N, K), (2 / K) ** 0.5)
        self.x = S.round_bf16(self.x.astype(np.float32)).astype(np.float64)
        self.a, self.b = bf("a", (adapters, R, K), K ** -0.5), bf("b", (adapters, N, R), R ** -0.5)
        self.bias = S.normal(0, name + "bias", (N,)).astype(np.float32).astype(np.float64)
        self.scale = S.uniform(0, name + "s", (adapters,), 0.5, 2.0).astype(np.float32).astype(np.float64)
        self.dy = bf("dy", (M, N))
        self.row_start, self.ids = requests(kind, M, adapters, seed)


def dev(a, dtype, ld=0):
    """(buffer, view): rows `ld` elements apart, 16-byte aligned."""
    import torch
    rows, C = a.shape
    ld = ld or C
    buf = torch.full((rows * ld + 64,), 1e4, dtype=dtype, device="cuda")
    v = torch.as_strided(buf, (rows, C), (ld, 1), 0)
    v.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float64)))
    return buf, v


def flat(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float64)).cuda().to(dtype).contiguous()


def ints(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def scratch(n):
    import torch
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")         # NaN wherever something is read before it is written


MARK = -768.0


def untouched(buf, view, rows_inside):
    """Rows of no request and what lies between the rows hold what they held."""
    v = view.clone()
    outside = np.ones(view.shape[0], bool)
    outside[rows_inside] = False
    assert bool((v[outside.nonzero()[0]] == MARK).all())
    view.fill_(1e4)
    assert bool((buf == buf.new_tensor(1e4)).all())
    return v.double().cpu().numpy()


def forward(dr, c, p=0.0, relu=False, bias=True, f32=False, scale=True, ldx=0, ldy=0, seed=77, offset=5, step=None, keep_t=True):
    import torch
    bf, ff = torch.bfloat16, torch.float32
    xb, x = dev(c.x, bf, ldx)
    yb, y = dev(np.full((c.M, c.N), MARK), ff if f32 else bf, ldy)
    tb, t = dev(np.full((c.M, c.R), MARK), ff)
    d = dr.dr_adapter_desc(Cin=c.K, Cout=c.N, rank=c.R, adapters=c.adapters, drop_p=p, drop_seed=seed, drop_offset=offset,
                           flags=dr.DR_BIAS * bias | dr.DR_RELU * relu | dr.DR_OUT_F32 * f32)
    ws = scratch(dr.dr_adapter_workspace_bytes(d, c.M, ldx))
    args = (flat(c.w, bf), flat(c.bias, ff) if bias else None, flat(c.a, bf), flat(c.b, bf), flat(c.scale, ff) if scale else None)
    dr.dr_adapter(d, c.M, x, ldx, *args, len(c.ids), ints(c.row_start), ints(c.ids), y, ldy, t if keep_t else None, step, ws, ws.numel())
    inside = slice(c.row_start[0], max(c.row_start[0], c.row_start[-1]))
    return untouched(yb, y, inside), untouched(tb, t, inside if keep_t else slice(0, 0)), inside


def check_forward(dr, c, p=0.0, relu=False, bias=True, f32=False, scale=True, seed=77, offset=5, **kw):
    gy, gt, inside = forward(dr, c, p, relu, bias, f32, scale, seed=seed, offset=offset, **kw)
    f = A.factors(c.M, c.K, p, seed, offset) if p else None
    s = c.scale if scale else None
    y, t = A.forward(c.x, c.w, c.bias if bias else None, c.a, c.b, s, c.row_start, c.ids, relu, f)
    size, tsize = A.forward(abs(c.x), abs(c.w), abs(c.bias) if bias else None, abs(c.a), abs(c.b), s, c.row_start, c.ids, False, f)
    main = abs(c.x) @ abs(c.w).T + (abs(c.bias) if bias else 0)
    tol = SUM(c.K) * size + (SUM(c.R) + SPLIT) * (size - main) + (U32 if f32 else U16) * abs(y)
    err = abs(gy - y)[inside]
    assert np.all(err <= tol[inside]), (np.max(err / tol[inside]), np.argmax(err / tol[inside]))
    if kw.get("keep_t", True):
        assert np.all(abs(gt - t)[inside] <= SUM(c.K) * tsize[inside])


def backward(dr, c, t, p=0.0, scale=True, ldx=0, lddy=0, lddx=0, seed=77, offset=5, want=(True, True, True), fill=0xFF):
    import torch
    bf, ff = torch.bfloat16, torch.float32
    xb, x = dev(c.x, bf, ldx)
    dyb, dy = dev(c.dy, bf, lddy)
    dxb, dx = dev(np.full((c.M, c.K), MARK), bf, lddx)
    d = dr.dr_adapter_desc(Cin=c.K, Cout=c.N, rank=c.R, adapters=c.adapters, flags=0, drop_p=p, drop_seed=seed, drop_offset=offset)
    ws = scratch(dr.dr_adapter_bwd_workspace_bytes(d, c.M, ldx, lddy))
    ws.fill_(fill)
    da = torch.full((c.adapters, c.R, c.K), float("nan"), device="cuda")
    db = torch.full((c.adapters, c.N, c.R), float("nan"), device="cuda")
    dr.dr_adapter_bwd(d, c.M, dy, lddy, x if want[1] else None, ldx, flat(c.w, bf), flat(c.a, bf), flat(c.b, bf), flat(c.scale, ff) if scale else None,
                      len(c.ids), ints(c.row_start), ints(c.ids), flat(t, ff) if want[2] else None, dx if want[0] else None, lddx, da if want[1] else None,
                      db if want[2] else None, None, ws, ws.numel())
    inside = slice(c.row_start[0], max(c.row_start[0], c.row_start[-1]))
    return untouched(dxb, dx, inside if want[0] else slice(0, 0)), da.double().cpu().numpy(), db.double().cpu().numpy(), inside


def check_backward(dr, c, p=0.0, scale=True, seed=77, offset=5, want=(True, True, True), **kw):
    f = A.factors(c.M, c.K, p, seed, offset) if p else None
    s = c.scale if scale else None
    t = np.nan_to_num(A.forward(c.x, c.w, None, c.a, c.b, s, c.row_start, c.ids, False, f)[1], nan=1e30).astype(np.float32).astype(np.float64)
    gdx, gda, gdb, inside = backward(dr, c, t, p, scale, seed=seed, offset=offset, want=want, **kw)
    dx, da, db = A.backward(c.dy, c.x, c.w, c.a, c.b, s, c.row_start, c.ids, t, f)
    adx, ada, adb = A.backward(abs(c.dy), abs(c.x), abs(c.w), abs(c.a), abs(c.b), s, c.row_start, c.ids, abs(t), f)
    if want[0]:
        main = abs(c.dy) @ abs(c.w)
        tol = SUM(c.N) * adx + (SUM(c.R) + SPLIT) * (adx - main) + U16 * abs(dx)
        err = abs(gdx - dx)[inside]
        assert np.all(err <= tol[inside]), np.max(err / tol[inside])
    if want[1]:
        assert np.all(abs(gda - da) <= (SUM(c.N) + SUM(c.M) + SPLIT) * ada), np.max(abs(gda - da) / (ada + 1e-300))
    if want[2]:
        assert np.all(abs(gdb - db) <= (SUM(c.M) + SPLIT) * adb), np.max(abs(gdb - db) / (adb + 1e-300))


SIZES = [  # rows, Cin, Cout, rank, variants
    (1, 1, 1, 1, 1), (1, 8, 8, 8, 1), (1, 1024, 1000, 8, 4), (2, 64, 40, 4, 2), (3, 7, 5, 3, 2), (8, 64, 64, 8, 3), (17, 72, 24, 5, 4), (31, 128, 256, 16, 31),
    (33, 200, 96, 12, 5), (49, 832, 384, 8, 1), (64, 1031, 333, 64, 3), (100, 56, 1000, 16, 7), (127, 96, 72, 256, 2), (128, 256, 128, 16, 9), (129, 264, 136, 33, 3),
    (200, 4096, 64, 8, 2), (256, 192, 96, 32, 6), (257, 147, 64, 5, 4), (300, 64, 520, 64, 3), (511, 128, 129, 24, 5), (640, 528, 160, 12, 9), (1000, 64, 256, 8, 64),
    (1025, 80, 48, 130, 2), (2049, 136, 272, 16, 3), (70, 9216, 72, 8, 2), (5000, 40, 24, 4, 3), (385, 512, 512, 64, 2)]


@pytest.mark.parametrize("kind", ["one", "ragged", "inner"])
@pytest.mark.parametrize("M,K,N,R,adapters", SIZES)
def test_forward(dr, M, K, N, R, adapters, kind):
    check_forward(dr, Case(M, K, N, R, adapters, kind), relu=kind == "ragged", f32=kind == "inner")


@pytest.mark.parametrize("kind", ["one", "ragged", "inner"])
@pytest.mark.parametrize("M,K,N,R,adapters", SIZES)
def test_backward(dr, M, K, N, R, adapters, kind):
    check_backward(dr, Case(M, K, N, R, adapters, kind))


@pytest.mark.parametrize("kind", ["rows", "even", "none"])
@pytest.mark.parametrize("M,K,N,R,adapters", [(5, 64, 48, 8, 3), (40, 256, 200, 16, 40), (128, 136, 264, 8, 128), (150, 64, 64, 12, 17), (300, 96, 136, 64, 70), (700, 72, 80, 5, 4)])
def test_requests_of_every_kind(dr, M, K, N, R, adapters, kind):
    c = Case(M, K, N, R, adapters, kind)
    check_forward(dr, c)
    check_backward(dr, c)


@pytest.mark.parametrize("M,K,N,R,adapters,kind", [
    (1, 64, 64, 8, 1, "one"), (32, 96, 40, 8, 4, "rows"), (130, 264, 136, 16, 3, "ragged"), (257, 147, 64, 5, 4, "ragged"), (640, 528, 160, 12, 9, "even"),
    (513, 64, 256, 8, 4, "inner"), (385, 512, 320, 64, 2, "one"), (90, 1031, 72, 33, 2, "ragged")])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_dropout_in_front_of_the_adapter(dr, M, K, N, R, adapters, kind, p):
    c = Case(M, K, N, R, adapters, kind)
    check_forward(dr, c, p=p, f32=True, seed=(1 << 63) + 5, offset=(1 << 35) + 1)
    check_backward(dr, c, p=p, seed=(1 << 63) + 5, offset=(1 << 35) + 1)


def test_everything_dropped_leaves_the_shared_layer(dr):
    c = Case(70, 64, 48, 8, 2)
    check_forward(dr, c, p=1.0)
    check_backward(dr, c, p=1.0)


@pytest.mark.parametrize("relu,bias,f32,scale", [(a, b, c, d) for a in (0, 1) for b in (0, 1) for c in (0, 1) for d in (0, 1)])
def test_options(dr, relu, bias, f32, scale):
    for M in (6, 200):
        check_forward(dr, Case(M, 80, 104, 8, 3), relu=bool(relu), bias=bool(bias), f32=bool(f32), scale=bool(scale), keep_t=bool(scale))


@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, False, True)])
def test_gradients_one_by_one(dr, want):
    for M in (6, 200):
        check_backward(dr, Case(M, 80, 104, 8, 3), want=want, scale=False)


@pytest.mark.parametrize("M,K,N,ldx,ldy", [(9, 64, 48, 72, 56), (9, 64, 48, 65, 49), (150, 64, 48, 64 + 8, 48 + 8), (150, 63, 47, 64, 48), (300, 72, 40, 73, 41), (300, 72, 200, 80, 203),
                                           (77, 9, 8, 16, 8)])
def test_strides(dr, M, K, N, ldx, ldy):
    c = Case(M, K, N, 8, 3)
    check_forward(dr, c, ldx=ldx, ldy=ldy)
    check_forward(dr, c, ldx=ldx, ldy=ldy, f32=True)
    check_backward(dr, c, ldx=ldx, lddy=ldy, lddx=ldx + 1)
    check_backward(dr, c, ldx=ldx, lddy=ldy, lddx=ldx, p=0.3)


@pytest.mark.parametrize("M", [24, 300])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_is_not_finite_stays_with_its_request(dr, M, bad):
    """A variant with a NaN or an infinity, and a row of x or dy with one, touch no other request's rows, gradients or variants."""
    c = Case(M, 72, 136, 8, 4, "even")
    c.a[1, 3, 5] = bad
    c.b[2, 70, 4] = bad
    c.b[2, 135, 7] = bad
    ids = np.repeat(c.ids, np.diff(c.row_start))
    row = int(np.nonzero(ids == 3)[0][-1])
    c.x[row, 9] = bad
    c.dy[row, 11] = bad
    with np.errstate(invalid="ignore"):
        y, t = A.forward(c.x, c.w, c.bias, c.a, c.b, c.scale, c.row_start, c.ids, False)
        gy, gt, _ = forward(dr, c, f32=True)
        assert np.array_equal(np.isfinite(gy), np.isfinite(y)) and np.array_equal(np.isfinite(gt), np.isfinite(t))
        assert np.array_equal(np.isnan(gy), np.isnan(y))
        tt = np.nan_to_num(t, nan=0.5, posinf=0.5, neginf=0.5).astype(np.float32).astype(np.float64)
        dx, da, db = A.backward(c.dy, c.x, c.w, c.a, c.b, c.scale, c.row_start, c.ids, tt)
        gdx, gda, gdb, _ = backward(dr, c, tt)
        for got, want in ((gdx, dx), (gda, da), (gdb, db)):
            assert np.array_equal(np.isfinite(got), np.isfinite(want))
        clean = np.isfinite(y)
        assert np.allclose(gy[clean], y[clean], rtol=1e-4, atol=1e-3)


@pytest.mark.parametrize("M,K,N,R,adapters,kind,p", [
    (14300, 520, 72, 24, 3, "ragged", 0.0), (14299, 576, 40, 130, 2, "inner", 0.0), (14336, 512, 520, 64, 5, "even", 0.0), (19000, 64, 256, 8, 4, "even", 0.0),
    (38100, 72, 24, 16, 3, "ragged", 0.1), (20000, 1024, 512, 8, 2, "one", 0.0), (9500, 136, 264, 16, 90, "ragged", 0.2)])
def test_many_rows(dr, M, K, N, R, adapters, kind, p):
    """The kernels for many rows: tiles on tensor cores for the first product, pairs of CTAs and pairs with two accumulators for the second, shares of rows that end
    inside an adapter for the gradients."""
    c = Case(M, K, N, R, adapters, kind)
    check_forward(dr, c, p=p, relu=R == 24, f32=R == 64)
    check_backward(dr, c, p=p)


@pytest.mark.parametrize("M,K,N,R,adapters,kind,p", [
    (60001, 40, 16, 8, 3, "ragged", 0.0), (40000, 72, 9, 5, 4, "inner", 0.1), (19003, 67, 131, 12, 6, "ragged", 0.1), (38001, 16, 72, 20, 3, "even", 0.0),
    (19003, 579, 131, 12, 6, "ragged", 0.1), (19003, 131, 579, 12, 6, "ragged", 0.0)])
def test_many_rows_of_narrow_and_odd_layers(dr, M, K, N, R, adapters, kind, p):
    """Several tiles to a CTA with the narrowest accumulators, and aligned copies of many rows."""
    c = Case(M, K, N, R, adapters, kind)
    check_forward(dr, c, p=p, relu=R == 8, f32=R == 5)
    check_backward(dr, c, p=p)


@pytest.mark.parametrize("M,K,N,p", [(19000, 264, 136, 0.0), (19000, 136, 264, 0.25), (19500, 1024, 1024, 0.0), (19000, 520, 136, 0.0), (19000, 136, 520, 0.0)])
@pytest.mark.parametrize("f32", [False, True])
def test_what_is_not_finite_stays_with_its_request_in_pairs(dr, M, K, N, p, f32):
    """The same for the tiles of two CTAs, which both drain what either of them reads of a variant."""
    c = Case(M, K, N, 16, 5, "ragged")
    c.a[1, 3, 5], c.a[2, 15, K - 1] = np.inf, np.nan
    c.b[2, 70, 4], c.b[0, N - 1, 15], c.b[3, 3, 0] = np.nan, -np.inf, np.inf
    ids = np.full(M, -1)
    for u, v, a in A.requests(c.row_start, c.ids, 5):
        ids[u:v] = a
    row = int(np.nonzero(ids == 4)[0][-1])
    c.x[row, 9], c.dy[row, 11] = np.inf, np.nan
    f = A.factors(M, K, p, 77, 5) if p else None
    with np.errstate(invalid="ignore"):
        y, t = A.forward(c.x, c.w, c.bias, c.a, c.b, c.scale, c.row_start, c.ids, False, f)
        gy, gt, inside = forward(dr, c, p, f32=f32)
        gy, y, gt, t = gy[inside], y[inside], gt[inside], t[inside]
        assert np.array_equal(np.isfinite(gt), np.isfinite(t))
        assert np.array_equal(np.isnan(gy), np.isnan(y)) and np.array_equal(np.isposinf(gy), np.isposinf(y)) and np.array_equal(np.isneginf(gy), np.isneginf(y))
        clean = np.isfinite(y)
        assert np.allclose(gy[clean], y[clean], rtol=2 * U16, atol=2 * U16)
        tt = np.nan_to_num(A.forward(c.x, c.w, None, c.a, c.b, c.scale, c.row_start, c.ids, False, f)[1], nan=0.5, posinf=0.5, neginf=0.5)
        tt = tt.astype(np.float32).astype(np.float64)
        dx, da, db = A.backward(c.dy, c.x, c.w, c.a, c.b, c.scale, c.row_start, c.ids, tt, f)
        gdx, gda, gdb, _ = backward(dr, c, tt, p)
        for got, want in ((gdx[inside], dx[inside]), (gda, da), (gdb, db)):
            assert np.array_equal(np.isfinite(got), np.isfinite(want))


def test_same_on_every_run(dr):
    for M, kind in ((40, "rows"), (700, "ragged"), (3000, "one")):
        c = Case(M, 136, 200, 16, 5, kind)
        t = np.nan_to_num(A.forward(c.x, c.w, None, c.a, c.b, c.scale, c.row_start, c.ids, False)[1])
        one, two = forward(dr, c, f32=True), forward(dr, c, f32=True)
        assert np.array_equal(one[0], two[0]) and np.array_equal(one[1], two[1])
        one, two = backward(dr, c, t, p=0.2), backward(dr, c, t, p=0.2, fill=0x55)
        assert all(np.array_equal(a, b) for a, b in zip(one[:3], two[:3]))


def test_offsets_that_decrease_read_and_write_nothing_out_of_range(dr):
    c = Case(150, 64, 48, 8, 3)
    c.row_start, c.ids = [40, 10, 300, -5, 90], [0, 2, 99, -7]
    import torch
    bf = torch.bfloat16
    xb, x = dev(c.x, bf)
    yb, y = dev(np.full((c.M, c.N), MARK), bf)
    d = dr.dr_adapter_desc(Cin=c.K, Cout=c.N, rank=c.R, adapters=c.adapters, flags=0)
    ws = scratch(dr.dr_adapter_workspace_bytes(d, c.M, 0))
    w, a, b = flat(c.w, bf), flat(c.a, bf), flat(c.b, bf)
    dr.dr_adapter(d, c.M, x, 0, w, None, a, b, None, 4, ints(c.row_start), ints(c.ids), y, 0, None, None, ws, ws.numel())
    got = y.double().cpu().numpy()
    # every row is one request's, or untouched
    options = [np.full_like(got, MARK)] + [A.forward(c.x, c.w, None, c.a, c.b, None, [0, c.M], [v], False)[0] for v in (-1, 0, 1, 2)]
    for m in range(c.M):
        assert min(np.abs(got[m] - o[m]).max() for o in options) < 0.1
    t = torch.zeros((c.M, c.R), device="cuda")
    da, db = torch.empty((3, 8, 64), device="cuda"), torch.empty((3, 48, 8), device="cuda")
    dx = torch.empty((c.M, c.K), dtype=bf, device="cuda")
    ws = scratch(dr.dr_adapter_bwd_workspace_bytes(d, c.M, 0, 0))
    dr.dr_adapter_bwd(d, c.M, flat(c.dy, bf), 0, x, 0, w, a, b, None, 4, ints(c.row_start), ints(c.ids), t, dx, 0, da, db, None, ws, ws.numel())
    assert dr.dr_device_status()[0] == 0


def test_no_requests_give_zero_gradients(dr):
    import torch
    d = dr.dr_adapter_desc(Cin=64, Cout=48, rank=8, adapters=3, flags=0)
    da, db = torch.full((3, 8, 64), 5.0, device="cuda"), torch.full((3, 48, 8), 5.0, device="cuda")
    dr.dr_adapter_bwd(d, 10, None, 0, None, 0, None, None, None, None, 0, None, None, None, None, 0, da, db, None, None, 0)
    assert not da.any() and not db.any()
    c = Case(20, 64, 48, 8, 3)
    c.row_start, c.ids = [0, 0, 0], [1, 2]                 # requests, but no rows in them
    check_backward(dr, c)
    check_forward(dr, c)


def test_captured_calls_follow_requests_and_counter(dr):
    """A captured pair of calls serves other requests, and draws another mask, when the device arrays have changed; two graphs share a workspace."""
    import torch
    c = Case(90, 64, 48, 8, 3, "even")
    bf, ff = torch.bfloat16, torch.float32
    x, w, a, b, s, dy = flat(c.x, bf), flat(c.w, bf), flat(c.a, bf), flat(c.b, bf), flat(c.scale, ff), flat(c.dy, bf)
    rs, ad, step = ints(c.row_start), ints(c.ids), torch.zeros(1, dtype=torch.int64, device="cuda")
    d = dr.dr_adapter_desc(Cin=c.K, Cout=c.N, rank=c.R, adapters=3, flags=dr.DR_OUT_F32, drop_p=0.25, drop_seed=3, drop_offset=100)
    ws = scratch(max(dr.dr_adapter_workspace_bytes(d, c.M, 0), dr.dr_adapter_bwd_workspace_bytes(d, c.M, 0, 0)))
    y, t = torch.zeros((c.M, c.N), device="cuda"), torch.zeros((c.M, c.R), device="cuda")
    dx, da, db = torch.zeros((c.M, c.K), dtype=bf, device="cuda"), torch.zeros((3, 8, 64), device="cuda"), torch.zeros((3, 48, 8), device="cuda")
    fwd = lambda: dr.dr_adapter(d, c.M, x, 0, w, None, a, b, s, len(c.ids), rs, ad, y, 0, t, step, ws, ws.numel())
    bwd = lambda: dr.dr_adapter_bwd(d, c.M, dy, 0, x, 0, w, a, b, s, len(c.ids), rs, ad, t, dx, 0, da, db, step, ws, ws.numel())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fwd()
        bwd()
    torch.cuda.synchronize()
    gf, gb = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(gf):
        fwd()
    with torch.cuda.graph(gb):
        bwd()
    for i, kind in enumerate(["even", "ragged", "even"]):
        row_start, ids = requests(kind, c.M, 3, i)
        n = len(c.ids)
        row_start, ids = (row_start + [row_start[-1]] * n)[:n + 1], (ids + [0] * n)[:n]
        rs.copy_(ints(row_start)), ad.copy_(ints(ids)), step.fill_(i)
        for g in (gf, gb):
            g.replay()
        torch.cuda.synchronize()
        inside = slice(0, row_start[-1])
        f = A.factors(c.M, c.K, 0.25, 3, 100 + i)
        ry, rt = A.forward(c.x, c.w, None, c.a, c.b, c.scale, row_start, ids, False, f)
        assert np.allclose(y.double().cpu().numpy()[inside], ry[inside], rtol=1e-4, atol=1e-3)
        rdx, rda, rdb = A.backward(c.dy, c.x, c.w, c.a, c.b, c.scale, row_start, ids, np.nan_to_num(rt), f)
        assert np.allclose(dx.double().cpu().numpy()[inside], rdx[inside], rtol=2.0 ** -7, atol=2e-2)
        assert np.allclose(da.double().cpu().numpy(), rda, rtol=1e-3, atol=1e-2) and np.allclose(db.double().cpu().numpy(), rdb, rtol=1e-3, atol=1e-2)


def test_two_calls_at_once_on_two_streams(dr):
    import torch
    c = Case(700, 256, 320, 16, 4, "ragged")
    bf, ff = torch.bfloat16, torch.float32
    x, w, a, b, s = flat(c.x, bf), flat(c.w, bf), flat(c.a, bf), flat(c.b, bf), flat(c.scale, ff)
    rs, ad = ints(c.row_start), ints(c.ids)
    d = dr.dr_adapter_desc(Cin=c.K, Cout=c.N, rank=c.R, adapters=4, flags=dr.DR_OUT_F32)
    n = dr.dr_adapter_workspace_bytes(d, c.M, 0)
    ref = torch.zeros((c.M, c.N), device="cuda")
    ws = [scratch(n), scratch(n)]
    dr.dr_adapter(d, c.M, x, 0, w, None, a, b, s, len(c.ids), rs, ad, ref, 0, None, None, ws[0], n)
    outs = [[torch.zeros_like(ref) for _ in range(10)] for _ in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(10):
        for k in range(2):
            dr.dr_adapter(d, c.M, x, 0, w, None, a, b, s, len(c.ids), rs, ad, outs[k][i], 0, None, None, ws[k], n, streams[k])
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for side in outs for o in side)


def test_differences(dr):
    """The gradients against differences of the forward pass itself: the loss is linear in one factor at a time, so the step may be large."""
    c = Case(200, 64, 48, 8, 3, "even")
    f = A.factors(c.M, c.K, 0.25, 77, 5)
    loss = lambda: (forward(dr, c, p=0.25, bias=False, f32=True)[0] * c.dy).sum()
    t = A.forward(c.x, c.w, None, c.a, c.b, c.scale, c.row_start, c.ids, False, f)[1]
    gdx, gda, gdb, _ = backward(dr, c, t.astype(np.float32).astype(np.float64), p=0.25)
    rng = np.random.default_rng(0)
    for arr, grad, rel in ((c.x, gdx, 2.0 ** -8), (c.a, gda, 1e-4), (c.b, gdb, 1e-4)):
        old = arr.copy()
        h = S.round_bf16(rng.normal(size=arr.shape).astype(np.float32) * 2.0 ** -4).astype(np.float64)
        up, down = S.round_bf16((old + h).astype(np.float32)).astype(np.float64), S.round_bf16((old - h).astype(np.float32)).astype(np.float64)
        arr[...] = up
        hi = loss()
        arr[...] = down
        lo = loss()
        arr[...] = old
        want = (grad * (up - down)).sum()
        # dx rounds each element by at most 2^-8; the losses carry the forward pass' tolerance of up to SPLIT + SUM(K) of their summands' sizes
        slack = rel * np.abs(grad * (up - down)).sum() + 2 * (SPLIT + SUM(c.K)) * (np.abs(c.dy) * A.forward(
            np.abs(c.x) + 0.25, np.abs(c.w), None, np.abs(c.a) + 0.25, np.abs(c.b) + 0.25, c.scale, c.row_start, c.ids, False, f)[0]).sum()
        assert abs(hi - lo - want) <= slack, (hi - lo, want, slack)
