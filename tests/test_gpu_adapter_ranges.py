"""The ends of what the low-rank adapters' arguments may hold: offsets that decrease in large tensors, many empty requests, elements beyond 2^32."""
import numpy as np
import pytest

import oracle.adapter as A
from test_gpu_adapter import Case, check_backward, check_forward, dr, ints  # noqa: F401  (dr: the fixture)

pytestmark = pytest.mark.gpu


def test_offsets_that_decrease_over_many_rows(dr):
    """2^24 rows, and 512 requests of which every other one has all of them: the lists of the gradients hold each row once, and nothing outside them is written."""
    import torch
    M, C, R, n = 1 << 24, 8, 8, 512
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    x, dy, w, a, b = normal(M, C), normal(M, C), normal(C, C), normal(2, R, C), normal(2, C, R)
    t = torch.randn((M, R), generator=g, device="cuda")
    d = dr.dr_adapter_desc(Cin=C, Cout=C, rank=R, adapters=2, flags=0)
    size, guard = dr.dr_adapter_bwd_workspace_bytes(d, M, 0, 0), 1 << 20
    buf = torch.full((size + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
    out = []
    for row_start, ids in (([0, M] * (n // 2) + [0], [1] * n), ([0, M], [1])):
        da, db = torch.full((2, R, C), 7.0, device="cuda"), torch.full((2, C, R), 7.0, device="cuda")
        dr.dr_adapter_bwd(d, M, dy, 0, x, 0, w, a, b, None, len(ids), ints(row_start), ints(ids), t, None, 0, da, db, None, buf[guard:], size)
        torch.cuda.synchronize()
        out.append((da, db))
    assert bool((buf[:guard] == 0xA5).all()) and bool((buf[guard + size:] == 0xA5).all())
    assert dr.dr_device_status()[0] == 0
    # the first request has every row already: the list is that of a single request
    assert torch.equal(out[0][1], out[1][1]) and not out[0][0][0].any() and bool(torch.isfinite(out[0][0]).all())


@pytest.mark.parametrize("M", [90, 300, 2500])
def test_many_empty_requests_among_neighbouring_rows(dr, M):
    """More offsets between the first and the last row of a warp than it counts out of registers."""
    rng = np.random.default_rng(M)
    c = Case(M, 72, 40, 8, 5)
    cuts = np.concatenate([[0] * 3, [10] * 100, [11] * 40, [12, 30], np.sort(rng.integers(30, M - 3, 70)), [M // 2] * 200, [M - 3] * 33])
    c.row_start = np.sort(cuts).tolist()
    c.ids = rng.integers(-1, 5, len(cuts) - 1).tolist()
    check_forward(dr, c)
    check_backward(dr, c)


@pytest.mark.parametrize("K", [8200, 8203])
def test_elements_beyond_32_bits(dr, K):
    """x of more than 2^32 elements behind a dropout: the first rows and the last ones, which are a variant's own, forward and backward."""
    import torch
    M, N, R, own, p, seed, offset = 530000, 16, 8, 5, 0.25, 31, 32
    g = torch.Generator(device="cuda")
    g.manual_seed(K)
    normal = lambda s, *shape: (s * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)
    x, dy = torch.empty((M, K), dtype=torch.bfloat16, device="cuda").normal_(generator=g), normal(1, M, N)
    w, a, b = normal(K ** -0.5, N, K), normal(K ** -0.5, 2, R, K), normal(R ** -0.5, 2, N, R)
    row_start, ids = ints([0, M - own, M]), ints([0, 1])
    d = dr.dr_adapter_desc(Cin=K, Cout=N, rank=R, adapters=2, flags=dr.DR_OUT_F32, drop_p=p, drop_seed=seed, drop_offset=offset)
    ws = torch.empty(max(dr.dr_adapter_workspace_bytes(d, M), dr.dr_adapter_bwd_workspace_bytes(d, M)), dtype=torch.uint8, device="cuda")
    y, t = torch.empty((M, N), device="cuda"), torch.empty((M, R), device="cuda")
    dr.dr_adapter(d, M, x, 0, w, None, a, b, None, 2, row_start, ids, y, 0, t, None, ws, ws.numel())
    dx, da, db = torch.empty_like(x), torch.empty((2, R, K), device="cuda"), torch.empty((2, N, R), device="cuda")
    dr.dr_adapter_bwd(d, M, dy, 0, x, 0, w, a, b, None, 2, row_start, ids, t, dx, 0, da, db, None, ws, ws.numel())
    host = lambda v: v.double().cpu().numpy()
    hw, ha, hb = host(w), host(a), host(b)
    for first, rows, variant in ((0, 3, 0), (M - own, own, 1)):
        part = slice(first, first + rows)
        f = A.factors(rows, K, p, seed, offset, first=first * K)
        hx, hdy, ht = host(x[part]), host(dy[part]), host(t[part])
        ry, rt = A.forward(hx, hw, None, ha, hb, None, [0, rows], [variant], False, f)
        # float32 sums of K products of numbers of both signs: their size is about that of the result, their rounding far below 1e-5 of it
        assert np.linalg.norm(ht - rt) <= 1e-5 * np.linalg.norm(rt) and np.linalg.norm(host(y[part]) - ry) <= 1e-5 * np.linalg.norm(ry)
        rdx, rda, rdb = A.backward(hdy, hx, hw, ha, hb, None, [0, rows], [variant], ht, f)
        assert np.linalg.norm(host(dx[part]) - rdx) <= 2.0 ** -8 * np.linalg.norm(rdx)          # bfloat16: half a unit in the last place
    assert np.linalg.norm(host(da[1]) - rda[1]) <= 1e-5 * np.linalg.norm(rda[1]) and np.linalg.norm(host(db[1]) - rdb[1]) <= 1e-5 * np.linalg.norm(rdb[1])


@pytest.mark.parametrize("M,K,N", [(1, 65536, 512), (20, 16384, 24), (5, 64, 20000)])
def test_few_rows_on_three_streams(dr, M, K, N):
    """Clusters of several calls at once share the SMs' tensor memory: all end, with the bits of a call alone."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    normal = lambda s, *shape: (s * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)
    x, w, a, b = normal(1, M, K), normal(K ** -0.5, N, K), normal(K ** -0.5, 1, 16, K), normal(0.25, 1, N, 16)
    row_start, ids = ints([0, M]), ints([0])
    d = dr.dr_adapter_desc(Cin=K, Cout=N, rank=16, adapters=1, flags=dr.DR_OUT_F32)
    n = dr.dr_adapter_workspace_bytes(d, M)
    streams = [torch.cuda.Stream() for _ in range(3)]
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in streams]
    call = lambda y, k, s: dr.dr_adapter(d, M, x, 0, w, None, a, b, None, 1, row_start, ids, y, 0, None, None, ws[k], n, s)
    alone = torch.empty((M, N), device="cuda")
    call(alone, 0, torch.cuda.current_stream())
    outs = [[torch.zeros_like(alone) for _ in range(12)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(12):
        for k, s in enumerate(streams):
            call(outs[k][i], k, s)
    torch.cuda.synchronize()
    assert all(torch.equal(y, alone) for side in outs for y in side) and dr.dr_device_status()[0] == 0


def test_as_many_requests_as_there_may_be(dr):
    """2^30 requests, all but three of them empty: the backward pass' lists take seconds, longer than any wait of the kernels behind them may last."""
    import torch
    M, n = 300, dr.DR_ADAPTER_MAX_ROWS
    c = Case(M, 72, 40, 8, 1)
    bf, flat = torch.bfloat16, lambda v, t: torch.from_numpy(np.ascontiguousarray(v)).cuda().to(t).contiguous()
    row_start, ids = torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.full((n,), -1, dtype=torch.int32, device="cuda")
    row_start[n // 3 + 1:] = 100                    # request n / 3 has the rows 0 .. 99, 2 n / 3 the rows 100 .. 249, the last one 250 .. 289
    row_start[2 * (n // 3) + 1:] = 250
    row_start[n:] = 290
    ids[n // 3] = ids[n - 1] = 0
    few = ([0, 100, 250, 290], [0, -1, 0])
    x, w, a, b, dy = (flat(v, bf) for v in (c.x, c.w, c.a, c.b, c.dy))
    d = dr.dr_adapter_desc(Cin=72, Cout=40, rank=8, adapters=1, flags=dr.DR_OUT_F32)
    ws = torch.empty(max(dr.dr_adapter_workspace_bytes(d, M), dr.dr_adapter_bwd_workspace_bytes(d, M)), dtype=torch.uint8, device="cuda")
    out = []
    for starts, variants, segments in ((row_start, ids, n), (ints(few[0]), ints(few[1]), 3)):
        y, t, dx = (torch.full((M, k), 7.0, dtype=ty, device="cuda") for k, ty in ((40, torch.float32), (8, torch.float32), (72, bf)))
        da, db = torch.full((1, 8, 72), 7.0, device="cuda"), torch.full((1, 40, 8), 7.0, device="cuda")
        dr.dr_adapter(d, M, x, 0, w, None, a, b, None, segments, starts, variants, y, 0, t, None, ws, ws.numel())
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        dr.dr_adapter_bwd(d, M, dy, 0, x, 0, w, a, b, None, segments, starts, variants, t, dx, 0, da, db, None, ws, ws.numel())
        end.record()
        torch.cuda.synchronize()
        print(f"{segments} requests: {begin.elapsed_time(end):.1f} ms")
        assert dr.dr_device_status()[0] == 0
        out.append((y, t, dx, da, db))
    assert all(torch.equal(p, q) for p, q in zip(*out))
    ry, _ = A.forward(c.x, c.w, None, c.a, c.b, None, *few, False)
    assert np.allclose(out[0][0].double().cpu().numpy()[:290], ry[:290], rtol=1e-4, atol=1e-4)
