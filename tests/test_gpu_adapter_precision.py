"""Precision of what the low-rank adapters return as float32 (t, y, da, db) against the formulas in float64, by the 2-norm.

The tensor cores cut a sum off where the next product is added: of a unit 2^-23 or less, half in the mean, so each of n products in a row (16 terms each)
takes at most 2^-24 of what the sum has reached, which for terms of both signs is 2/3 of the result in the mean over them, and for a float32 value of 0.72 units' size
in the mean; n 2^-25 is above 0.5 x 0.72 x 2/3 of 2^-23 for each.  The sums of parts and the factors are rounded a few times more: 2^-22 for eight halves
of a unit 2^-24."""
import pytest

pytestmark = pytest.mark.gpu

FEW = 2.0 ** -22
CHAIN = 32                      # products of 16 terms in a row: sums of 512


def cut(n):
    return n * 2.0 ** -25 + FEW


@pytest.fixture(scope="module")
def dr():
    import paper_1708_04728_b200 as dr
    return dr


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


class Layer:
    """One variant for each of `segments` equal requests; kept: what the dropout keeps, drawn by dr_dropout itself."""

    def __init__(self, dr, M, K, N, R, segments, p, shared):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(M + 3 * K + 5 * N + R)
        normal = lambda s, *shape: (s * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)
        self.M, self.segments = M, segments
        self.x, self.w, self.dy = normal(1, M, K), normal(shared * K ** -0.5, N, K), normal(1, M, N)
        self.a, self.b = normal(K ** -0.5, segments, R, K), normal(R ** -0.5, segments, N, R)
        self.cuts = [M * i // segments for i in range(segments + 1)]
        self.row_start, self.ids = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (self.cuts, range(segments)))
        self.desc = dr.dr_adapter_desc(Cin=K, Cout=N, rank=R, adapters=segments, flags=dr.DR_OUT_F32, drop_p=p, drop_seed=3, drop_offset=4)
        self.kept = None
        if p:
            self.kept = torch.ones((M, K), dtype=torch.bfloat16, device="cuda")
            dr.dr_dropout(M, K, self.kept, 0, None, 0, self.kept, 0, p, 3, 4)
            self.factor = 65536 / (65536 - int(p * 65536 + 0.5))

    def parts(self):
        """(variant, rows) in pieces that fit in float64."""
        for i in range(self.segments):
            for u in range(self.cuts[i], self.cuts[i + 1], 4096):
                yield i, slice(u, min(u + 4096, self.cuts[i + 1]))

    def dropped(self, rows):
        x = self.x[rows].double()
        return x if self.kept is None else x * (self.kept[rows] != 0) * self.factor

    def forward(self, dr):
        import torch
        M, N, R = self.M, self.w.shape[0], self.a.shape[1]
        y, t = torch.full((M, N), float("nan"), device="cuda"), torch.full((M, R), float("nan"), device="cuda")
        n = dr.dr_adapter_workspace_bytes(self.desc, M)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        dr.dr_adapter(self.desc, M, self.x, 0, self.w, None, self.a, self.b, None, self.segments, self.row_start, self.ids, y, 0, t, None, ws, n)
        yr, tr = torch.empty((M, N), dtype=torch.float64, device="cuda"), torch.empty((M, R), dtype=torch.float64, device="cuda")
        for i, rows in self.parts():
            tr[rows] = self.dropped(rows) @ self.a[i].double().T
            yr[rows] = tr[rows] @ self.b[i].double().T
            for c in range(0, N, 1024):
                yr[rows, c:c + 1024] += self.x[rows].double() @ self.w[c:c + 1024].double().T
        return rel(y, yr), rel(t, tr)

    def backward(self, dr):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(9)
        M, N, K, R = self.M, self.w.shape[0], self.w.shape[1], self.a.shape[1]
        t = torch.randn((M, R), generator=g, device="cuda")
        da, db = torch.full((self.segments, R, K), float("nan"), device="cuda"), torch.full((self.segments, N, R), float("nan"), device="cuda")
        n = dr.dr_adapter_bwd_workspace_bytes(self.desc, M)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        dr.dr_adapter_bwd(self.desc, M, self.dy, 0, self.x, 0, self.w, self.a, self.b, None, self.segments, self.row_start, self.ids, t, None, 0, da, db, None, ws, n)
        dar, dbr = torch.zeros_like(da, dtype=torch.float64), torch.zeros_like(db, dtype=torch.float64)
        for i, rows in self.parts():
            dy = self.dy[rows].double()
            dar[i] += (dy @ self.b[i].double()).T @ self.dropped(rows)
            dbr[i] += dy.T @ t[rows].double()
        return rel(da, dar), rel(db, dbr)


# rows, Cin, rank, requests, dropout: fragments (warps that share l, clusters that do, warps of rows of their own), tiles of 128 rows
FIRST = [(32, 65536, 16, 1, 0.0), (3000, 9216, 8, 3, 0.0), (3000, 9216, 24, 40, 0.1), (5000, 65536, 8, 1, 0.0), (20000, 9216, 8, 2, 0.0), (20000, 4608, 64, 300, 0.1),
         (40000, 512, 8, 1, 0.0), (40000, 9216, 8, 3, 0.0), (40000, 9216, 16, 1, 0.1), (38000, 4096, 40, 400, 0.0), (38000, 1032, 256, 1, 0.1), (20000, 9216, 64, 2, 0.0)]


@pytest.mark.parametrize("M,K,R,segments,p", FIRST)
def test_first_product(dr, M, K, R, segments, p):
    y, t = Layer(dr, M, K, 8, R, segments, p, 2.0 ** -6).forward(dr)
    assert t <= cut(CHAIN), t


@pytest.mark.parametrize("M,N,R,segments", [(40000, 4096, 8, 1), (40000, 9216, 16, 5), (3000, 16384, 8, 1), (20000, 9216, 64, 2)])
def test_gradients_of_a_wide_layer(dr, M, N, R, segments):
    """u's precision is da's: a sum of up to 512 l in a row, then one of up to 512 rows."""
    da, db = Layer(dr, M, 64, N, R, segments, 0.0, 1.0).backward(dr)
    assert da <= cut(CHAIN) + cut(CHAIN) and db <= cut(CHAIN), (da, db)


# up to 128 rows (with more sums than accumulators, too), tiles of one CTA, pairs with several tiles to each
Y = [(1, 16384, 8192, 16, 1), (32, 9216, 4096, 8, 3), (128, 32768, 9472, 16, 1), (128, 32768, 1000, 8, 5), (40, 65536, 520, 8, 4), (7, 4096, 24, 16, 2), (300, 4096, 200, 8, 2),
     (5000, 9216, 256, 24, 4), (19000, 4096, 1024, 64, 1), (19000, 1024, 1024, 16, 5)]


@pytest.mark.parametrize("shared", [2.0 ** 6, 2.0 ** -6])
@pytest.mark.parametrize("M,K,N,R,segments", Y)
def test_float32_results(dr, M, K, N, R, segments, shared):
    """Nearly all of y the shared part's, or the adapters' (which t's precision is part of); their 3 R columns end or begin one of the sums."""
    y, t = Layer(dr, M, K, N, R, segments, 0.0, shared).forward(dr)
    assert y <= cut(CHAIN + (3 * R + 15) // 16) + (2.0 ** -5 if shared > 1 else 1) * cut(CHAIN), y


@pytest.mark.parametrize("M", [32, 200])
def test_three_terms(dr, M):
    """Sums so short that a factor of 16 bits instead of 24 (2.5e-6 of the result for normal numbers) shows."""
    y, t = Layer(dr, M, 64, 96, 16, 2, 0.0, 2.0 ** -6).forward(dr)
    assert y <= cut(4 + 3) + cut(4) < 1e-6, y
    da, db = Layer(dr, M, 64, 96, 16, 2, 0.0, 1.0).backward(dr)
    assert da <= cut(7) + cut(6) < 1e-6 and db <= cut(7) < 1e-6, (da, db)
