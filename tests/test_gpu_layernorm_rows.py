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
