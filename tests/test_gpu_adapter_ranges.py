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
