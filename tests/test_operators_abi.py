"""Host-side checks of the layer-normalisation and orthogonalised-update entry points: refusals before any launch,
workspace queries (no GPU needed)."""
import ctypes as C

import pytest

import paper_1708_04728_b200 as dr

P = 4096                       # an address that is aligned for every argument; nothing is launched
BIG = 1 << 40


def refused(status, call, *args):
    n0 = dr.dr_launch_count()
    with pytest.raises(dr.DrError) as e:
        call(*args)
    assert e.value.status == status
    assert dr.dr_launch_count() == n0


LN = dict(npix=4, C=16, x=P, ldx=0, gamma=P, beta=P, eps=1e-5, y=P, ldy=0, mean=P, rstd=P, flags=0, stream=0)
LNB = dict(npix=4, C=16, dy=P, lddy=0, x=P, ldx=0, gamma=P, mean=P, rstd=P, dx=P, lddx=0, dgamma=P, dbeta=P, ws=P, nws=BIG, flags=0, stream=0)
NS = dict(batch=1, rows=32, cols=48, g=P, steps=5, coef=None, eps=1e-7, o=P, ws=P, nws=BIG, flags=0, stream=0)
MU = dict(batch=1, rows=32, cols=48, w=P, v=P, g=P, lr=0.1, momentum=0.9, decay=0.0, nesterov=1, steps=5, coef=None, eps=1e-7, w_bf16=P, ws=P, nws=BIG, stream=0)


@pytest.mark.parametrize("call,base,change,status", [
    (dr.dr_layernorm, LN, dict(x=None), -1), (dr.dr_layernorm, LN, dict(y=None), -1), (dr.dr_layernorm, LN, dict(C=0), -1),
    (dr.dr_layernorm, LN, dict(ldx=15), -1), (dr.dr_layernorm, LN, dict(ldy=-1), -1), (dr.dr_layernorm, LN, dict(eps=-1.0), -1),
    (dr.dr_layernorm, LN, dict(eps=float("nan")), -1), (dr.dr_layernorm, LN, dict(flags=4), -1), (dr.dr_layernorm, LN, dict(x=P + 1), -3),
    (dr.dr_layernorm, LN, dict(x=P + 2, flags=1), -3), (dr.dr_layernorm, LN, dict(gamma=P + 2), -3), (dr.dr_layernorm, LN, dict(mean=P + 1), -3),
    (dr.dr_layernorm_bwd, LNB, dict(dy=None), -1), (dr.dr_layernorm_bwd, LNB, dict(mean=None), -1), (dr.dr_layernorm_bwd, LNB, dict(rstd=None), -1),
    (dr.dr_layernorm_bwd, LNB, dict(dx=None), -1), (dr.dr_layernorm_bwd, LNB, dict(ws=None), -1), (dr.dr_layernorm_bwd, LNB, dict(lddy=3), -1),
    (dr.dr_layernorm_bwd, LNB, dict(C=-4), -1), (dr.dr_layernorm_bwd, LNB, dict(nws=8), -4), (dr.dr_layernorm_bwd, LNB, dict(ws=P + 128), -3),
    (dr.dr_layernorm_bwd, LNB, dict(dgamma=P + 2), -3), (dr.dr_layernorm_bwd, LNB, dict(flags=8), -1),
    (dr.dr_orthogonalise, NS, dict(g=None), -1), (dr.dr_orthogonalise, NS, dict(o=None), -1), (dr.dr_orthogonalise, NS, dict(ws=None), -1),
    (dr.dr_orthogonalise, NS, dict(rows=0), -1), (dr.dr_orthogonalise, NS, dict(cols=-1), -1), (dr.dr_orthogonalise, NS, dict(batch=-1), -1),
    (dr.dr_orthogonalise, NS, dict(steps=0), -1), (dr.dr_orthogonalise, NS, dict(steps=17), -2), (dr.dr_orthogonalise, NS, dict(rows=65537), -2),
    (dr.dr_orthogonalise, NS, dict(batch=65536), -2), (dr.dr_orthogonalise, NS, dict(nws=64), -4), (dr.dr_orthogonalise, NS, dict(ws=P + 16), -3),
    (dr.dr_orthogonalise, NS, dict(g=P + 2, flags=1), -3), (dr.dr_orthogonalise, NS, dict(o=P + 1), -3), (dr.dr_orthogonalise, NS, dict(flags=2), -1),
    (dr.dr_orthogonalise, NS, dict(eps=float("nan")), -1), (dr.dr_orthogonalise, NS, dict(coef=[1.0, float("inf"), 0.0] * 5), -1),
    (dr.dr_muon_update, MU, dict(w=None), -1), (dr.dr_muon_update, MU, dict(v=None), -1), (dr.dr_muon_update, MU, dict(g=None), -1),
    (dr.dr_muon_update, MU, dict(ws=None), -1), (dr.dr_muon_update, MU, dict(w=P + 2), -3), (dr.dr_muon_update, MU, dict(w_bf16=P + 1), -3),
    (dr.dr_muon_update, MU, dict(nws=64), -4), (dr.dr_muon_update, MU, dict(steps=-2), -1), (dr.dr_muon_update, MU, dict(rows=1 << 20), -2),
])
def test_refusals(call, base, change, status):
    refused(status, call, *{**base, **change}.values())


def test_wrong_number_of_coefficients():
    with pytest.raises(ValueError):
        dr.dr_orthogonalise(*{**NS, "coef": [1.0, 2.0, 3.0]}.values())


def test_workspace_queries():
    n = dr.dr_layernorm_bwd_workspace_bytes(200704, 256)
    assert n % 256 == 0 and 2 * 256 * 4 <= n <= 64 << 20
    assert dr.dr_layernorm_bwd_workspace_bytes(1, 1) >= 8
    a, b = dr.dr_orthogonalise_workspace_bytes(1, 192, 576), dr.dr_orthogonalise_workspace_bytes(6, 192, 576)
    assert a % 256 == 0 and a < b and dr.dr_orthogonalise_workspace_bytes(1, 576, 192) == a
    refused(-1, dr.dr_orthogonalise_workspace_bytes, 1, 0, 4)
    refused(-2, dr.dr_orthogonalise_workspace_bytes, 1, 70000, 4)
    refused(-1, dr.dr_layernorm_bwd_workspace_bytes, 4, 0)
    assert dr._lib.dr_layernorm_bwd_workspace_bytes(4, 4, None) == -1
    assert dr._lib.dr_orthogonalise_workspace_bytes(1, 4, 4, None) == -1


def test_nothing_to_do_is_no_error():
    n0 = dr.dr_launch_count()
    dr.dr_layernorm(*{**LN, "npix": 0}.values())
    dr.dr_orthogonalise(*{**NS, "batch": 0}.values())
    dr.dr_muon_update(*{**MU, "batch": 0}.values())
    assert dr.dr_launch_count() == n0
