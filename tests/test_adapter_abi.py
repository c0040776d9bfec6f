"""Host-side checks of the dropout and adapter entry points: refusals before any launch, workspace queries (no GPU needed)."""
import pytest

import paper_1708_04728_b200 as dr

P = 4096                       # an address that is aligned for every argument; nothing is launched
BIG = 1 << 50


def refused(status, call, *args):
    n0 = dr.dr_launch_count()
    with pytest.raises(dr.DrError) as e:
        call(*args)
    assert e.value.status == status
    assert dr.dr_launch_count() == n0


def desc(**change):
    return dr.dr_adapter_desc(**{**dict(Cin=64, Cout=48, rank=8, adapters=3, flags=dr.DR_BIAS, drop_p=0.1, drop_seed=1, drop_offset=2), **change})


DROP = dict(rows=4, C=16, x=P, ldx=0, residual=P, ldr=0, y=P, ldy=0, p=0.5, seed=1, offset=2, step=P, flags=0, stream=0)
AD = dict(desc=desc(), M=5, x=P, ldx=0, w=P, bias=P, a=P, b=P, scale=P, segments=2, row_start=P, adapter=P, y=P, ldy=0, t=P, step=P, ws=P, nws=BIG, stream=0)
AB = dict(desc=desc(), M=5, dy=P, lddy=0, x=P, ldx=0, w=P, a=P, b=P, scale=P, segments=2, row_start=P, adapter=P, t=P, dx=P, lddx=0, da=P, db=P, step=P,
          ws=P, nws=BIG, stream=0)
BAD_DESC = [(dict(Cin=0), -1), (dict(Cout=-3), -1), (dict(rank=0), -1), (dict(adapters=0), -1), (dict(flags=dr.DR_POOL), -1), (dict(flags=0x100), -1),
            (dict(drop_p=-0.1), -1), (dict(drop_p=1.5), -1), (dict(drop_p=float("nan")), -1), (dict(rank=257), -2), (dict(Cin=65537), -2), (dict(Cout=65537), -2),
            (dict(adapters=4097), -2)]


@pytest.mark.parametrize("change,status", [
    (dict(x=None), -1), (dict(y=None), -1), (dict(C=0), -1), (dict(C=-1), -1), (dict(ldx=15), -1), (dict(ldr=3), -1), (dict(ldy=-1), -1), (dict(p=-1e-9), -1),
    (dict(p=1.0001), -1), (dict(p=float("nan")), -1), (dict(flags=4), -1), (dict(rows=1 << 62), -1), (dict(x=P + 1), -3), (dict(x=P + 2, flags=1), -3),
    (dict(y=P + 1), -3), (dict(y=P + 2, flags=2), -3), (dict(residual=P + 2, flags=2), -3), (dict(step=P + 4), -3)])
def test_dropout_refusals(change, status):
    refused(status, dr.dr_dropout, *{**DROP, **change}.values())


@pytest.mark.parametrize("change,status", [
    (dict(x=None), -1), (dict(w=None), -1), (dict(bias=None), -1), (dict(a=None), -1), (dict(b=None), -1), (dict(row_start=None), -1), (dict(adapter=None), -1),
    (dict(y=None), -1), (dict(ws=None), -1), (dict(M=-1), -1), (dict(segments=-1), -1), (dict(ldx=63), -1), (dict(ldy=47), -1), (dict(M=(1 << 30) + 1), -2),
    (dict(x=P + 2), -3), (dict(w=P + 8), -3), (dict(a=P + 8), -3), (dict(b=P + 4), -3), (dict(y=P + 1), -3), (dict(y=P + 2, desc=desc(flags=dr.DR_OUT_F32)), -3),
    (dict(bias=P + 2), -3), (dict(scale=P + 1), -3), (dict(row_start=P + 2), -3), (dict(adapter=P + 2), -3), (dict(t=P + 2), -3), (dict(step=P + 4), -3),
    (dict(ws=P + 128), -3), (dict(nws=16), -4)] + [(dict(desc=desc(**d)), s) for d, s in BAD_DESC])
def test_adapter_refusals(change, status):
    refused(status, dr.dr_adapter, *{**AD, **change}.values())


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), -1), (dict(x=None), -1), (dict(w=None), -1), (dict(a=None), -1), (dict(b=None), -1), (dict(row_start=None), -1), (dict(adapter=None), -1),
    (dict(t=None), -1), (dict(ws=None), -1), (dict(M=-1), -1), (dict(segments=-1), -1), (dict(ldx=63), -1), (dict(lddx=63), -1), (dict(lddy=47), -1),
    (dict(M=(1 << 30) + 1), -2), (dict(dy=P + 2), -3), (dict(x=P + 2), -3), (dict(w=P + 8), -3), (dict(a=P + 8), -3), (dict(b=P + 4), -3), (dict(dx=P + 1), -3),
    (dict(scale=P + 1), -3), (dict(row_start=P + 2), -3), (dict(adapter=P + 2), -3), (dict(t=P + 2), -3), (dict(da=P + 2), -3), (dict(db=P + 2), -3),
    (dict(step=P + 4), -3), (dict(ws=P + 128), -3), (dict(nws=16), -4)] + [(dict(desc=desc(**d)), s) for d, s in BAD_DESC])
def test_adapter_bwd_refusals(change, status):
    refused(status, dr.dr_adapter_bwd, *{**AB, **change}.values())


def test_workspace_queries():
    for d in (desc(), desc(Cin=63, Cout=1000, rank=5)):
        a, b = dr.dr_adapter_workspace_bytes(d, 100, 0), dr.dr_adapter_workspace_bytes(d, 100000, 0)
        assert a % 256 == 0 and 0 < a < b
        a, b = dr.dr_adapter_bwd_workspace_bytes(d, 100, 0, 0), dr.dr_adapter_bwd_workspace_bytes(d, 100000, 0, 0)
        assert a % 256 == 0 and 0 < a < b
    for d, status in BAD_DESC:
        refused(status, dr.dr_adapter_workspace_bytes, desc(**d), 4, 0)
        refused(status, dr.dr_adapter_bwd_workspace_bytes, desc(**d), 4, 0, 0)
    refused(-1, dr.dr_adapter_workspace_bytes, desc(), -1, 0)
    refused(-1, dr.dr_adapter_workspace_bytes, desc(), 4, 63)
    refused(-1, dr.dr_adapter_bwd_workspace_bytes, desc(), 4, 64, 47)
    assert dr._lib.dr_adapter_workspace_bytes(desc(), 4, 0, None) == -1
    assert dr._lib.dr_adapter_workspace_bytes(None, 4, 0, None) == -1


def test_nothing_to_do_is_no_error():
    n0 = dr.dr_launch_count()
    dr.dr_dropout(*{**DROP, "rows": 0}.values())
    dr.dr_adapter(*{**AD, "M": 0}.values())
    dr.dr_adapter(*{**AD, "segments": 0}.values())
    dr.dr_adapter_bwd(*{**AB, "M": 0, "da": None, "db": None}.values())
    assert dr.dr_launch_count() == n0
