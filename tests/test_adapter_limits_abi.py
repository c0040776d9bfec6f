"""Host-side limits of the adapter entry points that their list of refusals lacked (no GPU needed)."""
import pytest

from test_adapter_abi import AB, AD, dr, refused

MOST = dr.DR_ADAPTER_MAX_ROWS


@pytest.mark.parametrize("call,args", [(dr.dr_adapter, AD), (dr.dr_adapter_bwd, AB)])
def test_more_requests_than_32_bits_count(call, args):
    for n in (MOST + 1, (1 << 31) - 1):
        refused(-2, call, *{**args, "segments": n}.values())
    refused(-4, call, *{**args, "segments": MOST, "nws": 16}.values())          # the limit itself gets as far as the workspace
