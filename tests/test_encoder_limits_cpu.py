"""CPU-only: a launch has fewer than 2^32 threads, and calls of more are refused before anything is
launched.  A call inside the limits is seen to pass the checks by its refusal of a workspace that is
too small, so that nothing is launched here either."""

import pytest

import paper_2505_04846_amd as hpr
from test_encoder_abi_cpu import _adapters, _attn_bwd, _attn_fwd, _desc

OUTSIDE, NO_WORKSPACE = 4, 5


@pytest.mark.parametrize("call,desc,status", [
    # 8 kv heads of one query head, sequences of 33 rows and more (256 threads a tile)
    (_attn_fwd, dict(n_q=70 << 20, n_k=70 << 20, n_seq=(2 << 20) - (70 << 13)), OUTSIDE),
    (_attn_fwd, dict(n_q=70 << 20, n_k=70 << 20, n_seq=(2 << 20) - (70 << 13) - 1), NO_WORKSPACE),
    # one row of each sequence (64 threads a tile): the forward goes on where the gradients end
    (_attn_fwd, dict(n_q=1 << 21, n_k=1 << 21, n_seq=1 << 21), NO_WORKSPACE),
    (_attn_bwd, dict(n_q=1 << 21, n_k=1 << 21, n_seq=1 << 21), OUTSIDE),
    (_attn_bwd, dict(n_q=1 << 7, n_k=1 << 7, n_seq=(1 << 21) - 1), OUTSIDE),
    (_attn_bwd, dict(n_q=1 << 7, n_k=1 << 7, n_seq=(1 << 21) - 2), NO_WORKSPACE),
    (_attn_bwd, dict(n_q=1, n_k=(1 << 28) - 129, n_seq=1), NO_WORKSPACE),
    (_attn_bwd, dict(n_q=1, n_k=1 << 28, n_seq=1), OUTSIDE),
    (_attn_fwd, dict(n_q=1 << 23, n_k=1 << 23, n_seq=1 << 23), OUTSIDE),
])
def test_attention(call, desc, status):
    assert call(_desc(heads=8, kv_heads=8, dim=8, **desc), ws_bytes=0) == status


@pytest.mark.parametrize("kw,status", [
    (dict(n=1 << 26, n_req=(1 << 24) - (1 << 21), k=8, m=8), OUTSIDE),
    (dict(n=32, n_req=(1 << 24) - 2, k=8, m=8), NO_WORKSPACE),
    (dict(n=32, n_req=(1 << 24) - 1, k=8, m=8), OUTSIDE),
    (dict(n=1 << 24, k=1 << 15, m=8), OUTSIDE),
    (dict(n=(1 << 24) - 256, k=1 << 15, m=8), NO_WORKSPACE),
    (dict(n=32, n_ad=1 << 14, k=1 << 16, m=8, r=1), OUTSIDE),
    (dict(n=32, n_ad=(1 << 14) - 32, k=1 << 16, m=8, r=1), NO_WORKSPACE),
])
def test_adapter_gradients(kw, status):
    assert _adapters("bwd", ws_bytes=0, **kw) == status


@pytest.mark.parametrize("kw", [dict(n=1 << 31), dict(n=1 << 29), dict(n=32, n_req=1 << 24),
                                dict(n=1 << 24, m=1 << 15, k=8)])
def test_adapter_forward(kw):
    assert _adapters("fwd", **kw) == OUTSIDE
    assert hpr.lib().hpr_last_error()


@pytest.mark.parametrize("n,r,n_ad,n_req", [(13_000, 64, 1, 13_000), (13_057, 64, 1, 216),
                                            (4_096, 16, 8, 4_096), (100_000, 64, 4, 100_000)])
def test_adapter_workspace_does_not_grow_with_requests(n, r, n_ad, n_req):
    """The partial sums follow the rows and the adapters: less than twice what one request per adapter
    takes, and 4 bytes a row."""
    size = hpr.lib().adapter_linear_bwd_workspace_size
    assert size(n, 4096, 4096, r, n_ad, n_req) <= 2 * size(n, 4096, 4096, r, n_ad, n_ad) + 4 * n
    # ... and with the requests where they are the fewer
    few = size(n, 4096, 4096, r, 1000, 1)
    assert size(n, 4096, 4096, r, 1000, 2) - few < 16 * r * 8192
