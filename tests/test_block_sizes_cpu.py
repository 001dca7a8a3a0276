"""CPU-only: the workspaces' sizes of widths that no call takes are 0."""

import ctypes

import pytest

import paper_2505_04846_amd as hpr
from test_block_abi_cpu import OUTSIDE, _desc, _gated, _norm


@pytest.mark.parametrize("width", [0, 4, 12, 63, 65535, 65544])
def test_gated(width):
    size = hpr.lib().gated_linear_bwd_workspace_size
    for k, f in ((width, 64), (64, width)):
        assert _gated("bwd", k=k, f=f) == OUTSIDE
        assert all(size(100, k, f, packed, dx, dw) == 0 for packed in (0, 1) for dx, dw in ((1, 0), (0, 1), (1, 1)))
    assert size(100, 64, 65536, 0, 1, 1) > 0 and size(100, 65536, 64, 0, 1, 1) > 0


@pytest.mark.parametrize("width", [0, 4, 12, 63, 16383, 16392])
def test_norm(width):
    size = hpr.lib().residual_norm_bwd_workspace_size
    assert _norm("bwd", dim=width) == OUTSIDE
    assert size(ctypes.byref(_desc(dim=width))) == 0
    assert size(ctypes.byref(_desc(dim=16384))) > 0
