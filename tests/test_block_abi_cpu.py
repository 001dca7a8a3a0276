"""CPU-only: the argument checks of the gated projections, the norms around a block and the checkpoints, in the
C ABI (before any device call) and in the binding."""

import ctypes

import pytest
import torch

import paper_2505_04846_amd as hpr

FAKE = 0x10000       # non-NULL, 16-byte aligned, never dereferenced on the host
FAKE_ODD = 0x10008   # misaligned
BIG = 1 << 44
INVALID, OUTSIDE, NO_WORKSPACE = 1, 4, 5


def _gated(call, **kw):
    a = dict(x=FAKE, x_exps=None, x_row=64, n=100, k=64, wg=FAKE, wu=FAKE, f=40, act=0, dtype=0, h=FAKE, dh=FAKE,
             dx=FAKE, dwg=FAKE, dwu=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    rows = [a[n] for n in ("x_row", "n", "k", "wg", "wu", "f", "act", "dtype")]
    if call == "fwd":
        return hpr.lib().gated_linear_fwd(a["x"], *rows, a["h"], None)
    return hpr.lib().gated_linear_bwd(a["dh"], a["x"], a["x_exps"], *rows, a["dx"], a["dwg"], a["dwu"], a["ws"],
                                      a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(dtype=2), INVALID), (dict(act=3), INVALID),
    (dict(act=-1), INVALID), (dict(k=0), OUTSIDE), (dict(k=12), OUTSIDE), (dict(k=65544), OUTSIDE),
    (dict(f=0), OUTSIDE), (dict(f=20), OUTSIDE), (dict(f=65544), OUTSIDE), (dict(x_row=60), OUTSIDE),
    (dict(x_row=-64), OUTSIDE), (dict(x_row=1 << 20), OUTSIDE), (dict(x=None), INVALID), (dict(wg=None), INVALID),
    (dict(wu=None), INVALID), (dict(x=FAKE_ODD), INVALID), (dict(wg=FAKE_ODD), INVALID),
    (dict(n=(1 << 31) - 1, f=65536), OUTSIDE),
])
def test_gated_rejects(kw, status):
    assert _gated("fwd", **kw) == status
    assert hpr.lib().hpr_last_error()
    assert _gated("bwd", **kw) == status


def test_gated_rejects_more():
    assert _gated("fwd", h=None) == INVALID and _gated("fwd", h=FAKE_ODD) == INVALID
    for kw in (dict(dh=None), dict(dh=FAKE_ODD), dict(dx=FAKE_ODD), dict(dwg=None), dict(dwu=None),
               dict(dwu=FAKE_ODD), dict(x_exps=FAKE_ODD)):
        assert _gated("bwd", **kw) == INVALID, kw
    assert _gated("bwd", ws=None) == NO_WORKSPACE and _gated("bwd", ws_bytes=100) == NO_WORKSPACE
    size = hpr.lib().gated_linear_bwd_workspace_size
    need = size(100, 64, 40, 0, 1, 1)
    assert _gated("bwd", ws_bytes=need - 1) == NO_WORKSPACE
    assert _gated("bwd", ws_bytes=size(100, 64, 40, 0, 1, 1), x_exps=FAKE) == NO_WORKSPACE  # the rows need a place
    # each half of the gradients needs no more than both, and nothing is asked for sizes that are refused
    assert size(100, 64, 40, 0, 1, 0) < need and size(100, 64, 40, 0, 0, 1) < need
    assert size(-1, 64, 40, 0, 1, 1) == 0 and size(100, 0, 40, 0, 1, 1) == 0 and size(100, 64, 70000, 0, 1, 1) == 0
    assert _gated("bwd", ws=FAKE_ODD) == INVALID and _norm("bwd", ws=FAKE_ODD) == INVALID
    # nothing to do
    assert _gated("fwd", n=0, x=None, h=None) == 0
    assert _gated("bwd", dx=None, dwg=None, dwu=None, ws=None, ws_bytes=0) == 0
    # the weights' gradients sum over rows in 32-bit offsets
    assert _gated("bwd", n=(1 << 21) + 1, ws_bytes=0) == OUTSIDE
    assert _gated("bwd", n=(1 << 21) + 1, ws_bytes=0, dwg=None, dwu=None) == NO_WORKSPACE
    # sizes do not wrap
    assert size((1 << 31) - 1, 65536, 65536, 1, 1, 1) > 1 << 48


def _desc(**kw):
    a = dict(n=100, x_row=64, b_row=64, dim=64, dtype=0, kind=1, gate_rows=0, scale=1.0, eps=1e-6)
    a.update({n: v for n, v in kw.items() if n in a})
    return hpr._NormDesc(*[a[n] for n, _ in hpr._NormDesc._fields_])


NORM = ("x", "b", "weight", "bias", "post_weight", "post_bias", "gate")


def _norm(call, **kw):
    a = {n: FAKE for n in NORM + ("r", "y", "dr", "dy", "dx", "db", "dweight", "dbias", "dpost_weight", "dpost_bias",
                                  "dgate", "ws")}
    a.update(x_exps=None, b_exps=None, ws_bytes=BIG)
    a.update({n: v for n, v in kw.items() if n in a})
    d = ctypes.byref(_desc(**kw))
    if call == "fwd":
        return hpr.lib().residual_norm_fwd(d, *[a[n] for n in NORM], a["r"], a["y"], None)
    return hpr.lib().residual_norm_bwd(
        d, a["dr"], a["dy"], a["x"], a["x_exps"], a["b"], a["b_exps"], a["weight"], a["post_weight"], a["post_bias"],
        a["gate"], a["dx"], a["db"], a["dweight"], a["dbias"], a["dpost_weight"], a["dpost_bias"], a["dgate"],
        a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(dtype=5), INVALID), (dict(kind=2), INVALID),
    (dict(gate_rows=2), INVALID), (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(dim=0), OUTSIDE), (dict(dim=20), OUTSIDE), (dict(dim=16392), OUTSIDE),
    (dict(x_row=4), OUTSIDE), (dict(b_row=-8), OUTSIDE), (dict(b_row=1 << 20), OUTSIDE), (dict(x=None), INVALID),
    (dict(b=None), INVALID), (dict(weight=None), INVALID), (dict(post_weight=None), INVALID),
    (dict(kind=0), INVALID), (dict(x=FAKE_ODD), INVALID), (dict(gate=FAKE_ODD), INVALID),
    (dict(n=1 << 26, dim=64), OUTSIDE), (dict(n=1 << 23, dim=8192), OUTSIDE),
])
def test_norm_rejects(kw, status):
    assert _norm("fwd", **kw) == status
    assert hpr.lib().hpr_last_error()
    assert _norm("bwd", **kw) == status


def test_norm_rejects_more():
    assert hpr.lib().residual_norm_fwd(None, *[FAKE] * 9, None) == INVALID
    assert hpr.lib().residual_norm_bwd_workspace_size(None) == 0
    # what there is no forward of has no gradient
    rms = dict(kind=0, bias=None, post_bias=None, dbias=None, dpost_bias=None)
    assert _norm("bwd", **dict(rms, dbias=FAKE)) == INVALID and _norm("bwd", **dict(rms, dpost_bias=FAKE)) == INVALID
    assert _norm("bwd", gate=None) == INVALID
    assert _norm("bwd", post_weight=None, post_bias=None, dpost_bias=None) == INVALID
    assert _norm("bwd", weight=None, dweight=None, dbias=None) == INVALID  # dy
    one = dict(b=None, post_weight=None, post_bias=None, gate=None, dpost_weight=None, dpost_bias=None, dgate=None)
    assert _norm("bwd", **one) == INVALID  # db
    # both rows in 8 bits, or neither
    assert _norm("bwd", x_exps=FAKE) == INVALID and _norm("bwd", b_exps=FAKE) == INVALID
    assert _norm("bwd", x_exps=FAKE_ODD, b_exps=FAKE) == INVALID
    assert _norm("bwd", ws_bytes=0) == NO_WORKSPACE and _norm("bwd", ws=None) == NO_WORKSPACE
    # (a checkpoint's rows are dense: the strides are not read)
    assert _norm("bwd", x_exps=FAKE, b_exps=FAKE, x_row=3, b_row=-1, ws_bytes=0) == NO_WORKSPACE
    # rows of 64 values go four to a workgroup of 256 threads: inside the limit of a launch
    assert _norm("bwd", n=(1 << 26) - 4, ws_bytes=0) == NO_WORKSPACE
    size = hpr.lib().residual_norm_bwd_workspace_size
    assert size(ctypes.byref(_desc(n=1 << 30))) == size(ctypes.byref(_desc(n=1 << 20)))
    # nothing to do
    assert _norm("fwd", n=0, x=None, b=None, r=None, y=None) == 0
    assert _norm("fwd", r=None, y=None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(dim=0), OUTSIDE), (dict(dim=12), OUTSIDE),
    (dict(dim=65544), OUTSIDE), (dict(dtype=2), INVALID), (dict(x=None), INVALID), (dict(codes=None), INVALID),
    (dict(exps=None), INVALID), (dict(x=FAKE_ODD), INVALID), (dict(codes=FAKE_ODD), INVALID),
    (dict(exps=FAKE_ODD), INVALID), (dict(n=1 << 30, dim=64), OUTSIDE), (dict(n=0, x=None), 0),
])
def test_checkpoint_rejects(kw, status):
    a = dict(x=FAKE, n=100, dim=64, dtype=0, codes=FAKE, exps=FAKE)
    a.update(kw)
    L = hpr.lib()
    assert L.checkpoint_pack(a["x"], 64, a["n"], a["dim"], a["dtype"], a["codes"], a["exps"], None) == status
    assert L.checkpoint_unpack(a["codes"], a["exps"], a["n"], a["dim"], a["dtype"], a["x"], None) == status


def test_checkpoint_stride():
    for row in (60, -64, 1 << 20):
        assert hpr.lib().checkpoint_pack(FAKE, row, 10, 64, 0, FAKE, FAKE, None) == OUTSIDE


def test_binding_rejects():
    """Wrong types and shapes, before any library call (CPU tensors are refused too)."""
    w = torch.zeros(16, 8, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        hpr.gated_linear_fwd(w, w.float(), w)
    with pytest.raises(ValueError, match="CUDA"):
        hpr.gated_linear_fwd(w, w, w)
    with pytest.raises(TypeError):
        hpr.checkpoint_pack(w.float())
    with pytest.raises(TypeError):
        hpr.checkpoint_pack([1.0])
    with pytest.raises(ValueError, match="CUDA"):
        hpr.checkpoint_pack(w)
    with pytest.raises(TypeError):
        hpr.checkpoint_unpack(w)
    with pytest.raises(ValueError, match="kind"):
        hpr.residual_norm_fwd(w, kind="batch")
    with pytest.raises(TypeError):
        hpr.residual_norm_fwd(w.float())
    with pytest.raises(TypeError, match="both"):
        hpr.residual_norm_bwd(w, w, w, hpr.Checkpoint(w, w, torch.bfloat16), w[0])
    with pytest.raises(ValueError, match="nothing to do"):
        hpr.residual_norm(w)
    with pytest.raises(ValueError, match="frozen"):
        hpr.residual_norm(w, w, w[0], scale=torch.ones((), requires_grad=True))
