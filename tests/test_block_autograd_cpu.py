"""CPU-only: what the autograd functions of the gated projections and of the norms around a block do around their
kernels, which plain torch stands in for."""

import pytest
import torch

import paper_2505_04846_amd as hpr

NAMES = ("x", "b", "weight", "bias", "post_weight", "post_bias", "gate")


def _gated(x, wg, wu):
    return torch.nn.functional.silu(x @ wg.T) * (x @ wu.T)


def _norm(x, b, weight, bias, post_weight, post_bias, gate, scale=1.0, eps=1e-6, kind="rms"):
    def normed(v, w, c):
        if kind == "layer":
            v = v - v.mean(-1, keepdim=True)
        v = v / (v.square().mean(-1, keepdim=True) + eps).sqrt() * w
        return v if c is None else v + c

    p = b if post_weight is None or b is None else normed(b, post_weight, post_bias)
    r = x if b is None else x + scale * (p if gate is None else gate * p)
    return r, None if weight is None else normed(r, weight, bias)


@pytest.fixture
def plain(monkeypatch):
    """Nothing that these compute is seen by autograd.  A checkpoint is the rows rounded to halves."""
    asked = []

    def rows(t):
        return t.codes if isinstance(t, hpr.Checkpoint) else t

    def gated_fwd(x, wg, wu, act="silu"):
        return {"h": _gated(x, wg, wu)}

    def gated_bwd(dh, x, wg, wu, act="silu", need_dx=True, need_dw=True):
        asked.append((need_dx, need_dw))
        with torch.enable_grad():
            t = [v.detach().requires_grad_() for v in (rows(x), wg, wu)]
            g = torch.autograd.grad(_gated(*t), t, dh)
        return {"dx": g[0] if need_dx else None, "dw_gate": g[1] if need_dw else None,
                "dw_up": g[2] if need_dw else None}

    def norm_fwd(*args, **how):
        return dict(zip(("r", "y"), _norm(*args, **how)))

    def norm_bwd(dr, dy, *args, need_dx=True, need_db=True, need_dw=True, need_dgate=True, **how):
        asked.append((dr is not None, dy is not None))
        with torch.enable_grad():
            t = [None if v is None else rows(v).detach().requires_grad_() for v in args]
            out = [(o, d) for o, d in zip(_norm(*t, **how), (dr, dy)) if d is not None]
            leaves = [v for v in t if v is not None]
            g = iter(torch.autograd.grad([o for o, _ in out], leaves, [d for _, d in out], allow_unused=True))
        got = {"d" + n: None if v is None else next(g) for n, v in zip(NAMES, t)}
        need = {"dx": need_dx, "db": need_db, "dgate": need_dgate}
        return {n: v if need.get(n, need_dw) else None for n, v in got.items()}

    def pack(x):
        return hpr.Checkpoint((2 * x).round() / 2, x.new_zeros(1), x.dtype)

    for name, fn in (("gated_linear_fwd", gated_fwd), ("gated_linear_bwd", gated_bwd),
                     ("residual_norm_fwd", norm_fwd), ("residual_norm_bwd", norm_bwd), ("checkpoint_pack", pack)):
        monkeypatch.setattr(hpr, name, fn)
    return asked


def _tensors(*shapes, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g, dtype=torch.float64) for s in shapes]


def test_gated(plain):
    x, wg, wu, dh = _tensors((5, 4), (6, 4), (6, 4), (5, 6))
    for leaves in ([0], [1, 2], [2], [0, 1, 2]):
        t = [v.clone().requires_grad_(i in leaves) for i, v in enumerate((x, wg, wu))]
        got = torch.autograd.grad(hpr.gated_linear(*t), [t[i] for i in leaves], dh)
        want = torch.autograd.grad(_gated(*t), [t[i] for i in leaves], dh)
        assert all(torch.allclose(a, b) for a, b in zip(got, want))
        assert plain[-1] == (0 in leaves, 1 in leaves or 2 in leaves)


def test_gated_from_a_checkpoint(plain):
    x, wg, wu, dh = _tensors((5, 4), (6, 4), (6, 4), (5, 6))
    t = [v.requires_grad_() for v in (x, wg, wu)]
    h = hpr.gated_linear(*t, checkpoint=True)
    assert torch.equal(h, _gated(*t))  # the forward reads x itself
    # x itself is not kept
    assert not any(v.data_ptr() == x.data_ptr() for v in h.grad_fn.saved_tensors)
    got = torch.autograd.grad(h, t, dh)
    rough = [((2 * x).round() / 2).detach().requires_grad_(), wg, wu]
    want = torch.autograd.grad(_gated(*rough), rough, dh)
    assert all(torch.allclose(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("there", [NAMES, ("x", "b", "weight"), ("x", "weight"), ("x", "b", "gate"),
                                   ("x", "b", "weight", "post_weight", "gate")])
@pytest.mark.parametrize("checkpoint", [False, True])
def test_norm(plain, there, checkpoint):
    v = dict(zip(NAMES, _tensors((5, 8), (5, 8), 8, 8, 8, 8, 8)))
    t = {n: v[n].requires_grad_() if n in there else None for n in NAMES}
    kind = "layer" if "bias" in there else "rms"
    dr, dy = _tensors((5, 8), (5, 8), seed=1)
    r, y = hpr.residual_norm(**t, scale=0.5, kind=kind, checkpoint=checkpoint)
    if "b" not in there:
        assert r is t["x"]
    rough = {n: ((2 * t[n]).round() / 2).detach().requires_grad_() if checkpoint and n in "xb" and t[n] is not None
             else t[n] for n in NAMES}
    want_r, want_y = _norm(**rough, scale=0.5, kind=kind)
    outs = [(r, want_r, dr)] + ([(y, want_y, dy)] if y is not None else [])
    if "b" not in there:
        outs = outs[1:]
    leaves = [n for n in NAMES if n in there]
    got = torch.autograd.grad([o for o, _, _ in outs], [t[n] for n in leaves], [d for _, _, d in outs])
    want = torch.autograd.grad([o for _, o, _ in outs], [rough[n] for n in leaves], [d for _, _, d in outs])
    for n, a, b in zip(leaves, got, want):
        assert torch.allclose(a, b), n
    # one output alone: the other's gradient is not made up
    r, y = hpr.residual_norm(**t, scale=0.5, kind=kind)
    if y is not None and "b" in there:
        y.sum().backward()
        assert plain[-1] == (False, True)


def test_second_derivatives_raise(plain):
    x, wg, wu, b, w = _tensors((5, 4), (6, 4), (6, 4), (5, 4), 4)
    for t in (x, wg, wu, b, w):
        t.requires_grad_()
    for out in (hpr.gated_linear(x, wg, wu).sum(), hpr.residual_norm(x, b, w)[1].sum()):
        g = torch.autograd.grad(out, x, create_graph=True)[0]
        with pytest.raises(RuntimeError, match="second"):
            g.sum().backward()
    for out in (hpr.gated_linear(x, wg, wu, checkpoint=True).sum(),
                hpr.residual_norm(x, b, w, checkpoint=True)[1].sum()):
        with pytest.raises(RuntimeError, match="second"):
            torch.autograd.grad(out, x, create_graph=True)


def test_what_was_kept_must_not_change(plain):
    x, wg, wu = _tensors((5, 4), (6, 4), (6, 4))
    wg.requires_grad_()
    h = hpr.gated_linear(x, wg, wu)
    x.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        h.sum().backward()
