"""CPU-only pins of oracle/block.py: closed forms, central differences and brute force."""

import numpy as np
import pytest

from oracle import block as B

RNG = np.random.default_rng


def _differences(fn, inputs, grads, rng):
    """sum(fn * seed) against `grads` by central differences, every coordinate."""
    for name, x in inputs.items():
        for i in np.ndindex(x.shape):
            h = 1e-5
            keep = x[i]
            x[i] = keep + h
            up = fn()
            x[i] = keep - h
            down = fn()
            x[i] = keep
            assert abs((up - down) / (2 * h) - grads[name][i]) <= 1e-7 * (1 + abs(grads[name][i])), (name, i)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gated_gradients(act):
    rng = RNG(0)
    x, wg, wu = rng.normal(size=(3, 4)), rng.normal(size=(5, 4)), rng.normal(size=(5, 4))
    dh = rng.normal(size=(3, 5))
    r = B.gated_linear(x, wg, wu, act, dh)
    _differences(lambda: (B.gated_linear(x, wg, wu, act)["h"] * dh).sum(), {"x": x, "wg": wg, "wu": wu},
                 {"x": r["dx"], "wg": r["dw_gate"], "wu": r["dw_up"]}, rng)


def test_activations():
    g = np.array([-800.0, -5.0, -1.0, 0.0, 1.0, 5.0, 800.0])
    for act in ("silu", "gelu", "gelu_tanh"):
        a, slope = B.activation(act, g)[:2]
        assert np.isfinite(a).all() and np.isfinite(slope).all()
        assert a[3] == 0 and slope[3] == 0.5 and a[0] == 0 and slope[0] == 0 and a[6] == 800 and slope[6] == 1
        # x act(1) splits: act(g) - act(-g) = g
        assert np.allclose(a - B.activation(act, -g)[0], g, atol=1e-12)
    assert abs(B.activation("silu", np.array([1.0]))[0][0] - 0.7310585786300049) < 1e-15
    assert abs(B.activation("gelu", np.array([1.0]))[0][0] - 0.8413447460685429) < 1e-15
    assert abs(B.activation("gelu_tanh", np.array([1.0]))[0][0] - 0.8411919906082768) < 1e-15


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", [None, "vector", "rows"])
def test_norm_gradients(kind, post, gate):
    rng = RNG(1)
    n, d = 3, 6
    bias = kind == "layer"
    t = {"x": rng.normal(size=(n, d)) + 0.3, "b": rng.normal(size=(n, d)), "weight": rng.normal(size=d)}
    if bias:
        t["bias"] = rng.normal(size=d)
    if post:
        t["post_weight"] = rng.normal(size=d)
        if bias:
            t["post_bias"] = rng.normal(size=d)
    if gate:
        t["gate"] = rng.normal(size=d if gate == "vector" else (n, d))
    dr, dy = rng.normal(size=(n, d)), rng.normal(size=(n, d))
    how = dict(scale=0.7, eps=1e-3, kind=kind)

    def value():
        r = B.residual_norm(**t, **how)
        return (r["r"] * dr + r["y"] * dy).sum()

    g = B.residual_norm(**t, **how, dr=dr, dy=dy)
    _differences(value, t, {name: g["d" + name] for name in t}, rng)


def test_norm_closed_forms():
    x = np.array([[3.0, -3.0, 3.0, -3.0]])
    one = np.ones(4)
    assert np.allclose(B.residual_norm(x, weight=one, eps=1e-300)["y"], [[1, -1, 1, -1]])
    assert np.allclose(B.residual_norm(x + 100, weight=one, eps=1e-300, kind="layer")["y"], [[1, -1, 1, -1]])
    r = B.residual_norm(x, 2 * x, gate=0.5 * one, scale=3.0)
    assert np.allclose(r["r"], 4 * x) and "y" not in r
    # the gradient of a norm is orthogonal to its row, and a layer norm's sums to zero
    rng = RNG(2)
    v, dy = rng.normal(size=(2, 8)), rng.normal(size=(2, 8))
    g = B.residual_norm(v, weight=np.ones(8), eps=1e-300, dy=dy)["dx"]
    assert np.allclose((g * v).sum(1), 0)
    g = B.residual_norm(v, weight=np.ones(8), eps=1e-300, kind="layer", dy=dy)["dx"]
    assert np.allclose((g * v).sum(1), 0) and np.allclose(g.sum(1), 0)


def test_checkpoint():
    x = np.zeros((3, 40))
    x[0, :4] = [1.0, 0.5, 1 / 128, 1 / 64]      # 2^-6: 64, 32, ties to even 0.5 -> 0, 1
    x[0, 4:6] = [1.984375, -1.99]               # 127, and -127.36 -> -127
    x[0, 6] = 1.996                             # 127.7 -> 127, not 128
    x[1, 33] = -3e-9                            # below the least step of fp16
    x[2, 39] = np.inf
    codes, exps = B.checkpoint_pack(x, -24)
    assert list(codes[0, :7]) == [64, 32, 0, 1, 127, -127, 127]
    assert exps.tolist() == [[121, 103], [103, 103], [103, 255]] and not codes[1].any()
    v = B.checkpoint_values(codes, exps)
    assert np.isnan(v[2, 32:]).all() and (v[2, :32] == 0).all()
    assert v[0, 0] == 1.0 and v[0, 3] == 1 / 64
    rng = RNG(3)
    x = rng.normal(size=(50, 100)) * np.exp(rng.normal(size=(50, 1)) * 3)
    codes, exps = B.checkpoint_pack(x, -126)
    v = B.checkpoint_values(codes, exps)
    step = np.ldexp(1.0, np.repeat(exps.astype(int) - 127, 32, 1)[:, :100])
    assert (np.abs(v - x) <= np.where(np.abs(x) > 127.5 * step, step, step / 2)).all()
    again = B.checkpoint_pack(v, -126)  # packing the values again changes nothing
    assert (again[0] == codes).all() and (again[1] == exps).all()


def test_bounds_hold_for_fp32_and_are_not_loose():
    """The same formulas in fp32 stay inside the bounds, by no more than the bounds' own counting."""
    rng = RNG(4)
    x, wg, wu, dh = (rng.normal(size=s).astype(np.float32) for s in ((20, 64), (48, 64), (48, 64), (20, 48)))
    r = B.gated_linear(*(t.astype(float) for t in (x, wg, wu)), "silu", dh.astype(float), u=2.0 ** -11,
                       tiny=2.0 ** -25)
    g, v = x @ wg.T, x @ wu.T
    s = 1 / (1 + np.exp(-g))
    dg, du = dh * v * s * (1 + g * (1 - s)), dh * g * s
    for name, got in (("h", g * s * v), ("dx", dg @ wg + du @ wu), ("dw_gate", dg.T @ x), ("dw_up", du.T @ x)):
        assert (np.abs(got - r[name]) <= r["bound"][name]).all()
        wrong = got + 0.02 * np.abs(r[name]).mean()
        assert (np.abs(wrong - r[name]) > r["bound"][name]).mean() > 0.5
