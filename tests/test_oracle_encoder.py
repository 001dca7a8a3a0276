"""CPU pins of the fp64 oracle of the encoder's operators: closed forms, invariants and central
differences for every gradient."""

import numpy as np
import pytest

from oracle import encoder as E


def _rand(seed, *shapes):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal(s) for s in shapes]


def _numeric(f, x, eps=1e-6):
    g = np.zeros_like(x)
    flat, out = x.reshape(-1), g.reshape(-1)
    for i in range(flat.size):
        keep = flat[i]
        flat[i] = keep + eps
        hi = f()
        flat[i] = keep - eps
        lo = f()
        flat[i] = keep
        out[i] = (hi - lo) / (2 * eps)
    return g


LAYOUTS = [
    ([5, 0, 3], [5, 0, 3], None, True, 0),
    ([5, 2], [5, 2], None, False, 0),
    ([4, 3], [2, 5], None, True, 0),      # rows that see nothing, and a context before the queries
    ([6], [6], None, True, 2),
    ([1, 1], [4, 4], [3, 0], True, 0),    # single tokens over a cache with room, one of them empty
]


@pytest.mark.parametrize("q_lens,k_lens,k_len,causal,window", LAYOUTS)
def test_attention_gradients_against_differences(q_lens, k_lens, k_len, causal, window):
    q_off, k_off = np.cumsum([0] + q_lens), np.cumsum([0] + k_lens)
    q, k, v, g = _rand(1, (q_off[-1], 4, 3), (k_off[-1], 2, 3), (k_off[-1], 2, 3), (q_off[-1], 4, 3))
    args = (q_off, k_off, k_len, causal, window, 0.7)
    r = E.packed_attention(q, k, v, *args, dout=g)

    def loss():
        return float((E.packed_attention(q, k, v, *args)["out"] * g).sum())

    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        assert np.abs(_numeric(loss, x) - r[name]).max() < 1e-8


def test_attention_closed_forms():
    q, k, v = _rand(2, (6, 2, 4), (6, 2, 4), (6, 2, 4))
    off = [0, 6]
    r = E.packed_attention(q, k, v, off, off, None, True, 0, 1.0)
    # the first token sees itself only; a window of one is the same for every token
    assert np.allclose(r["out"][0], v[0])
    assert np.allclose(E.packed_attention(q, k, v, off, off, None, True, 1, 1.0)["out"], v)
    # equal keys: the mean of the visible values
    same = np.broadcast_to(k[:1], k.shape)
    r = E.packed_attention(q, same, v, off, off, None, True, 0, 1.0)
    for i in range(6):
        assert np.allclose(r["out"][i], v[:i + 1].mean(0))
        assert np.allclose(r["lse"][i], (q[i] * k[0]).sum(-1) + np.log(i + 1))
    # two sequences packed are the two alone; the last token of a prompt is the token form
    r = E.packed_attention(q, k, v, off, off, None, True, 0, 1.0)["out"]
    two = E.packed_attention(q, k, v, [0, 2, 6], [0, 2, 6], None, True, 0, 1.0)["out"]
    assert np.allclose(two[:2], r[:2])
    assert np.allclose(E.packed_attention(q[5:], k, v, [0, 1], off, None, True, 0, 1.0)["out"][0], r[5])
    assert np.allclose(E.packed_attention(q[3:4], k, v, [0, 1], off, [4], True, 0, 1.0)["out"][0], r[3])
    # grouped heads are the ungrouped ones with repeated keys
    q4 = _rand(3, (6, 4, 4))[0]
    g = E.packed_attention(q4, k, v, off, off, None, True, 0, 1.0)["out"]
    full = E.packed_attention(q4, k.repeat(2, 1), v.repeat(2, 1), off, off, None, True, 0, 1.0)["out"]
    assert np.allclose(g, full)


def test_attention_rows_that_see_nothing():
    q, k, v, g = _rand(4, (5, 1, 3), (2, 1, 3), (2, 1, 3), (5, 1, 3))
    r = E.packed_attention(q, k, v, [0, 5], [0, 2], None, True, 0, 1.0, dout=g)
    assert (r["out"][:3] == 0).all() and (r["lse"][:3] == -np.inf).all() and (r["dq"][:3] == 0).all()
    assert np.isfinite(r["lse"][3:]).all()


def test_adapter_gradients_against_differences():
    n, k, m, rank = 7, 5, 4, 2
    x, W, A, B, dy = _rand(5, (n, k), (m, k), (3, rank, k), (3, m, rank), (n, m))
    scale = np.array([0.5, 1.5, 2.0])
    off, adapter = [0, 2, 2, 5, 7], [2, 1, 0, -1]
    r = E.adapter_linear(x, W, A, B, scale, off, adapter, dy)

    def loss():
        return float((E.adapter_linear(x, W, A, B, scale, off, adapter)["y"] * dy).sum())

    for name, t in (("dx", x), ("da", A), ("db", B)):
        assert np.abs(_numeric(loss, t) - r[name]).max() < 1e-8
    assert (r["da"][1] == 0).all() and (r["db"][1] == 0).all()  # its only request has no row
    full = x[:2] @ (W + 2.0 * B[2] @ A[2]).T
    assert np.allclose(r["y"][:2], full) and np.allclose(r["y"][5:], x[5:] @ W.T)


def test_rotary_closed_forms():
    x, = _rand(6, (3, 2, 10))
    angle = np.array([[0.0, 0.0], [0.3, 1.1], [2.0, -0.4]])
    cos, sin = np.cos(angle), np.sin(angle)
    pos = np.array([0, 2, 1])
    y = E.rotary(x, pos, cos, sin)
    assert np.allclose(y[0], x[0]) and np.allclose(y[..., 4:], x[..., 4:])
    z = (x[1, :, :2] + 1j * x[1, :, 2:4]) * np.exp(1j * angle[2])
    assert np.allclose(y[1, :, :2], z.real) and np.allclose(y[1, :, 2:4], z.imag)
    assert np.allclose(E.rotary(y, pos, cos, sin, inverse=True), x)
    # the gradient is the rotation back
    g, = _rand(7, x.shape)
    num = _numeric(lambda: float((E.rotary(x, pos, cos, sin) * g).sum()), x)
    assert np.abs(num - E.rotary(g, pos, cos, sin, inverse=True)).max() < 1e-8


def test_bounds_hold_for_rounded_operands_and_reject_mistakes():
    """The bounds accept a computation with operands rounded to bf16, and reject a key left out."""
    def bf16(a):
        b = np.asarray(a, np.float32).view(np.uint32)
        return ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).view(np.float32).astype(np.float64)

    q, k, v = [bf16(a) for a in _rand(8, (40, 1, 16), (40, 1, 16), (40, 1, 16))]
    off = [0, 40]
    r = E.packed_attention(q, k, v, off, off, None, True, 0, 0.25, u=2.0 ** -8)
    see = E.visible(40, 40, True, 0)

    def rounded(see):
        x = np.where(see, 0.25 * (q[:, 0] @ k[:, 0].T), -np.inf)
        e = np.exp(x - x.max(1, keepdims=True))
        return bf16((bf16(e) @ v[:, 0]) / e.sum(1, keepdims=True))

    assert (np.abs(rounded(see) - r["out"][:, 0]) <= r["bound"]["out"][:, 0]).all()
    wrong = see.copy()
    wrong[30, 7] = False
    assert (np.abs(rounded(wrong) - r["out"][:, 0]) > r["bound"]["out"][:, 0]).any()
