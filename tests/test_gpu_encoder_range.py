"""fp16 gradients whose intermediate values lie below fp16's normal range, where the results do not: by
norm against the fp64 oracle.

The tolerance: every rounding of an operand is by at most u = 2^-11 of it, in no common direction, so
that a gradient, a sum of many such terms, is off by less than u of its norm from each of the roundings
(p or ds, the forward's output in delta; g or h), and 4 u hold all of them.  Added is what rounding the
exact result to fp16 takes, which is more than that where the result itself is small."""

import numpy as np
import pytest
import torch

import paper_2505_04846_amd as hpr
from oracle import encoder as E
from test_gpu_encoder import DEV, f64, gen, off

pytestmark = pytest.mark.gpu

U = 2.0 ** -11


def near(got, want, what):
    got = f64(got)
    assert np.isfinite(got).all(), f"{what}: not finite"
    size = np.linalg.norm(want)
    rounded = np.linalg.norm(want.astype(np.float16).astype(np.float64) - want)
    err = np.linalg.norm(got - want)
    assert size > 0 and err <= 4 * U * size + rounded, \
        f"{what}: off by {err / size:.2e} of the norm, rounding alone by {rounded / size:.2e}"


def half(t):
    return t.to(torch.float16).to(DEV)


# lengths, heads, kv heads, D, causal, window
SHAPES = {"both_ways": ([2048], 2, 1, 64, False, 0), "causal": ([900, 1500], 4, 2, 128, True, 0),
          "window": ([1700], 3, 1, 80, True, 600)}
# standard deviation of dout; with "rows" it doubles every 100 rows, and that of v, from 2^-8, every 160
# keys
DOUT = {"1e-3": (1e-3, False), "1e-4": (1e-4, False), "1e-5": (1e-5, False), "300": (300.0, False),
        "rows": (1e-5, True)}


@pytest.mark.parametrize("large", ["q", "k"])
@pytest.mark.parametrize("dout", DOUT)
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_gradients_of_any_size(shape, dout, large):
    """Large keys keep dq in the normal range, and large queries dk; the scores are the same."""
    lens, H, Hk, D, causal, window = SHAPES[shape]
    std, grows = DOUT[dout]
    g = gen(600)
    n = sum(lens)
    row = torch.arange(n, dtype=torch.float64)[:, None, None]
    up = 16.0 if large == "q" else 1 / 16
    q = half(torch.randn(n, H, D, generator=g, dtype=torch.float64) * up)
    k = half(torch.randn(n, Hk, D, generator=g, dtype=torch.float64) / up)
    v = half(torch.randn(n, Hk, D, generator=g, dtype=torch.float64)
             * (2 ** (row / 160 - 8) if grows else 1))
    do = half(torch.randn(n, H, D, generator=g, dtype=torch.float64)
              * (std * 2 ** (row / 100) if grows else std))
    o = off(lens)
    how = dict(causal=causal, window=window)
    r = hpr.packed_attention_fwd(q, k, v, o, **how)
    b = hpr.packed_attention_bwd(do, q, k, v, r["out"], r["lse"], o, **how)
    host = o.cpu().numpy()
    want = E.packed_attention(f64(q), f64(k), f64(v), host, host, None, causal, window, D ** -0.5,
                              dout=f64(do))
    for name in ("dq", "dk", "dv"):
        near(b[name], want[name], name)


@pytest.mark.parametrize("n_q,n,D", [(1, 8192, 128), (1, 300, 64), (200, 900, 64), (64, 2500, 96)])
def test_attention_beside_one_key_that_takes_most(n_q, n, D):
    """Probabilities of about 2^-24.4 beside one of almost 1, whose value is 0."""
    g = gen(602)
    q, k = [torch.randn(m, h, D, generator=g, dtype=torch.float64) * 0.1 for m, h in ((n_q, 4), (n, 2))]
    q[..., 0] = 16.0
    k[..., 0] = -16.9 * D ** 0.5 / 16.0
    k[0] = 0.0
    v = 50.0 + torch.randn(n, 2, D, generator=g, dtype=torch.float64)
    v[0] = 0.0
    q, k, v = half(q), half(k), half(v)
    q_off, k_off = off([n_q]), off([n])
    r = hpr.packed_attention_fwd(q, k, v, q_off, k_off=k_off, causal=False)
    want = E.packed_attention(f64(q), f64(k), f64(v), [0, n_q], [0, n], None, False, 0, D ** -0.5)
    assert 0 < np.abs(want["out"]).max() < 0.1
    near(r["out"], want["out"], "out")


def test_attention_gradients_of_keys_that_get_little_attention():
    """Keys whose probabilities are below 2^-22 in every row."""
    n, D = 1024, 64
    g = gen(601)
    q, k = [torch.randn(n, 1, D, generator=g, dtype=torch.float64) * 0.5 for _ in range(2)]
    q[..., 0] = 24.0
    k[..., 0] = 0.0
    far = torch.arange(n) % 2 == 1
    k[far, :, 0] = -3.0
    q, k = half(q), half(k)
    v = half(torch.randn(n, 1, D, generator=g, dtype=torch.float64))
    do = half(torch.randn(n, 1, D, generator=g, dtype=torch.float64) * 4096)
    o = off([n])
    r = hpr.packed_attention_fwd(q, k, v, o, causal=False)
    b = hpr.packed_attention_bwd(do, q, k, v, r["out"], r["lse"], o, causal=False)
    want = E.packed_attention(f64(q), f64(k), f64(v), [0, n], [0, n], None, False, 0, D ** -0.5,
                              dout=f64(do))
    far = far.numpy()
    for rows in (far, ~far):
        for name in ("dk", "dv"):
            near(b[name][torch.from_numpy(rows).to(DEV)], want[name][rows], name)
    near(b["dq"], want["dq"], "dq")


# rows per request, their adapters, k, m, rank, n_ad
ADAPTERS = {
    "one": ([2048], [0], 512, 1024, 16, 1),
    "rank_70": ([900, 300], [0, 1], 136, 520, 70, 2),
    "few_rows": ([60, 1, 3], [0, 1, 1], 4096, 768, 8, 2),
    # rows ordered by adapter (see test_gpu_adapter_order.py)
    "ordered": ([7] * 130, [i % 2 for i in range(130)], 1024, 1024, 33, 2),
}


# standard deviations of x, A, B and dy: g is about B dy sqrt(m), h about x A sqrt(k)
@pytest.mark.parametrize("stds", [(1.0, 0.03, 1e-3, 1e-4), (1.0, 0.03, 1e-4, 1e-4), (300.0, 0.03, 1e-4, 1e-5),
                                  (1e-4, 1e-3, 0.1, 30.0), (1e-3, 1e-4, 0.1, 30.0),
                                  (3.0, 0.3, 0.3, 3.0)],
                         ids=["B-3_dy-4", "B-4_dy-4", "B-4_dy-5", "x-4_A-3", "x-3_A-4", "large"])
@pytest.mark.parametrize("shape", ADAPTERS)
def test_adapter_gradients_of_any_size(shape, stds):
    lens, adapter, k, m, r, n_ad = ADAPTERS[shape]
    g = gen(610)
    n = sum(lens)
    x, A, B, dy = [half(torch.randn(*s, generator=g, dtype=torch.float64) * std)
                   for s, std in zip(((n, k), (n_ad, r, k), (n_ad, m, r), (n, m)), stds)]
    W = half(torch.randn(m, k, generator=g, dtype=torch.float64) * k ** -0.5)
    scale = (0.5 + torch.rand(n_ad, generator=g)).to(DEV)
    args = (x, W, A, B, scale, off(lens), torch.tensor(adapter, dtype=torch.int32, device=DEV))
    b = hpr.adapter_linear_bwd(dy, *args, hpr.adapter_linear_fwd(*args)["h"])
    want = E.adapter_linear(*[f64(t) for t in args[:5]], args[5].cpu().numpy(), adapter, f64(dy))
    for name in ("dx", "da", "db"):
        near(b[name], want[name], name)
    for i in range(n_ad):  # each adapter by itself, and each rank of it
        near(b["da"][i], want["da"][i], f"da[{i}]")
        near(b["db"][i, :, r - 1], want["db"][i, :, r - 1], f"db[{i}]")
