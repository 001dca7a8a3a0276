"""GPU: the block operators' kernels where a workgroup takes rows in turn, or a wave takes more of them at a time, than
small calls make it: the norm gradients past their number of workgroups, fp16's maxima and checkpoints of large calls."""

import numpy as np
import pytest
import torch

import paper_2505_04846_amd as hpr
from oracle import block as B
from test_gpu_block import DEV, TYPES, f64, gen, hold, norm_oracle, rand

pytestmark = pytest.mark.gpu

# rows, d, type, kind, post, gate, bias: past 1,024 workgroups of 4, 2 and 1 rows, or 512 of one, into a second or third
# turn that some workgroups have no row in, or some of their rows
TURNS = [
    (4101, 264, "bf16", "layer", True, "rows", True), (4099, 512, "f16", "rms", True, "vector", False),
    (2051, 768, "f16", "layer", True, "vector", True), (2049, 1000, "bf16", "layer", False, "rows", True),
    (1031, 1032, "f16", "rms", True, "rows", False), (1031, 2048, "bf16", "layer", True, "rows", True),
    (1100, 4096, "bf16", "rms", True, "rows", False), (1037, 4096, "f16", "layer", True, "vector", True),
    (521, 4104, "bf16", "layer", True, "rows", True), (1030, 8192, "f16", "rms", True, "vector", False),
    (521, 8200, "bf16", "layer", True, "rows", True), (515, 16384, "f16", "rms", True, "rows", False),
]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("i", range(len(TURNS)))
def test_norm_gradients_of_rows_in_turn(i, packed):
    n, d, ty, kind, post, gate, bias = TURNS[i]
    dt, _, _, least = TYPES[ty]
    g = gen(300 + i)
    x, b = rand(g, n, d, dtype=dt, std=2.0, mean=0.2), rand(g, n, d, dtype=dt, std=0.7, mean=-0.2)
    t = dict(weight=rand(g, d, dtype=dt, std=0.3, mean=1.0), gate=rand(g, *((d,) if gate == "vector" else (n, d)), dtype=dt))
    if bias:
        t["bias"] = rand(g, d, dtype=dt, std=0.2)
    if post:
        t["post_weight"] = rand(g, d, dtype=dt, std=0.3, mean=1.0)
        if bias:
            t["post_bias"] = rand(g, d, dtype=dt, std=0.2)
    how = dict(scale=0.5, eps=1e-5, kind=kind)
    dr, dy = rand(g, n, d, dtype=dt, std=0.3), rand(g, n, d, dtype=dt, std=0.3)
    vx, vb = f64(x), f64(b)
    if packed:
        vx, vb = (B.checkpoint_values(*B.checkpoint_pack(v, least)) for v in (vx, vb))
        x, b = hpr.checkpoint_pack(x), hpr.checkpoint_pack(b)
    # every row's own gradients
    want = norm_oracle(vx, vb, t, how, dr, dy, ty)
    got = hpr.residual_norm_bwd(dr, dy, x, b, **t, **how)
    for name in ("dx", "db") + ("dgate",) * (gate == "rows"):
        hold(got[name], want[name], want["bound"][name], name)
    # Sums over rows, of a few rows at the ends of the turns: one of them left out is far past the bound.  The others
    # add zeros.
    groups = 1024 if d <= 2048 else 512
    per = 4 if d <= 512 else 2 if d <= 1024 else 1
    at = sorted({0, 1, per * groups - 1, per * groups, n - 2, n - 1})
    others = torch.ones(n, dtype=torch.bool)
    others[at] = False
    dr[others], dy[others] = 0, 0
    few = {name: v[at] if name == "gate" and gate == "rows" else v for name, v in t.items()}
    want = norm_oracle(vx[at], vb[at], few, how, dr[at], dy[at], ty)
    got = hpr.residual_norm_bwd(dr, dy, x, b, **t, **how)
    for name, v in got.items():
        if v is None:
            continue
        if v.shape == (n, d):
            assert not v[others].any(), name
            v = v[at]
        hold(v, want[name], want["bound"][name], name)


def test_maxima_of_large_calls():
    """dh in fp16 with single values 2^22 times the rest of their row and column: a maximum that misses one makes it
    infinite, one that holds another row's or column's leaves nothing of the rest."""
    n, k, f, dt = 4201, 72, 8200, torch.float16
    g = gen(1)
    x, wg, wu = rand(g, n, k, dtype=dt), *(rand(g, f, k, dtype=dt, std=k ** -0.5) for _ in range(2))
    dh = rand(g, n, f, dtype=dt, std=2.0 ** -13)
    far = torch.randint(0, f, (n,), generator=g)
    spikes = torch.arange(n) % 2 == 0
    dh[spikes, far[spikes].to(DEV)] = 2.0 ** 9
    got = hpr.gated_linear_bwd(dh, x, wg, wu)
    # rows of every place among the 64 of a workgroup, and the last ones; columns likewise among 512
    rows = torch.cat([torch.arange(0, 64) * 65, torch.arange(n - 9, n)])
    cols = torch.cat([torch.arange(0, 16) * 513, far[:40][spikes[:40]], torch.arange(f - 9, f)]).unique()
    want = B.gated_linear(f64(x[rows]), f64(wg), f64(wu), "silu", f64(dh[rows]), *TYPES["f16"][1:3])
    hold(got["dx"][rows.to(DEV)], want["dx"], want["bound"]["dx"], "dx")
    at = cols.to(DEV)
    want = B.gated_linear(f64(x), f64(wg[at]), f64(wu[at]), "silu", f64(dh[:, at]), *TYPES["f16"][1:3])
    for name in ("dw_gate", "dw_up"):
        hold(got[name][at], want[name], want["bound"][name], name)


@pytest.mark.parametrize("ty", ["bf16", "f16"])
def test_checkpoint_of_large_calls(ty):
    """Four runs a wave, the last of them past the last row."""
    dt, _, _, least = TYPES[ty]
    x = torch.randn(20001, 1000, generator=gen(1)) * torch.exp(3 * torch.randn(20001, 1, generator=gen(2)))
    x = x.clamp(-60000, 60000).to(dt).to(DEV)
    c = hpr.checkpoint_pack(x)
    codes, exps = B.checkpoint_pack(f64(x), least)
    assert (c.codes.cpu().numpy() == codes).all() and (c.exps.cpu().numpy() == exps).all()
    assert np.array_equal(f64(hpr.checkpoint_unpack(c)), B.checkpoint_values(codes, exps))
