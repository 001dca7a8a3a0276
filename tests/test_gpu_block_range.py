"""GPU: the gated projections' gradients where g or u are far larger than what h shows of them."""

import numpy as np
import pytest
import torch

import paper_2505_04846_amd as hpr
from oracle import block as B
from test_gpu_block import DEV, TYPES, f64, gen, hold

pytestmark = pytest.mark.gpu


# a tile of each kind: up to 32 rows, 64 x 32, 128 x 64, 256 x 128
@pytest.mark.parametrize("n,f", [(5, 24), (40, 72), (300, 1928), (2309, 2056)])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("ty", ["bf16", "f16"])
@pytest.mark.parametrize("g,u", [(0.5, 80000.0), (0.5, 60000.0), (2.5, 57500.0), (60000.0, 0.5)])
def test_gradients_where_a_factor_is_large(n, f, act, ty, g, u):
    """g and u of one row as given in every 512th column: h is a number of fp16 (but for g = 2.5), dh ends just below a
    power of two, and the exact gradients are far inside the type.  Every term is positive, so that each output is
    off by an operand's rounding and its own, 2 u, and what 32 bits lose; in fp16 no operand that counts is below
    the normal range."""
    dt = TYPES[ty][0]
    x = torch.zeros(n, 16)
    x[:, 0] = x[:, 1] = 1
    x[3, 0], x[3, 1] = 250 * min(1.0, g / 250), 250
    wg, wu = torch.zeros(f, 16), torch.zeros(f, 16)
    wg[:, 0], wu[:, 1] = 0.5, u / 60000
    far = torch.arange(f) % 512 == 1
    wg[far, 0], wu[far, 1] = g / x[3, 0].item(), u / 250
    dh = (torch.rand(n, f, generator=gen(1)) + 0.5) * 2.0 ** -10
    dh[:, 1] = 1.9 * 2.0 ** -10
    x, wg, wu, dh = (t.to(dt).to(DEV) for t in (x, wg, wu, dh))
    want = B.gated_linear(f64(x), f64(wg), f64(wu), act, f64(dh), *TYPES[ty][1:3])
    got = hpr.gated_linear_bwd(dh, x, wg, wu, act)
    for name in got:
        hold(got[name], want[name], want["bound"][name], name)
        assert (np.abs(f64(got[name]) - want[name]) <= 2.1 * TYPES[ty][1] * np.abs(want[name])).all(), name


def test_gradients_that_are_parts_of_a_larger_buffer():
    """torch.cat's backward pass gives views that begin anywhere."""
    dt = torch.bfloat16
    x, b, wg, wu, w = (torch.randn(s, generator=gen(i)).to(dt).to(DEV).requires_grad_()
                       for i, s in enumerate([(9, 64), (9, 64), (40, 64), (40, 64), (64,)]))
    one = torch.ones(3, dtype=dt, device=DEV, requires_grad=True)

    def grads(join):
        r, y = hpr.residual_norm(x, b, w)
        h = hpr.gated_linear(y, wg, wu)
        out = join(r, h)
        weight = torch.linspace(-1, 1, r.numel() + h.numel(), device=DEV).to(dt)
        return torch.autograd.grad((out * weight).sum(), [x, b, wg, wu, w])

    want = grads(lambda *t: torch.cat([v.flatten() for v in t]))
    got = grads(lambda *t: torch.cat([one] + [v.flatten() for v in t])[3:])
    for a, c in zip(got, want):
        assert torch.equal(a, c)
