"""GPU parity of the gated projections, the norms around a block and activations in 8 bits against the fp64
oracle, entry by entry, at bounds that the oracle derives from the roundings (oracle/block.py)."""

import math

import numpy as np
import pytest
import torch

import paper_2505_04846_amd as hpr
from oracle import block as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
# unit roundoff, half the spacing below the normal range, and the lowest step of a checkpoint
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 0.0, -126), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25, -24)}


def f64(t):
    return t.detach().cpu().double().numpy()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rand(g, *shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).to(DEV)


def hold(got, want, bound, what):
    if got.dtype is torch.float16:
        # a number from 65520 on is infinite in fp16: so is an exact one of which the bound leaves that much
        past = (np.abs(want) + bound >= 65520) & (f64(got) == np.where(want > 0, np.inf, -np.inf))
        got = torch.where(torch.from_numpy(past).to(got.device), torch.from_numpy(want).to(got.device), got.double())
    got = f64(got)
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), f"{what}: {over.max():.3e} past the bound at " \
        f"{np.unravel_index(over.argmax(), over.shape)}, {(over > 0).sum()} of {over.size}"


# ---- activations in 8 bits ------------------------------------------------------------------


def same_rows(got, want):
    return np.array_equal(f64(got), want, equal_nan=True)


@pytest.mark.parametrize("ty", ["bf16", "f16"])
@pytest.mark.parametrize("n,d", [(1, 8), (3, 32), (5, 40), (64, 768), (7, 1000), (33, 4096), (1000, 24), (0, 64)])
def test_checkpoint(ty, n, d):
    dt, _, _, least = TYPES[ty]
    g = gen(n * 7 + d)
    x = rand(g, n, d, dtype=torch.float32) * torch.exp(3 * rand(g, n, 1, dtype=torch.float32))
    x = x.to(dt)
    c = hpr.checkpoint_pack(x)
    codes, exps = B.checkpoint_pack(f64(x), least)
    assert (c.codes.cpu().numpy() == codes).all() and (c.exps.cpu().numpy() == exps).all()
    back = hpr.checkpoint_unpack(c)
    assert back.dtype is dt and same_rows(back, B.checkpoint_values(codes, exps))
    again = hpr.checkpoint_pack(back)
    assert torch.equal(again.codes, c.codes) and torch.equal(again.exps, c.exps)


@pytest.mark.parametrize("ty", ["bf16", "f16"])
def test_checkpoint_of_every_number(ty):
    """Every finite value of the type, in blocks with its neighbours and with far larger ones; and blocks with
    infinities and NaN, whose neighbours stay as they are."""
    dt, _, _, least = TYPES[ty]
    bits = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16)
    every = bits.view(dt)
    every = every[torch.isfinite(every.float())]
    every = every[:every.numel() // 32 * 32]
    mixed = every[torch.randperm(every.numel(), generator=gen(1))]
    x = torch.cat([every, mixed]).view(-1, 64).to(DEV)
    x[3, 5], x[7, 40], x[9, 0], x[9, 63] = math.inf, math.nan, -math.inf, math.nan
    c = hpr.checkpoint_pack(x)
    codes, exps = B.checkpoint_pack(f64(x), least)
    assert (c.exps.cpu().numpy() == exps).all() and (exps == 255).sum() == 4
    assert (c.codes.cpu().numpy() == codes).all()
    assert same_rows(hpr.checkpoint_unpack(c), B.checkpoint_values(codes, exps))


def test_checkpoint_of_columns_of_a_wider_tensor():
    x = rand(gen(3), 37, 200, dtype=torch.bfloat16)
    a, b = hpr.checkpoint_pack(x[:, 16:112]), hpr.checkpoint_pack(x[:, 16:112].contiguous())
    assert torch.equal(a.codes, b.codes) and torch.equal(a.exps, b.exps)


# ---- the gated projections ------------------------------------------------------------------

# rows, k, f, type, activation: one and few rows (32 by 16 and their tails), and each tile of the projections, of
# dx and of the weights' gradients on both sides of the rules that choose it
GATED = [
    (1, 8, 8, "bf16", "silu"), (1, 768, 2304, "f16", "gelu"), (7, 72, 40, "bf16", "gelu_tanh"),
    (31, 64, 16, "f16", "silu"), (32, 136, 24, "bf16", "gelu"), (33, 200, 8, "f16", "gelu_tanh"),
    (64, 1000, 72, "bf16", "silu"), (65, 64, 136, "bf16", "silu"), (100, 24, 1000, "f16", "silu"),
    (130, 72, 72, "bf16", "gelu"), (257, 520, 264, "f16", "gelu"), (300, 64, 1928, "bf16", "gelu_tanh"),
    (1100, 40, 1288, "bf16", "silu"), (1500, 72, 1032, "f16", "gelu_tanh"), (2309, 72, 2056, "bf16", "silu"),
    (2500, 136, 2000, "f16", "silu"), (6001, 1600, 64, "bf16", "gelu"), (9, 8, 5000, "bf16", "silu"),
    (515, 4104, 8, "bf16", "silu"), (40, 4096, 4104, "f16", "gelu"), (700, 1288, 3000, "bf16", "silu"),
    # few rows, odd columns, widths that end inside a stage
    (2, 72, 1000, "f16", "silu"), (32, 200, 3336, "bf16", "gelu"), (63, 1096, 520, "f16", "gelu_tanh"),
    (129, 72, 2504, "bf16", "silu"), (192, 264, 712, "f16", "silu"), (193, 264, 712, "f16", "silu"),
    # k split between workgroups: tiles of 128 rows, and of 256
    (449, 776, 2312, "f16", "gelu"), (1100, 2056, 8200, "bf16", "silu"),
    # large tiles whose stages of 64 rows of the weights end with the first matrix, and do not
    (900, 2048, 8256, "f16", "silu"), (2000, 4096, 1088, "bf16", "gelu"), (4200, 4104, 520, "f16", "silu"),
    # the weights' gradients with their rows split between workgroups, the two matrices' edge inside a tile
    (9001, 264, 328, "f16", "gelu"), (5003, 520, 136, "bf16", "silu"),
]


def gated_case(i):
    n, k, f, ty, act = GATED[i]
    dt = TYPES[ty][0]
    g = gen(100 + i)
    wide = rand(g, n, k + 24, dtype=dt)
    x = wide[:, 16:16 + k]  # columns of a wider tensor
    wg, wu = (rand(g, f, k, dtype=dt, std=1.5 * k ** -0.5) for _ in range(2))
    dh = rand(g, n, f, dtype=dt, std=0.3)
    dh[n // 2] = 0  # a row without a gradient
    return x, wg, wu, dh, act, ty


@pytest.mark.parametrize("i", range(len(GATED)))
def test_gated_parity(i):
    x, wg, wu, dh, act, ty = gated_case(i)
    want = B.gated_linear(f64(x), f64(wg), f64(wu), act, f64(dh), *TYPES[ty][1:3])
    h = hpr.gated_linear_fwd(x, wg, wu, act)["h"]
    g = hpr.gated_linear_bwd(dh, x, wg, wu, act)
    torch.cuda.synchronize()
    hold(h, want["h"], want["bound"]["h"], "h")
    for name in ("dx", "dw_gate", "dw_up"):
        hold(g[name], want[name], want["bound"][name], name)
    # one of them alone is the same, bit for bit, and so is a second call
    assert torch.equal(hpr.gated_linear_bwd(dh, x, wg, wu, act, need_dw=False)["dx"], g["dx"])
    w = hpr.gated_linear_bwd(dh, x, wg, wu, act, need_dx=False)
    assert w["dx"] is None and torch.equal(w["dw_gate"], g["dw_gate"]) and torch.equal(w["dw_up"], g["dw_up"])
    assert torch.equal(hpr.gated_linear_fwd(x, wg, wu, act)["h"], h)


@pytest.mark.parametrize("i", [2, 5, 8, 10, 12, 15])
def test_gated_gradients_from_a_checkpoint(i):
    x, wg, wu, dh, act, ty = gated_case(i)
    c = hpr.checkpoint_pack(x)
    rows = hpr.checkpoint_unpack(c)
    a = hpr.gated_linear_bwd(dh, c, wg, wu, act)
    b = hpr.gated_linear_bwd(dh, rows, wg, wu, act)
    for name in a:
        assert torch.equal(a[name], b[name]), name
    want = B.gated_linear(B.checkpoint_values(*B.checkpoint_pack(f64(x), TYPES[ty][3])), f64(wg), f64(wu), act,
                          f64(dh), *TYPES[ty][1:3])
    for name in a:
        hold(a[name], want[name], want["bound"][name], name)
    alone = hpr.gated_linear_bwd(dh, c, wg, wu, act, need_dw=False)
    assert torch.equal(alone["dx"], a["dx"])


@pytest.mark.parametrize("size", [1e-6, 3e-3, 3e4])
@pytest.mark.parametrize("i", [7, 8, 10])
def test_gated_gradients_of_any_size(i, size):
    """dh of a loss that is not scaled, or scaled far up; rows and columns of their own sizes among it."""
    x, wg, wu, dh, act, ty = gated_case(i)
    g = gen(i)
    n, f = dh.shape
    rows, cols = (2.0 ** torch.randint(-6, 1, s, generator=g).float().to(DEV) for s in ((n, 1), (1, f)))
    dh = (torch.randn(n, f, generator=g).clamp(-2, 2).to(DEV) * rows * cols * size).to(dh.dtype)
    wg, wu = wg * 0.25, wu * 0.25  # (dx and dw stay inside fp16)
    want = B.gated_linear(f64(x), f64(wg), f64(wu), act, f64(dh), *TYPES[ty][1:3])
    got = hpr.gated_linear_bwd(dh, x, wg, wu, act)
    for name in got:
        fine = np.abs(want[name]) < 6e4 if ty == "f16" else np.ones(want[name].shape, bool)
        over = np.abs(f64(got[name]) - want[name]) - want["bound"][name]
        assert (over[fine] <= 0).all(), (name, over[fine].max())


def test_gated_large_arguments():
    """Activations far into both tails."""
    for ty in TYPES:
        dt = TYPES[ty][0]
        for act in ("silu", "gelu", "gelu_tanh"):
            x = torch.zeros(40, 16, dtype=dt, device=DEV)
            x[:, 0] = torch.linspace(-200, 200, 40).to(dt)
            x[:, 1] = 1
            wg = torch.zeros(8, 16, dtype=dt, device=DEV)
            wu = torch.zeros(8, 16, dtype=dt, device=DEV)
            wg[:, 0] = 1
            wu[:, 1] = torch.linspace(-2, 2, 8).to(dt)
            dh = rand(gen(5), 40, 8, dtype=dt)
            want = B.gated_linear(f64(x), f64(wg), f64(wu), act, f64(dh), *TYPES[ty][1:3])
            got = {**hpr.gated_linear_fwd(x, wg, wu, act), **hpr.gated_linear_bwd(dh, x, wg, wu, act)}
            for name in got:
                hold(got[name], want[name], want["bound"][name], (ty, act, name))


@pytest.mark.parametrize("n", [20, 300, 2500])
def test_gated_rows_that_are_not_finite_stay_their_own(n):
    dt = torch.bfloat16
    g = gen(8)
    x, wg, wu, dh = rand(g, n, 72, dtype=dt), rand(g, 2000, 72, dtype=dt), rand(g, 2000, 72, dtype=dt), rand(
        g, n, 2000, dtype=dt)
    bad = x.clone()
    bad[n - 1] = math.nan
    bad[3, 1] = math.inf
    keep = [i for i in range(n) if i not in (3, n - 1)]
    a, b = hpr.gated_linear_fwd(x, wg, wu)["h"], hpr.gated_linear_fwd(bad, wg, wu)["h"]
    assert torch.equal(a[keep], b[keep]) and not torch.isfinite(b[[3, n - 1]]).all()
    a = hpr.gated_linear_bwd(dh, x, wg, wu, need_dw=False)["dx"]
    b = hpr.gated_linear_bwd(dh, bad, wg, wu, need_dw=False)["dx"]
    assert torch.equal(a[keep], b[keep])


def test_gated_without_rows():
    w = rand(gen(9), 24, 40, dtype=torch.float16)
    x, dh = torch.empty(0, 40, dtype=torch.float16, device=DEV), torch.empty(0, 24, dtype=torch.float16, device=DEV)
    assert hpr.gated_linear_fwd(x, w, w)["h"].shape == (0, 24)
    for rows in (x, hpr.checkpoint_pack(x)):
        g = hpr.gated_linear_bwd(dh, rows, w, w)
        assert g["dx"].shape == (0, 40) and not g["dw_gate"].any() and not g["dw_up"].any()


def test_gated_writes_its_output_alone():
    """Rows and columns around the outputs stay as they are."""
    for n, f in ((33, 40), (300, 264), (2309, 2056)):
        x, w = rand(gen(1), n, 64, dtype=torch.bfloat16), rand(gen(2), f, 64, dtype=torch.bfloat16)
        guard = torch.full((n + 600, f), 7.0, dtype=torch.bfloat16, device=DEV)
        hpr.gated_linear_fwd(x, w, w, out=guard[:n])
        assert (guard[n:] == 7).all()


# ---- norms around a block -------------------------------------------------------------------

# rows, d, type, kind, post, gate, bias, scale
NORM = [
    (1, 8, "bf16", "rms", True, "vector", False, 1.0), (1, 4096, "f16", "rms", True, "rows", False, 0.5),
    (3, 264, "bf16", "layer", True, "vector", True, 1.0), (5, 512, "f16", "rms", False, None, False, 1.0),
    (7, 520, "bf16", "rms", True, None, False, -0.75), (64, 768, "f16", "layer", False, None, True, 1.0),
    (65, 1000, "bf16", "layer", True, "rows", True, 0.25), (130, 1024, "f16", "rms", True, "vector", False, 1.0),
    (33, 1032, "bf16", "rms", False, "rows", False, 2.0), (9, 2048, "bf16", "layer", True, "vector", False, 1.0),
    (21, 2056, "f16", "layer", True, "rows", True, 1.0), (300, 4096, "bf16", "rms", True, "vector", False, 0.5),
    (6, 4104, "bf16", "rms", True, "vector", False, 1.0), (5, 8192, "f16", "layer", True, "vector", True, 1.0),
    (4, 8200, "bf16", "rms", True, "rows", False, 1.0), (3, 16384, "f16", "layer", True, "vector", True, 1.0),
    (5000, 16, "bf16", "layer", True, "vector", True, 1.0), (4099, 1024, "bf16", "rms", True, "vector", False, 1.0),
]


def norm_case(i, offset=0.2):
    n, d, ty, kind, post, gate, bias, scale = NORM[i]
    dt = TYPES[ty][0]
    g = gen(200 + i)
    x = rand(g, n, d + 8, dtype=dt, std=2.0, mean=offset)[:, 8:]
    b = rand(g, n, 2 * d, dtype=dt, std=0.7, mean=-offset)[:, :d]
    x[:, d // 2] *= 20  # a channel far larger than the others
    t = dict(weight=rand(g, d, dtype=dt, std=0.3, mean=1.0))
    if bias:
        t["bias"] = rand(g, d, dtype=dt, std=0.2)
    if post:
        t["post_weight"] = rand(g, d, dtype=dt, std=0.3, mean=1.0)
        if bias:
            t["post_bias"] = rand(g, d, dtype=dt, std=0.2)
    if gate:
        t["gate"] = rand(g, *((d,) if gate == "vector" else (n, d)), dtype=dt)
    how = dict(scale=scale, eps=1e-6 if kind == "rms" else 1e-5, kind=kind)
    dr, dy = rand(g, n, d, dtype=dt, std=0.3), rand(g, n, d, dtype=dt, std=0.3)
    return x, b, t, how, dr, dy, ty


def norm_oracle(x, b, t, how, dr, dy, ty):
    of = {name: f64(v) for name, v in t.items()}
    return B.residual_norm(x, b, **of, **how, dr=None if dr is None else f64(dr), dy=None if dy is None else f64(dy),
                           u=TYPES[ty][1], tiny=TYPES[ty][2])


@pytest.mark.parametrize("i", range(len(NORM)))
def test_norm_parity(i):
    x, b, t, how, dr, dy, ty = norm_case(i)
    want = norm_oracle(f64(x), f64(b), t, how, dr, dy, ty)
    f = hpr.residual_norm_fwd(x, b, **t, **how)
    g = hpr.residual_norm_bwd(dr, dy, x, b, **t, **how)
    torch.cuda.synchronize()
    for name in ("r", "y"):
        hold(f[name], want[name], want["bound"][name], name)
    for name, got in g.items():
        assert (got is None) == (name not in want), name
        if got is not None:
            hold(got, want[name], want["bound"][name], name)
    again = hpr.residual_norm_bwd(dr, dy, x, b, **t, **how)
    assert all(v is None or torch.equal(v, g[name]) for name, v in again.items())
    # every gradient alone is the same
    for need, names in (("need_dx", ["dx"]), ("need_db", ["db"]), ("need_dgate", ["dgate"]),
                        ("need_dw", ["dweight", "dbias", "dpost_weight", "dpost_bias"])):
        only = {"need_dx": False, "need_db": False, "need_dw": False, "need_dgate": False, need: True}
        one = hpr.residual_norm_bwd(dr, dy, x, b, **t, **how, **only)
        for name, v in one.items():
            assert (v is None) == (name not in names or g[name] is None)
            assert v is None or torch.equal(v, g[name])


@pytest.mark.parametrize("i", [0, 1, 2, 6, 8, 10, 11, 13, 14])
def test_norm_gradients_from_checkpoints(i):
    x, b, t, how, dr, dy, ty = norm_case(i)
    cx, cb = hpr.checkpoint_pack(x), hpr.checkpoint_pack(b)
    got = hpr.residual_norm_bwd(dr, dy, cx, cb, **t, **how)
    rows = hpr.residual_norm_bwd(dr, dy, hpr.checkpoint_unpack(cx), hpr.checkpoint_unpack(cb), **t, **how)
    least = TYPES[ty][3]
    want = norm_oracle(*(B.checkpoint_values(*B.checkpoint_pack(f64(v), least)) for v in (x, b)), t, how, dr, dy, ty)
    for name, v in got.items():
        if v is not None:  # (two kernels, which may contract products and sums in different places)
            hold(v, want[name], want["bound"][name], name)
            hold(rows[name], want[name], want["bound"][name], name)


@pytest.mark.parametrize("i", [2, 4, 5, 11, 13])
def test_norm_parts(i):
    """Without b (a norm alone), without weight (a residual sum alone), and with one of the two gradients."""
    x, b, t, how, dr, dy, ty = norm_case(i)
    pre = {name: t[name] for name in ("weight", "bias") if name in t}
    alone = dict(how, scale=1.0)
    want = norm_oracle(f64(x), None, pre, alone, dr, dy, ty)
    f = hpr.residual_norm_fwd(x, **pre, **alone)
    assert f["r"] is x
    hold(f["y"], want["y"], want["bound"]["y"], "y")
    g = hpr.residual_norm_bwd(dr, dy, x, **pre, **alone)
    for name in ("dx", "dweight") + ("dbias",) * ("bias" in t):
        hold(g[name], want[name], want["bound"][name], name)
    assert g["db"] is None and g["dgate"] is None and g["dpost_weight"] is None
    post = {name: v for name, v in t.items() if name not in pre}
    want = norm_oracle(f64(x), f64(b), post, how, dr, None, ty)
    f = hpr.residual_norm_fwd(x, b, **post, **how)
    assert f["y"] is None
    hold(f["r"], want["r"], want["bound"]["r"], "r")
    g = hpr.residual_norm_bwd(dr, None, x, b, **post, **how)
    assert torch.equal(g["dx"], dr)
    for name in ("dx", "db", "dpost_weight", "dpost_bias", "dgate"):
        if g[name] is not None:
            hold(g[name], want[name], want["bound"][name], name)
    for one, other in ((dr, None), (None, dy)):
        want = norm_oracle(f64(x), f64(b), t, how, one, other, ty)
        g = hpr.residual_norm_bwd(one, other, x, b, **t, **how)
        for name, v in g.items():
            if v is not None:
                hold(v, want[name], want["bound"][name], name)


def test_layer_norm_far_from_zero():
    """A mean 100 times the deviation: the squares of the values would lose it in 32 bits."""
    for i in (2, 5, 10, 13):
        x, b, t, how, dr, dy, ty = norm_case(i, offset=150.0)
        want = norm_oracle(f64(x), f64(b), t, how, dr, dy, ty)
        got = {**hpr.residual_norm_fwd(x, b, **t, **how), **hpr.residual_norm_bwd(dr, dy, x, b, **t, **how)}
        for name, v in got.items():
            if v is not None:
                hold(v, want[name], want["bound"][name], name)


def test_norm_of_rows_that_are_not_finite_stay_their_own():
    x, b, t, how, dr, dy, ty = norm_case(11)
    n = x.shape[0]
    bad, keep = x.clone(), [i for i in range(n) if i not in (4, n - 1)]
    bad[4, 7], bad[n - 1] = math.inf, math.nan
    a, c = hpr.residual_norm_fwd(x, b, **t, **how), hpr.residual_norm_fwd(bad, b, **t, **how)
    assert torch.equal(a["y"][keep], c["y"][keep]) and torch.equal(a["r"][keep], c["r"][keep])
    a, c = hpr.residual_norm_bwd(dr, dy, x, b, **t, **how), hpr.residual_norm_bwd(dr, dy, bad, b, **t, **how)
    assert torch.equal(a["dx"][keep], c["dx"][keep]) and torch.equal(a["db"][keep], c["db"][keep])
    # rows of zeros have a gradient: eps keeps them finite
    zero = torch.zeros_like(x.contiguous())
    g = hpr.residual_norm_bwd(dr, dy, zero, zero, **t, **how)
    assert all(torch.isfinite(v).all() for v in g.values() if v is not None)


def test_norm_without_rows():
    x = torch.empty(0, 72, dtype=torch.bfloat16, device=DEV)
    w = rand(gen(1), 72, dtype=torch.bfloat16)
    f = hpr.residual_norm_fwd(x, x, w, post_weight=w, gate=w)
    assert f["r"].shape == (0, 72) and f["y"].shape == (0, 72)
    g = hpr.residual_norm_bwd(x, x, x, x, w, post_weight=w, gate=w)
    assert not g["dweight"].any() and not g["dpost_weight"].any() and not g["dgate"].any()


# ---- graphs, streams, autograd --------------------------------------------------------------


def block_pass(x, b, wg, wu, t, how, dh, packed):
    """A run of them together: norm, projections, and the way back."""
    f = hpr.residual_norm_fwd(x, b, **t, **how)
    h = hpr.gated_linear_fwd(f["y"], wg, wu)["h"]
    rows = hpr.checkpoint_pack(f["y"]) if packed else f["y"]
    g = hpr.gated_linear_bwd(dh, rows, wg, wu)
    cx, cb = (hpr.checkpoint_pack(x), hpr.checkpoint_pack(b)) if packed else (x, b)
    back = hpr.residual_norm_bwd(f["r"], g["dx"], cx, cb, **t, **how)
    return [f["r"], f["y"], h, *g.values(), *(v for v in back.values() if v is not None)]


def block_inputs(ty, seed, n=333):
    dt = TYPES[ty][0]
    g = gen(seed)
    d, f = 264, 520
    t = dict(weight=rand(g, d, dtype=dt, std=0.3, mean=1.0), post_weight=rand(g, d, dtype=dt, std=0.3, mean=1.0),
             gate=rand(g, d, dtype=dt))
    return (rand(g, n, d, dtype=dt), rand(g, n, d, dtype=dt), rand(g, f, d, dtype=dt, std=d ** -0.5),
            rand(g, f, d, dtype=dt, std=d ** -0.5), t, dict(scale=0.5), rand(g, n, f, dtype=dt, std=0.1))


@pytest.mark.parametrize("ty", ["bf16", "f16"])
@pytest.mark.parametrize("packed", [False, True])
def test_block_in_a_graph(ty, packed):
    """Captured and replayed with new inputs, eager work between the replays."""
    args = block_inputs(ty, 1)
    block_pass(*args, packed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block_pass(*args, packed)
    for seed in range(2, 6):
        new = block_inputs(ty, seed)
        for to, frm in zip((*args[:4], *args[4].values(), args[6]), (*new[:4], *new[4].values(), new[6])):
            to.copy_(frm)
        want = block_pass(*new, packed)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_block_on_two_streams():
    """Two calls at a time, each on a stream of its own."""
    cases = [block_inputs("f16", s, n) for s, n in ((1, 700), (2, 45))]
    want = [block_pass(*c, True) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            got.append([block_pass(*c, True) for _ in range(3)])
    torch.cuda.synchronize()
    for runs, w in zip(got, want):
        for r in runs:
            assert all(torch.equal(a, b) for a, b in zip(r, w))


@pytest.mark.parametrize("checkpoint", [False, True])
def test_autograd(checkpoint):
    x, b, wg, wu, t, how, dh = block_inputs("bf16", 7)
    leaves = [v.requires_grad_() for v in (x, b, wg, wu, *t.values())]
    r, y = hpr.residual_norm(x, b, **t, **how, checkpoint=checkpoint)
    h = hpr.gated_linear(y, wg, wu, checkpoint=checkpoint)
    grads = torch.autograd.grad([r, h], leaves, [y.detach(), dh])
    with torch.no_grad():
        x, b, wg, wu = (v.detach() for v in (x, b, wg, wu))
        rows = hpr.checkpoint_pack(y) if checkpoint else y
        g = hpr.gated_linear_bwd(dh, rows, wg, wu)
        cx, cb = (hpr.checkpoint_pack(x), hpr.checkpoint_pack(b)) if checkpoint else (x, b)
        back = hpr.residual_norm_bwd(y, g["dx"], cx, cb, **t, **how)
    want = [back["dx"], back["db"], g["dw_gate"], g["dw_up"], back["dweight"], back["dpost_weight"], back["dgate"]]
    for a, c in zip(grads, want):
        assert torch.equal(a, c)


def test_autograd_by_differences():
    """A step along the gradient changes the loss by the gradient's square, to the rounding of the outputs."""
    x, b, wg, wu, t, how, dh = block_inputs("f16", 9, n=40)
    leaves = [v.requires_grad_() for v in (x, b, wg, wu, *t.values())]

    def loss():
        r, y = hpr.residual_norm(x, b, **t, **how)
        h = hpr.gated_linear(y, wg, wu)
        return (h.double() * dh.double()).sum() + (r.double() * 0.1).sum()

    grads = torch.autograd.grad(loss(), leaves)
    with torch.no_grad():
        before = [v.clone() for v in leaves]
        for v, keep, g in zip(leaves, before, grads):
            step = 0.05 / g.float().norm().item()
            moved = []
            for sign in (1, -1):
                v.copy_((keep.float() + sign * step * g.float()).to(v.dtype))
                moved.append((loss().item(), v.double().clone()))
            v.copy_(keep)
            (up, v_up), (down, v_down) = moved
            along = (g.double() * (v_up - v_down)).sum().item()
            # h and r are rounded to 2^-11 of themselves: about 40 x 520 of dh's 0.1 and 40 x 264 of 0.1, each at
            # random, twice; a straight line holds to the step's square
            noise = 2.0 ** -11 * 0.1 * (2 * (40 * 520 + 40 * 264)) ** 0.5
            assert abs((up - down) - along) <= 4 * noise + 0.02 * abs(along), (up - down, along)


def test_backward_in_a_graph():
    """A whole step through autograd, captured and replayed: leaves of its own, so that no eager graph holds them."""
    def step(args, packed):
        x, b, wg, wu, t, how, dh = args
        x, b, wg, wu, *t_leaves = (v.detach().requires_grad_() for v in (x, b, wg, wu, *t.values()))
        r, y = hpr.residual_norm(x, b, **dict(zip(t, t_leaves)), **how, checkpoint=packed)
        h = hpr.gated_linear(y, wg, wu, checkpoint=packed)
        return [r.detach(), h.detach(), *torch.autograd.grad([r, h], [x, b, wg, wu, *t_leaves], [b.detach(), dh])]

    for packed in (False, True):
        args = block_inputs("f16", 1, 150)
        step(args, packed)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(args, packed)
        for seed in (2, 3, 4):
            new = block_inputs("f16", seed, 150)
            for to, frm in zip((*args[:4], *args[4].values(), args[6]), (*new[:4], *new[4].values(), new[6])):
                to.copy_(frm)
            want = step(new, packed)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(out, want))


def test_two_threads():
    """Calls of two threads at once, each on its stream: no state is shared."""
    import threading
    cases = [block_inputs(ty, s, n) for ty, s, n in (("bf16", 3, 520), ("f16", 4, 61))]
    want = [block_pass(*c, False) for c in cases]
    torch.cuda.synchronize()
    same = [False, False]

    def run(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            runs = [block_pass(*cases[i], False) for _ in range(5)]
            torch.cuda.current_stream().synchronize()
        same[i] = all(torch.equal(a, b) for r in runs for a, b in zip(r, want[i]))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert same == [True, True]


def test_gated_workspace():
    """A workspace of the size that is asked for, or larger, with anything in it; one that is too small is not used."""
    for n, k, f, ty in ((20, 72, 264, "bf16"), (150, 200, 520, "f16"), (449, 776, 2312, "f16")):
        dt = TYPES[ty][0]
        g = gen(n)
        x, wg, wu, dh = (rand(g, *s, dtype=dt, std=0.3) for s in ((n, k), (f, k), (f, k), (n, f)))
        want = hpr.gated_linear_bwd(dh, x, wg, wu)
        need = hpr.lib().gated_linear_bwd_workspace_size(n, k, f, 0, 1, 1)
        for size in (need, need + 4096, need - 1, 16):
            ws = torch.full((size + 256,), 0xff, dtype=torch.uint8, device=DEV)
            got = hpr.gated_linear_bwd(dh, x, wg, wu, ws=ws[:size])
            assert all(torch.equal(got[name], v) for name, v in want.items())
            assert (ws[size:] == 0xff).all() and (size >= need or (ws == 0xff).all())
        odd = torch.full((2 * need + 512,), 0xff, dtype=torch.uint8, device=DEV)
        for ws in (odd[8:], odd[::2], odd.cpu()):  # not aligned, not dense, elsewhere: not used
            got = hpr.gated_linear_bwd(dh, x, wg, wu, ws=ws)
            assert all(torch.equal(got[name], v) for name, v in want.items()) and (odd == 0xff).all()


# ---- offsets past 32 bits -------------------------------------------------------------------


def far_rows(n):
    """Rows at the start, on both sides of the middle, and at the end."""
    return torch.cat([torch.arange(40), torch.arange(n // 2 - 40, n // 2 + 40), torch.arange(n - 90, n)])


@pytest.mark.parametrize("n,k,f,dw", [((1 << 20) + 300, 2056, 1032, True), ((1 << 28) + 5, 8, 8, False)])
def test_gated_far_rows(n, k, f, dw):
    """Rows, and d's, past 2^31 values; and so many rows of so few columns that small tiles are more than one launch
    holds.  Rows of dh between those that are looked at are 0: they add nothing to the weights' gradients."""
    dt, at = torch.bfloat16, far_rows(n).to(DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.empty(n, k, dtype=dt, device=DEV).normal_(generator=g)
    wg, wu = (rand(gen(s), f, k, dtype=dt, std=k ** -0.5) for s in (2, 3))
    dh = torch.zeros(n, f, dtype=dt, device=DEV)
    dh[at] = rand(gen(4), len(at), f, dtype=dt, std=0.3)
    want = B.gated_linear(f64(x[at]), f64(wg), f64(wu), "silu", f64(dh[at]), *TYPES["bf16"][1:3])
    hold(hpr.gated_linear_fwd(x, wg, wu)["h"][at], want["h"], want["bound"]["h"], "h")
    got = hpr.gated_linear_bwd(dh, x, wg, wu, need_dw=dw)
    hold(got["dx"][at], want["dx"], want["bound"]["dx"], "dx")
    assert torch.count_nonzero(got["dx"].abs().amax(1)) <= len(at)
    for name in ("dw_gate", "dw_up") if dw else ():
        hold(got[name], want[name], want["bound"][name], name)


@pytest.mark.parametrize("n", [5, 300])
def test_gated_far_columns(n):
    """Weights past 2^31 values.  Columns of dh between those that are looked at are 0."""
    k, f, dt = 40960, 65536, torch.bfloat16
    at = far_rows(f).to(DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    wg, wu = (torch.empty(f, k, dtype=dt, device=DEV).normal_(std=k ** -0.5, generator=g) for _ in range(2))
    x = rand(gen(1), n, k, dtype=dt)
    dh = torch.zeros(n, f, dtype=dt, device=DEV)
    dh[:, at] = rand(gen(2), n, len(at), dtype=dt, std=0.3)
    want = B.gated_linear(f64(x), f64(wg[at]), f64(wu[at]), "silu", f64(dh[:, at]), *TYPES["bf16"][1:3])
    hold(hpr.gated_linear_fwd(x, wg, wu)["h"][:, at], want["h"], want["bound"]["h"], "h")
    got = hpr.gated_linear_bwd(dh, x, wg, wu)
    hold(got["dx"], want["dx"], want["bound"]["dx"], "dx")
    for name in ("dw_gate", "dw_up"):
        hold(got[name][at], want[name], want["bound"][name], name)
        assert torch.count_nonzero(got[name].abs().amax(1)) <= len(at)


def test_norm_far_rows():
    n, d, dt = (1 << 20) + 300, 2056, torch.bfloat16
    at = far_rows(n).to(DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x, b = (torch.empty(n, d, dtype=dt, device=DEV).normal_(generator=g) for _ in range(2))
    t = dict(weight=rand(gen(2), d, dtype=dt, std=0.3, mean=1.0),
             post_weight=rand(gen(3), d, dtype=dt, std=0.3, mean=1.0), gate=rand(gen(4), d, dtype=dt))
    how = dict(scale=0.5, eps=1e-6, kind="rms")
    dr, dy = (torch.zeros(n, d, dtype=dt, device=DEV) for _ in range(2))
    dr[at], dy[at] = (rand(gen(s), len(at), d, dtype=dt, std=0.3) for s in (5, 6))
    want = norm_oracle(f64(x[at]), f64(b[at]), t, how, dr[at], dy[at], "bf16")
    f = hpr.residual_norm_fwd(x, b, **t, **how)
    for name in ("r", "y"):
        hold(f[name][at], want[name], want["bound"][name], name)
    del f
    got = hpr.residual_norm_bwd(dr, dy, x, b, **t, **how)
    for name, v in got.items():
        if v is not None:
            hold(v[at] if name in ("dx", "db") else v, want[name], want["bound"][name], name)
    del got
    c = hpr.checkpoint_pack(x)
    codes, exps = B.checkpoint_pack(f64(x[at]), -126)
    assert (c.codes[at].cpu().numpy() == codes).all() and (c.exps[at].cpu().numpy() == exps).all()
    assert same_rows(hpr.checkpoint_unpack(c)[at], B.checkpoint_values(codes, exps))
