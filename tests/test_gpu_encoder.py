"""GPU parity of the encoder's operators against the fp64 oracle, entry by entry, at bounds that the
oracle derives from the rounding of the 16-bit operands (oracle/encoder.py)."""

import math

import numpy as np
import pytest
import torch

import paper_2505_04846_amd as hpr
from oracle import encoder as E

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
# unit roundoff, and half the spacing below the normal range
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 0.0), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25)}


def f64(t):
    return t.detach().cpu().double().numpy()


def rand(gen, *shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen) * std).to(dtype).to(DEV)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def off(lens):
    return torch.tensor(np.cumsum([0] + list(lens)), dtype=torch.int64, device=DEV)


def hold(got, want, bound, what):
    got = f64(got)
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - want) - bound
    assert (over <= 0).all(), f"{what}: {over.max():.3e} past the bound at " \
        f"{np.unravel_index(over.argmax(), over.shape)}, {(over > 0).sum()} of {over.size}"


# ---- attention ------------------------------------------------------------------------------

EDGE = [1, 0, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 200]

# q lengths, k lengths (None: the same), room per sequence (None: none), H, Hk, D, type, causal, window
ATTENTION = [
    (EDGE, None, None, 8, 2, 128, "bf16", True, 0),
    (EDGE, None, None, 4, 4, 64, "f16", False, 0),
    (EDGE, None, None, 6, 2, 96, "bf16", True, 0),
    (EDGE, None, None, 7, 1, 64, "bf16", True, 37),
    (EDGE, None, None, 2, 2, 8, "f16", True, 0),
    (EDGE, None, None, 5, 1, 40, "bf16", False, 0),
    (EDGE, None, None, 2, 1, 120, "f16", True, 1),
    ([300, 5], None, None, 32, 1, 128, "f16", True, 0),
    ([64] * 3, None, None, 12, 12, 64, "bf16", False, 0),
    # more queries than keys (rows that see nothing), and fewer (a context before them)
    ([40, 130, 3, 70], [7, 64, 0, 300], None, 8, 2, 128, "bf16", True, 0),
    ([40, 130, 3, 70], [7, 64, 0, 300], None, 4, 2, 72, "f16", True, 20),
    ([40, 0, 3, 70], [7, 64, 0, 300], None, 4, 2, 64, "bf16", False, 0),
    # one token each over caches with spare room
    ([1] * 7, [1, 64, 65, 700, 0, 3, 1024], 1024, 8, 2, 128, "bf16", True, 0),
    ([1] * 5, [2, 500, 333, 1, 77], 512, 12, 12, 64, "f16", True, 100),
    ([1, 0, 2, 1], [900, 10, 40, 0], 1000, 6, 2, 80, "bf16", True, 0),
    # few rows over many keys: the keys are split over workgroups
    ([1], [5000], None, 8, 2, 128, "bf16", True, 0),
    ([3, 2], [4000, 2500], None, 4, 1, 64, "f16", True, 0),
    ([60], [3000], None, 8, 8, 128, "f16", False, 0),
    ([9], [2600], None, 4, 2, 128, "bf16", True, 700),
    ([1500], None, None, 2, 1, 128, "bf16", True, 0),
]


def attention_case(case, seed=0, strided=True, spread=1.0):
    q_lens, k_lens, room, H, Hk, D, ty, causal, window = case
    dt = TYPES[ty][0]
    g = gen(seed)
    same = k_lens is None
    k_lens = list(q_lens) if same else k_lens
    n_q, n_k = sum(q_lens), room * len(k_lens) if room else sum(k_lens)
    if strided and same:  # views of one projection's output, with columns of another use between
        x = rand(g, n_q, (H + 2 * Hk) * D + 16, dtype=dt)
        x[:, :H * D] *= spread
        q = x[:, :H * D].view(n_q, H, D) if n_q else x[:, :H * D].reshape(0, H, D)
        k = x[:, H * D + 8:(H + Hk) * D + 8].unflatten(1, (Hk, D))
        v = x[:, (H + Hk) * D + 16:].unflatten(1, (Hk, D))
    else:
        q = rand(g, n_q, H, D, dtype=dt, std=spread)
        # heads before rows in memory
        k = rand(g, Hk, n_k, D, dtype=dt).transpose(0, 1)
        v = rand(g, Hk, n_k, D, dtype=dt).transpose(0, 1)
    q_off = off(q_lens)
    k_off = off([room] * len(k_lens) if room else k_lens)
    k_len = torch.tensor(k_lens, dtype=torch.int64, device=DEV) if room else None
    if room:  # the room past each length holds anything
        for s, n in enumerate(k_lens):
            k[s * room + n:(s + 1) * room] = math.nan
            v[s * room + n:(s + 1) * room] = math.inf
    how = dict(k_off=None if same else k_off, k_len=k_len, causal=causal, window=window,
               scale=D ** -0.5)
    dout = rand(g, n_q, H, D, dtype=dt, std=0.5)
    return q, k, v, q_off, k_off, k_len, how, dout


def attention_oracle(case, q, k, v, q_off, k_off, k_len, dout):
    _, _, room, H, Hk, D, ty, causal, window = case
    u, tiny = TYPES[ty][1:]
    k64, v64 = f64(k), f64(v)
    return E.packed_attention(f64(q), np.where(np.isfinite(k64), k64, 0.0),
                              np.where(np.isfinite(v64), v64, 0.0), q_off.cpu().numpy(),
                              k_off.cpu().numpy(), None if k_len is None else k_len.cpu().numpy(),
                              causal, window, D ** -0.5, dout=f64(dout), u=u, tiny=tiny)


@pytest.mark.parametrize("i", range(len(ATTENTION)))
def test_attention_parity(i):
    case = ATTENTION[i]
    q, k, v, q_off, k_off, k_len, how, dout = attention_case(case, seed=i)
    want = attention_oracle(case, q, k, v, q_off, k_off, k_len, dout)
    r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
    b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
    torch.cuda.synchronize()
    hold(r["out"], want["out"], want["bound"]["out"], "out")
    lse = f64(r["lse"])
    empty = np.isneginf(want["lse"])
    assert (np.isneginf(lse) == empty).all()
    assert (np.abs(lse - want["lse"])[~empty] <= want["bound"]["lse"][~empty]).all()
    assert (f64(r["out"])[empty] == 0).all()
    for name in ("dq", "dk", "dv"):
        hold(b[name], want[name], want["bound"][name], name)
    assert (f64(b["dq"])[empty] == 0).all()
    if k_len is not None:  # gradients of the spare room are zero
        for s, n in enumerate(case[1]):
            room = slice(s * case[2] + n, (s + 1) * case[2])
            assert not b["dk"][room].any() and not b["dv"][room].any()


@pytest.mark.parametrize("ty", ["bf16", "f16"])
def test_attention_far_apart_scores(ty):
    """Scores of up to about 200: maxima that rise by far more than the deferred rescaling allows."""
    case = ([200, 70, 33], None, None, 4, 2, 64, ty, True, 0)
    q, k, v, q_off, k_off, k_len, how, dout = attention_case(case, seed=50, spread=40.0)
    want = attention_oracle(case, q, k, v, q_off, k_off, k_len, dout)
    assert np.abs(want["lse"]).max() > 100
    r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
    hold(r["out"], want["out"], want["bound"]["out"], "out")
    b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
    for name in ("dq", "dk", "dv"):
        hold(b[name], want[name], want["bound"][name], name)


def test_attention_rising_maximum():
    """Keys in the order of their scores, so that every tile raises the maximum."""
    n, D = 400, 64
    g = gen(3)
    v = rand(g, n, 1, D, dtype=torch.bfloat16)
    q = torch.ones(n, 1, D, dtype=torch.bfloat16, device=DEV)
    k = (torch.linspace(-8, 8, n)[:, None, None] * torch.ones(1, 1, D)).to(torch.bfloat16).to(DEV)
    o = off([n])
    want = E.packed_attention(f64(q), f64(k), f64(v), [0, n], [0, n], None, True, 0, 0.25,
                              u=2.0 ** -8)
    r = hpr.packed_attention_fwd(q, k, v, o, scale=0.25)
    hold(r["out"], want["out"], want["bound"]["out"], "out")


def test_attention_many_sequences():
    """More sequences than one step of the search for a workgroup's sequence covers."""
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 9, 5000)]
    case = (lens, None, None, 2, 1, 16, "bf16", True, 0)
    q, k, v, q_off, k_off, k_len, how, dout = attention_case(case, seed=51)
    want = attention_oracle(case, q, k, v, q_off, k_off, k_len, dout)
    r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
    b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
    hold(r["out"], want["out"], want["bound"]["out"], "out")
    for name in ("dq", "dk", "dv"):
        hold(b[name], want[name], want["bound"][name], name)


def test_attention_cache_past_32_bit_offsets():
    """The last sequences of a cache of 2.4e9 values per tensor."""
    Hk, D, room = 8, 128, 8192
    n_seq = 290
    k = torch.zeros(n_seq * room, Hk, D, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    lens = [0] * (n_seq - 2) + [777, 8192]
    g = gen(7)
    for s in (n_seq - 2, n_seq - 1):
        k[s * room:(s + 1) * room] = rand(g, room, Hk, D, dtype=torch.bfloat16)
        v[s * room:(s + 1) * room] = rand(g, room, Hk, D, dtype=torch.bfloat16)
    q = rand(g, n_seq, 16, D, dtype=torch.bfloat16)
    q_off = torch.arange(n_seq + 1, device=DEV)
    k_len = torch.tensor(lens, device=DEV)
    r = hpr.packed_attention_fwd(q, k, v, q_off, k_off=q_off * room, k_len=k_len)
    assert not r["out"][:n_seq - 2].any()
    kk, vv = f64(k[-2 * room:]), f64(v[-2 * room:])
    want = E.packed_attention(f64(q[-2:]), kk, vv, [0, 1, 2], [0, room, 2 * room], lens[-2:], True, 0,
                              D ** -0.5, u=2.0 ** -8)
    hold(r["out"][-2:], want["out"], want["bound"]["out"], "out")


def test_attention_sequences_do_not_touch():
    """A sequence of infinities and NaN leaves its neighbours as they were."""
    case = ([50, 40, 70], None, None, 4, 2, 64, "bf16", True, 0)
    q, k, v, q_off, _, _, how, dout = attention_case(case, seed=52)
    clean = hpr.packed_attention_fwd(q, k, v, q_off, **how)
    cb = hpr.packed_attention_bwd(dout, q, k, v, clean["out"], clean["lse"], q_off, **how)
    for x in (q, k, v):
        x[50:90] = math.nan
        x[60:70] = math.inf
    r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
    b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
    for s in (slice(0, 50), slice(90, 160)):
        assert torch.equal(r["out"][s], clean["out"][s]) and torch.equal(r["lse"][s], clean["lse"][s])
        for name in ("dq", "dk", "dv"):
            assert torch.equal(b[name][s], cb[name][s])


@pytest.mark.parametrize("ty", ["bf16", "f16"])
@pytest.mark.parametrize("q_lens,k_lens,H,Hk,D,window", [
    ([1] * 5, [2, 500, 333, 1, 77], 12, 12, 64, 50),     # a token each: few rows
    ([40, 3], [300, 64], 4, 2, 72, 20),
    ([130, 257], [401, 300], 8, 2, 128, 33),
    ([9], [2600], 4, 2, 128, 700),                       # the keys split over workgroups
    ([70], [5000], 2, 1, 64, 100),
])
def test_attention_keys_that_no_query_sees(ty, q_lens, k_lens, H, Hk, D, window):
    """Rows that every query's window has left behind may hold anything."""
    case = (q_lens, k_lens, None, H, Hk, D, ty, True, window)
    q, k, v, q_off, k_off, _, how, dout = attention_case(case, seed=54)

    def run():
        r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
        b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
        return [r["out"], r["lse"], b["dq"], b["dk"], b["dv"]]

    clean, gone, start = run(), [], 0
    for lq, lk in zip(q_lens, k_lens):
        gone += range(start, start + max(lk - lq - window + 1, 0))
        start += lk
    assert gone
    k[gone], v[gone] = math.inf, math.nan
    for x, y in zip(run(), clean):
        assert torch.equal(x, y)
    k[gone], v[gone] = math.nan, -math.inf
    for x, y in zip(run(), clean):
        assert torch.equal(x, y)
    assert not clean[3][gone].any() and not clean[4][gone].any()


@pytest.mark.parametrize("ty", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hk,D", [(8, 2, 128), (12, 12, 64), (4, 1, 40)])
def test_attention_gradient_of_one_visible_key(ty, H, Hk, D):
    """The first row of a causal sequence sees one key with probability 1: its dq is 0, up to fp32 sums,
    whatever the rounding of out."""
    case = ([1, 2, 17, 200, 64], None, None, H, Hk, D, ty, True, 0)
    q, k, v, q_off, _, _, how, dout = attention_case(case, seed=55)
    r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
    b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
    first = q_off[:-1].tolist()
    # |ds| <= (error of p and of two sums of D products) * sum |g v|, a hundred roundings of fp32 and more
    most = ((D + 100) * 2.0 ** -24 * np.abs(f64(dout)[first]).max() * np.abs(f64(v)[first]).max() * D
            * D ** -0.5 * np.abs(f64(k)[first]).max())
    assert np.abs(f64(b["dq"])[first]).max() <= most
    # ... and a sequence of one token gives no dk
    assert np.abs(f64(b["dk"])[first[0]]).max() <= most * (H // Hk) * max(
        1.0, np.abs(f64(q)[first]).max() / np.abs(f64(k)[first]).max())


def test_attention_bits_repeat_and_streams():
    case = ([300, 1, 77, 500], None, None, 8, 2, 128, "bf16", True, 0)
    q, k, v, q_off, _, _, how, dout = attention_case(case, seed=53)

    def both():
        r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
        b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
        return [r["out"], r["lse"], b["dq"], b["dk"], b["dv"]]

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, other))


def test_attention_graph_replays():
    """Forward (split keys, so both launches) and backward under a HIP graph, replayed with other
    inputs and eager work between."""
    case = ([3, 2], [2000, 1500], None, 8, 2, 128, "bf16", True, 0)
    q, k, v, q_off, _, _, how, dout = attention_case(case, seed=54)

    def both():
        r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
        b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
        return [r["out"], b["dq"], b["dk"], b["dv"]]

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        q.copy_(rand(gen(60 + i), *q.shape, dtype=q.dtype))
        eager = [t.clone() for t in both()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


def test_attention_autograd():
    case = ([70, 5], None, None, 4, 2, 64, "bf16", True, 0)
    q, k, v, q_off, k_off, k_len, how, dout = attention_case(case, seed=55)
    want = attention_oracle(case, q, k, v, q_off, k_off, k_len, dout)
    q, k, v = [t.detach().clone().requires_grad_() for t in (q, k, v)]
    out = hpr.packed_attention(q, k, v, q_off)
    out.backward(dout, retain_graph=True)
    for t, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        hold(t.grad, want[name], want["bound"][name], name)
    # a gradient of another layout, and only some inputs' gradients
    gk, = torch.autograd.grad(out, k, dout.transpose(0, 1).contiguous().transpose(0, 1))
    assert torch.equal(gk, k.grad)
    # keys shared between heads by broadcasting
    one = torch.randn(75, 1, 64, generator=gen(1)).to(torch.bfloat16).to(DEV).requires_grad_()
    o2 = hpr.packed_attention(q.detach(), one.expand(75, 2, 64), v.detach(), q_off)
    o2.backward(dout)
    full = one.detach().expand(75, 2, 64).contiguous()
    r = hpr.packed_attention_fwd(q.detach(), full, v.detach(), q_off)
    b = hpr.packed_attention_bwd(dout, q.detach(), full, v.detach(), r["out"], r["lse"], q_off)
    assert torch.equal(one.grad, b["dk"].sum(1, keepdim=True))


def test_attention_empty_calls():
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    none = torch.zeros(1, dtype=torch.int64, device=DEV)
    assert hpr.packed_attention_fwd(q, k, k, none)["out"].shape == (0, 4, 64)
    # queries without a key, and keys without a query
    q = torch.ones(5, 4, 64, dtype=torch.bfloat16, device=DEV)
    o5, o0 = off([5]), off([0])
    r = hpr.packed_attention_fwd(q, k, k, o5, k_off=o0)
    assert not r["out"].any() and torch.isneginf(r["lse"]).all()
    assert not hpr.packed_attention_bwd(q, q, k, k, r["out"], r["lse"], o5, k_off=o0)["dq"].any()
    k = torch.ones(5, 2, 64, dtype=torch.bfloat16, device=DEV)
    q = q[:0]
    r = hpr.packed_attention_fwd(q, k, k, o0, k_off=o5)
    b = hpr.packed_attention_bwd(q, q, k, k, r["out"], r["lse"], o0, k_off=o5)
    assert not b["dk"].any() and not b["dv"].any()


# ---- adapters -------------------------------------------------------------------------------

# rows per request, their adapters, k, m, rank, n_ad, type
ADAPTERS = [
    ([5, 0, 40, 1, 300], [1, 0, -1, 2, 0], 136, 200, 16, 3, "bf16"),
    ([1] * 32, list(range(16)) * 2, 512, 320, 16, 16, "bf16"),
    ([1], [0], 64, 8, 1, 1, "f16"),
    ([33, 64, 65], [0, 1, 0], 768, 2304, 8, 2, "f16"),
    ([700, 20], [1, 0], 264, 128, 64, 2, "bf16"),
    ([130], [0], 72, 520, 128, 1, "f16"),
    ([90, 90], [2, 1], 128, 256, 5, 4, "bf16"),
    ([17, 3, 50], [0, 7, -5], 96, 96, 33, 2, "bf16"),   # adapters out of range: none
    ([600, 0, 601], [0, 1, 1], 1000, 1016, 20, 2, "bf16"),
    ([1100, 1900], [0, 0], 128, 2048, 16, 1, "f16"),
    ([2] * 150, [i % 4 for i in range(150)], 200, 144, 4, 4, "f16"),
]


def adapter_case(case, seed=0):
    lens, adapter, k, m, r, n_ad, ty = case
    dt = TYPES[ty][0]
    g = gen(seed)
    n = sum(lens)
    x = rand(g, n, k, dtype=dt)
    W = rand(g, m, k, dtype=dt, std=k ** -0.5)
    A = rand(g, n_ad, r, k, dtype=dt, std=k ** -0.5)
    B = rand(g, n_ad, m, r, dtype=dt, std=0.3)
    scale = (0.5 + torch.rand(n_ad, generator=g)).to(DEV)
    dy = rand(g, n, m, dtype=dt, std=0.5)
    return x, W, A, B, scale, off(lens), torch.tensor(adapter, dtype=torch.int32, device=DEV), dy


def adapter_oracle(case, x, W, A, B, scale, o, adapter, dy):
    u, tiny = TYPES[case[-1]][1:]
    return E.adapter_linear(f64(x), f64(W), f64(A), f64(B), f64(scale), o.cpu().numpy(),
                            adapter.cpu().numpy(), f64(dy), u=u, tiny=tiny)


@pytest.mark.parametrize("i", range(len(ADAPTERS)))
def test_adapter_parity(i):
    t = adapter_case(ADAPTERS[i], seed=100 + i)
    want = adapter_oracle(ADAPTERS[i], *t)
    args, dy = t[:-1], t[-1]
    f = hpr.adapter_linear_fwd(*args)
    b = hpr.adapter_linear_bwd(dy, *args, f["h"])
    hold(f["y"], want["y"], want["bound"]["y"], "y")
    for name in ("dx", "da", "db"):
        hold(b[name], want[name], want["bound"][name], name)
    # each gradient alone is the same
    for name in ("dx", "da", "db"):
        one = hpr.adapter_linear_bwd(dy, *args, f["h"], need_dx=name == "dx", need_da=name == "da",
                                     need_db=name == "db")
        assert torch.equal(one[name], b[name])
        assert [n for n in one if one[n] is not None] == [name]


def test_adapter_no_requests_and_no_rows():
    t = adapter_case(([40], [0], 64, 48, 8, 2, "bf16"), seed=120)
    x, W, A, B, scale, _, _, dy = t
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    f = hpr.adapter_linear_fwd(x, W, A, B, scale, off([]), none)
    base = hpr.adapter_linear_fwd(x, W, A, B, scale, off([40]), none.new_tensor([-1]))
    assert torch.equal(f["y"], base["y"])
    b = hpr.adapter_linear_bwd(dy, x, W, A, B, scale, off([]), none, f["h"])
    assert not b["da"].any() and not b["db"].any() and b["dx"].any()
    f = hpr.adapter_linear_fwd(x[:0], W, A, B, scale, off([0]), none.new_tensor([1]))
    b = hpr.adapter_linear_bwd(dy[:0], x[:0], W, A, B, scale, off([0]), none.new_tensor([1]), f["h"])
    assert f["y"].shape == (0, 48) and not b["da"].any() and not b["db"].any()


def test_adapter_autograd_streams_and_bits():
    t = adapter_case(([70, 5, 300], [1, 0, 1], 256, 384, 16, 2, "bf16"), seed=121)
    want = adapter_oracle(([], [], 0, 0, 0, 0, "bf16"), *t)
    x, W, A, B, scale, o, ad, dy = t
    x, A, B = [z.requires_grad_() for z in (x, A, B)]
    y = hpr.adapter_linear(x, W, A, B, scale, o, ad)
    y.backward(dy)
    for z, name in ((x, "dx"), (A, "da"), (B, "db")):
        hold(z.grad, want[name], want["bound"][name], name)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f = hpr.adapter_linear_fwd(x.detach(), W, A.detach(), B.detach(), scale, o, ad)
        b = hpr.adapter_linear_bwd(dy, x.detach(), W, A.detach(), B.detach(), scale, o, ad, f["h"])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(f["y"], y) and torch.equal(b["dx"], x.grad)
    assert torch.equal(b["da"], A.grad) and torch.equal(b["db"], B.grad)
    with pytest.raises(ValueError, match="frozen"):
        hpr.adapter_linear(x, W.requires_grad_(), A, B, scale, o, ad)


def test_adapter_requests_do_not_touch():
    """A request of NaN rows, and an adapter of NaN, reach only their own outputs."""
    t = adapter_case(([50, 40, 70], [0, 1, 0], 128, 192, 8, 2, "bf16"), seed=122)
    x, W, A, B, scale, o, ad, dy = t
    clean = hpr.adapter_linear_fwd(*t[:-1])
    cb = hpr.adapter_linear_bwd(dy, *t[:-1], clean["h"])
    x[50:90] = math.nan
    dy[50:90] = math.nan
    A[1], B[1] = math.nan, math.inf
    f = hpr.adapter_linear_fwd(*t[:-1])
    b = hpr.adapter_linear_bwd(dy, *t[:-1], f["h"])
    for s in (slice(0, 50), slice(90, 160)):
        assert torch.equal(f["y"][s], clean["y"][s]) and torch.equal(b["dx"][s], cb["dx"][s])
    assert torch.equal(b["da"][0], cb["da"][0]) and torch.equal(b["db"][0], cb["db"][0])


# ---- rotary ---------------------------------------------------------------------------------


@pytest.mark.parametrize("n,H,Hk,D,rot,ty", [
    (1, 1, 0, 64, 64, "bf16"), (77, 8, 2, 128, 128, "bf16"), (301, 3, 1, 96, 48, "f16"),
    (64, 32, 8, 128, 64, "f16"), (5, 2, 2, 24, 16, "bf16"), (1000, 12, 12, 64, 64, "f16")])
def test_rotary_parity(n, H, Hk, D, rot, ty):
    dt, u, tiny = TYPES[ty]
    g = gen(200 + n)
    x = rand(g, n, H + Hk + 3, D, dtype=dt)
    q, k = x[:, 1:1 + H], x[:, 1 + H:1 + H + Hk] if Hk else None
    angle = torch.rand(50, rot // 2, generator=g, dtype=torch.float64) * 100
    cos, sin = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
    pos = torch.randint(0, 50, (n,), generator=g, dtype=torch.int32).to(DEV)
    for inverse in (False, True):
        out = hpr.rotary_apply(q, k, pos, cos, sin, inverse=inverse)
        for got, src in zip(out, (q, k)):
            if src is None:
                assert got is None
                continue
            want = E.rotary(f64(src), pos.cpu().numpy(), f64(cos), f64(sin), inverse)
            size = np.abs(f64(src))
            size = np.concatenate([size[..., :rot // 2] + size[..., rot // 2:rot]] * 2
                                  + [size[..., rot:]], -1)
            hold(got, want, u * np.abs(want) + 4 * E.F32 * size + tiny, "rotary")
            assert torch.equal(got[..., rot:], src[..., rot:])


def test_rotary_autograd_and_bad_positions():
    g = gen(210)
    x = rand(g, 40, 6, 64, dtype=torch.bfloat16)
    angle = torch.rand(16, 32, generator=g) * 6
    cos, sin = angle.cos().to(DEV), angle.sin().to(DEV)
    pos = torch.randint(0, 16, (40,), generator=g, dtype=torch.int32).to(DEV)
    q, k = x[:, :4].clone().requires_grad_(), x[:, 4:].clone().requires_grad_()
    gq, gk = rand(g, 40, 4, 64, dtype=torch.bfloat16), rand(g, 40, 2, 64, dtype=torch.bfloat16)
    a, b = hpr.rotary(q, k, pos, cos, sin)
    torch.autograd.backward((a, b), (gq, gk), retain_graph=True)
    wq, wk = hpr.rotary_apply(gq, gk, pos, cos, sin, inverse=True)
    assert torch.equal(q.grad, wq) and torch.equal(k.grad, wk)
    q.grad = k.grad = None
    b.backward(gk)
    assert torch.equal(k.grad, wk) and (q.grad is None or not q.grad.any())
    pos[3], pos[7] = -1, 16
    a, _ = hpr.rotary_apply(x[:, :4], None, pos, cos, sin)
    bad = torch.isnan(a.float()).all(-1).all(-1)
    assert bad.nonzero()[:, 0].tolist() == [3, 7] and torch.isfinite(a[~bad].float()).all()
