"""Adapter gradients of calls of many requests, whose rows are ordered by adapter first: against the
fp64 oracle at its derived bounds (see test_gpu_encoder.py), and against the same rows in one request."""

import math
import random

import pytest
import torch

import paper_2505_04846_amd as hpr
from test_gpu_encoder import adapter_case, adapter_oracle, hold, off, rand, gen

pytestmark = pytest.mark.gpu

_rng = random.Random(5)
# rows per request, their adapters, k, m, rank, n_ad, type
CASES = {
    "one_row_each": ([1] * 3000, [i * 5 % 8 - 1 for i in range(3000)], 72, 136, 20, 7, "bf16"),
    "long_and_short": ([1000, 1, 0, 700, 3, 16, 17, 15, 64, 65] * 3,
                       [_rng.randrange(-1, 3) for _ in range(30)], 2056, 1544, 40, 3, "f16"),
    # more than one workgroup's adapters, more than one look's requests a wave, some adapters without a row
    "many_adapters": ([_rng.randrange(0, 4) for _ in range(3600)],
                      [_rng.randrange(-1, 602) for _ in range(3600)], 64, 72, 4, 600, "bf16"),
    "one_adapter": ([_rng.randrange(0, 60) for _ in range(90)], [0] * 90, 520, 264, 70, 1, "f16"),
    # 1,024 rows a slot
    "long_slots": ([311] * 40, [i % 2 for i in range(40)], 64, 8192, 8, 2, "bf16"),
    "nobody": ([5] * 40, [-1] * 40, 4096, 2048, 8, 3, "bf16"),
}


def ordered(case):
    """The rule of adapters.hip: parts of 12 MB and more that slots of single requests would add."""
    lens, _, k, m, r, n_ad, _ = case
    return (len(lens) - n_ad) * ((r + 15) // 16 * 16) * (k + m) * 4 >= 12 << 20


@pytest.mark.parametrize("name", sorted(CASES))
def test_parity(name):
    case = CASES[name]
    assert ordered(case)
    t = adapter_case(case, seed=500)
    want = adapter_oracle(case, *t)
    f = hpr.adapter_linear_fwd(*t[:-1])
    b = hpr.adapter_linear_bwd(t[-1], *t[:-1], f["h"])
    for n in ("dx", "da", "db"):
        hold(b[n], want[n], want["bound"][n], n)
    again = hpr.adapter_linear_bwd(t[-1], *t[:-1], f["h"])
    for n in ("dx", "da", "db"):
        assert torch.equal(again[n], b[n])
        one = hpr.adapter_linear_bwd(t[-1], *t[:-1], f["h"], need_dx=n == "dx", need_da=n == "da",
                                     need_db=n == "db")
        assert torch.equal(one[n], b[n])


def test_one_adapter_in_requests_or_in_one():
    """The same rows of one adapter: the same bits, however many requests hold them."""
    case = ([13, 0, 700, 1, 1, 90, 400] * 3, [0] * 21, 4096, 4096, 24, 1, "bf16")
    assert ordered(case)
    x, W, A, B, scale, o, ad, dy = adapter_case(case, seed=501)
    h = hpr.adapter_linear_fwd(x, W, A, B, scale, o, ad)["h"]
    many = hpr.adapter_linear_bwd(dy, x, W, A, B, scale, o, ad, h)
    one = hpr.adapter_linear_bwd(dy, x, W, A, B, scale, off([x.shape[0]]), ad[:1], h)
    assert all(torch.equal(many[n], one[n]) for n in ("da", "db"))


def test_adapters_do_not_touch():
    """Rows of NaN of one adapter, between those of another, leave the other's gradients."""
    case = ([3, 40, 5, 64, 70, 9], [0, 1, 0, 1, 0, 1], 8192, 4096, 72, 2, "bf16")
    assert ordered(case)
    t = adapter_case(case, seed=502)
    x, W, A, B, scale, o, ad, dy = t
    clean = hpr.adapter_linear_bwd(dy, *t[:-1], hpr.adapter_linear_fwd(*t[:-1])["h"])
    ends = o.tolist()
    for s in (1, 3, 5):
        x[ends[s]:ends[s + 1]] = math.nan
        dy[ends[s]:ends[s + 1]] = math.inf
    b = hpr.adapter_linear_bwd(dy, *t[:-1], hpr.adapter_linear_fwd(*t[:-1])["h"])
    assert torch.equal(b["da"][0], clean["da"][0]) and torch.equal(b["db"][0], clean["db"][0])
    assert not torch.isfinite(b["da"][1].float()).any()


def test_graph_replays():
    case = ([30, 5, 0, 200, 1, 64], [0, 1, -1, 1, 0, 0], 8192, 4096, 72, 2, "bf16")
    assert ordered(case)
    t = adapter_case(case, seed=503)
    x, o, ad, dy = t[0], t[-3], t[-2], t[-1]

    def both():
        f = hpr.adapter_linear_fwd(*t[:-1])
        b = hpr.adapter_linear_bwd(dy, *t[:-1], f["h"])
        return [f["y"], b["dx"], b["da"], b["db"]]

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        # other rows, lengths and adapters: the order is made on the device
        x.copy_(rand(gen(510 + i), *x.shape, dtype=x.dtype))
        o.copy_(off(case[0][i:] + case[0][:i]))
        ad.copy_(torch.tensor(case[1][2 * i:] + case[1][:2 * i], dtype=torch.int32))
        eager = [z.clone() for z in both()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
