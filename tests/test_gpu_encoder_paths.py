"""The encoder operators' kernels by size: every tile, plan and stage of work that a call's sizes choose,
against the fp64 oracle at its derived bounds (see test_gpu_encoder.py)."""

import numpy as np
import pytest
import torch

import paper_2505_04846_amd as hpr
from oracle import encoder as E
from test_gpu_encoder import (DEV, TYPES, adapter_case, adapter_oracle, attention_case,
                              attention_oracle, f64, gen, hold, off, rand)

pytestmark = pytest.mark.gpu

# (lens, k lens, room, H, Hk, D, type, causal, window): see test_gpu_encoder.ATTENTION
SIZES = {
    # tiles enough for a plan, short sequences; the gradients plan both of their kernels
    "planned_short": ([190, 0, 210] * 14, None, None, 32, 8, 128, "bf16", True, 0),
    "planned_short_both_ways": ([130, 257] * 12, None, None, 24, 24, 64, "f16", False, 0),
    # long sequences, whole and with a plan, a window inside them
    "long": ([2100, 2050], None, None, 32, 8, 32, "bf16", True, 0),
    "planned_long": ([2075] * 4, None, None, 32, 8, 16, "bf16", True, 300),
    # few rows a sequence, tiles enough for a plan
    "planned_few": ([3, 1, 0, 2] * 300, [40, 7, 5, 90] * 300, None, 8, 8, 64, "bf16", True, 0),
}


@pytest.mark.parametrize("name", sorted(SIZES))
def test_attention_by_size(name):
    case = SIZES[name]
    q, k, v, q_off, k_off, k_len, how, dout = attention_case(case, seed=400)
    want = attention_oracle(case, q, k, v, q_off, k_off, k_len, dout)
    r = hpr.packed_attention_fwd(q, k, v, q_off, **how)
    hold(r["out"], want["out"], want["bound"]["out"], "out")
    b = hpr.packed_attention_bwd(dout, q, k, v, r["out"], r["lse"], q_off, **how)
    for n in ("dq", "dk", "dv"):
        hold(b[n], want[n], want["bound"][n], n)


def test_planned_attention_graph_replays():
    case = SIZES["planned_short"]
    q, k, v, q_off, _, _, how, dout = attention_case(case, seed=401)

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
        # other lengths as well: the plan is made on the device
        q_off.copy_(off(np.roll(case[0], i)))
        q.copy_(rand(gen(410 + i), *q.shape, dtype=q.dtype))
        eager = [t.clone() for t in both()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


ADAPTER_SIZES = {
    # the large tile with its last round left to the middle one, the end of k inside a stage
    "large": ([1000, 3, 0, 1500, 1697], [1, 0, 0, 2, 1], 72, 4096, 16, 3, "bf16"),
    # one round of the large tile, ragged on both sides
    "large_ragged": ([2400, 77], [1, 0], 136, 4008, 8, 2, "f16"),
    "middle": ([700, 900, 500], [0, 1, -1], 136, 2048, 8, 2, "f16"),
    # more requests than one look covers inside a tile's rows, most of them empty
    "empty_requests": ([3] + [0] * 100 + [20] + [0] * 70 + [25], [i % 3 - 1 for i in range(173)], 72, 8192,
                       16, 2, "bf16"),
    "empty_requests_few": ([3] + [0] * 100 + [20] + [0] * 70 + [25], [i % 3 - 1 for i in range(173)], 136,
                           200, 20, 2, "f16"),
    # ranks over workgroups, past one block of 32
    "rank_128_few_rows": ([40, 3, 0, 90], [1, 0, 1, -1], 520, 264, 128, 2, "bf16"),
    # 64 rows a workgroup for h at ranks above 32
    "rank_64_many_rows": ([5000, 4000], [1, 0], 72, 64, 64, 2, "bf16"),
    "rank_40_many_rows": ([8300, 33], [0, 0], 64, 72, 40, 1, "f16"),
    # 1,024 rows a slot for dA and dB
    "long_slots": ([12000, 500], [0, 1], 64, 8192, 8, 2, "bf16"),
}


@pytest.mark.parametrize("name", sorted(ADAPTER_SIZES))
def test_adapters_by_size(name):
    case = ADAPTER_SIZES[name]
    t = adapter_case(case, seed=420)
    want = adapter_oracle(case, *t)
    f = hpr.adapter_linear_fwd(*t[:-1])
    hold(f["y"], want["y"], want["bound"]["y"], "y")
    b = hpr.adapter_linear_bwd(t[-1], *t[:-1], f["h"])
    for n in ("dx", "da", "db"):
        hold(b[n], want[n], want["bound"][n], n)


def test_adapter_graph_replays():
    t = adapter_case(([300, 5, 40], [0, 1, -1], 256, 384, 16, 2, "bf16"), seed=430)
    x, dy = t[0], t[-1]

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
        x.copy_(rand(gen(440 + i), *x.shape, dtype=x.dtype))
        t[-2].copy_(torch.tensor([i % 2, 1 - i % 2, -1], dtype=torch.int32))
        eager = [o.clone() for o in both()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


@pytest.mark.parametrize("ty", ["bf16", "f16"])
def test_rotary_larger_than_the_caches(ty):
    dt, u, tiny = TYPES[ty]
    n, H, Hk, D = 20000, 24, 8, 128
    x = torch.randn(n, H + Hk, D, device=DEV).to(dt)
    angle = torch.rand(300, D // 2, generator=gen(1), dtype=torch.float64) * 50
    cos, sin = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
    pos = torch.randint(0, 300, (n,), generator=gen(2), dtype=torch.int32).to(DEV)
    q, k = hpr.rotary_apply(x[:, :H], x[:, H:], pos, cos, sin)
    at = torch.randint(0, n, (300,), generator=gen(3)).to(DEV)
    at[0], at[1] = 0, n - 1
    src = f64(x[at])
    want = E.rotary(src, pos[at].cpu().numpy(), f64(cos), f64(sin))
    size = np.abs(src)
    size = np.concatenate([size[..., :D // 2] + size[..., D // 2:]] * 2, -1)
    hold(torch.cat([q, k], 1)[at], want, u * np.abs(want) + 4 * E.F32 * size + tiny, "rotary")
    # and every row by the rotation back
    bq, bk = hpr.rotary_apply(q, k, pos, cos, sin, inverse=True)
    back = torch.cat([bq, bk], 1).float() - x.float()
    assert back.abs().max().item() <= 6 * u * x.float().abs().max().item()
