"""Strides of dimensions that are never stepped over: one row, or one head."""

import pytest
import torch

import paper_2505_04846_amd as hpr


class _OnCard(torch.Tensor):
    """A host tensor that says it is on the card, for the binding's checks alone."""
    is_cuda = True


@pytest.mark.parametrize("shape,stride,want", [
    ((1, 4, 64), (1 << 23, 128, 1), (0, 128)),      # one row of a long projection's output
    ((100, 1, 64), (64, 1 << 23, 1), (64, 0)),      # one head of a cache with its heads first
    ((1, 1, 64), (12, 20, 1), (0, 0)),
    ((2, 2, 64), (256, 64, 1), (256, 64)),
    ((0, 2, 64), (1 << 23, 64, 1), (0, 64)),
])
def test_strides_that_count(shape, stride, want):
    base = torch.zeros(1 << 16, dtype=torch.bfloat16)
    t = base.as_strided(shape, stride).as_subclass(_OnCard)
    assert hpr._need_heads(t, "q", torch.bfloat16, t.device) == want


def _on_gpu(*shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.bfloat16).to("cuda:0")


def _dense(t):
    return torch.empty(t.shape, dtype=t.dtype, device=t.device).copy_(t)


@pytest.mark.gpu
def test_one_row_of_a_long_projection():
    """The last token of one sequence, its keys in the projection's output: a row stride past 2^22."""
    T, H, D = 400, 32, 128
    qkv = _on_gpu(1, T, 3, H, D, seed=1)
    q, k, v = qkv[:, -1, 0], qkv[0, :, 1], qkv[0, :, 2]
    assert q.stride(0) >= 1 << 22
    one, all_keys = [torch.tensor([0, n], device="cuda:0") for n in (1, T)]
    got, want = [hpr.packed_attention_fwd(x, k, v, one, k_off=all_keys) for x in (q, _dense(q))]
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    got, want = [hpr.packed_attention_bwd(got["out"], x, k, v, want["out"], want["lse"], one,
                                          k_off=all_keys) for x in (q, _dense(q))]
    assert all(torch.equal(got[n], want[n]) for n in ("dq", "dk", "dv"))


@pytest.mark.gpu
def test_one_head_of_a_cache_with_its_heads_first():
    n, D = 1 << 15, 128
    cache = _on_gpu(2, 1, n, D, seed=2)
    k, v = cache.transpose(1, 2)
    assert k.stride(1) >= 1 << 22
    q = _on_gpu(3, 4, D, seed=3)
    q_off, k_off = [torch.tensor([0, m], device="cuda:0") for m in (3, n)]
    got, want = [hpr.packed_attention_fwd(q, *kv, q_off, k_off=k_off)
                 for kv in ((k, v), (_dense(k), _dense(v)))]
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
