"""CPU-only: gradients that autograd hands over as parts of a larger buffer reach the kernels dense and at multiples of 16
bytes, which the library asks for.  Plain torch stands in for the kernels."""

import pytest
import torch

import paper_2505_04846_amd as hpr
from test_block_autograd_cpu import _gated, _norm, _tensors, plain  # noqa: F401


def _parts(*outs):
    """The outputs in one row, an odd number of values past its start, and as columns of a wider tensor: the backward
    passes of torch.cat give views."""
    first = outs[0].new_zeros(1, requires_grad=True)
    row = torch.cat([first] + [o.flatten() for o in outs])
    wide = torch.cat([o.new_zeros(o.shape[0], 1) for o in outs] + list(outs), 1)
    weight = torch.linspace(-1, 1, row.numel(), dtype=row.dtype)
    return (row * weight).sum(), (wide * wide.detach().cos()).sum()


def _watch(monkeypatch, name, count):
    run, seen = getattr(hpr, name), []

    def aligned(*args, **how):
        for t in args[:count]:
            assert t is None or (t.is_contiguous() and t.data_ptr() % 16 == 0), name
            seen.append(t)
        return run(*args, **how)

    monkeypatch.setattr(hpr, name, aligned)
    return seen


@pytest.mark.parametrize("loss", [0, 1])
def test_block(plain, monkeypatch, loss):  # noqa: F811
    x, wg, wu, b, w = (t.requires_grad_() for t in _tensors((5, 4), (6, 4), (6, 4), (5, 4), 4))
    seen = _watch(monkeypatch, "gated_linear_bwd", 1), _watch(monkeypatch, "residual_norm_bwd", 2)
    got = torch.autograd.grad(_parts(hpr.gated_linear(x, wg, wu))[loss], [x, wg, wu])
    want = torch.autograd.grad(_parts(_gated(x, wg, wu))[loss], [x, wg, wu])
    assert all(torch.allclose(a, c) for a, c in zip(got, want))
    got = torch.autograd.grad(_parts(*hpr.residual_norm(x, b, w))[loss], [x, b, w])
    want = torch.autograd.grad(_parts(*_norm(x, b, w, None, None, None, None))[loss], [x, b, w])
    assert all(torch.allclose(a, c) for a, c in zip(got, want))
    assert all(seen)


@pytest.mark.parametrize("loss", [0, 1])
def test_encoder(monkeypatch, loss):
    """The attention's, the adapters' and the rotation's."""
    q, x = (t.requires_grad_() for t in _tensors((6, 2, 3), (6, 6), seed=2))
    off = torch.tensor([0, 6])
    monkeypatch.setattr(hpr, "packed_attention_fwd", lambda q, *a, **how: {"out": 2 * q, "lse": q.new_zeros(6, 2)})
    monkeypatch.setattr(hpr, "packed_attention_bwd", lambda d, q, k, v, *a, **how: {
        "dq": 2 * d, "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)})
    monkeypatch.setattr(hpr, "adapter_linear_fwd", lambda x, *a: {"y": 3 * x, "h": x})
    monkeypatch.setattr(hpr, "adapter_linear_bwd", lambda d, *a, **how: {"dx": 3 * d, "da": None, "db": None})

    def turn(q, k, pos, cos, sin, inverse=False):
        return (-q if inverse else q * -1), None if k is None else -k

    monkeypatch.setattr(hpr, "rotary_apply", turn)
    seen = [_watch(monkeypatch, name, 1) for name in ("packed_attention_bwd", "adapter_linear_bwd", "rotary_apply")]
    runs = [(hpr.packed_attention(q, q, q, off).flatten(1), q, 2.0),
            (hpr.adapter_linear(x, x.detach(), x.detach()[None], x.detach()[None], torch.ones(1), off, off), x, 3.0),
            (hpr.rotary(q, q, off, off.double(), off.double())[0].flatten(1), q, -1.0)]
    for out, leaf, by in runs:
        got, = torch.autograd.grad(_parts(out)[loss], leaf)
        want, = torch.autograd.grad(_parts(by * leaf.flatten(1))[loss], leaf)
        assert torch.allclose(got, want)
    assert all(seen)
