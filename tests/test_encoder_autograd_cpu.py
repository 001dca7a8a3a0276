"""CPU-only: what the encoder operators' autograd functions do around their kernels, which plain torch
stands in for."""

import pytest
import torch

import paper_2505_04846_amd as hpr


def _attention(q, k, v):
    x = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) * q.shape[2] ** -0.5
    return torch.matmul(x.softmax(-1), v.transpose(0, 1)).transpose(0, 1)


def _adapters(x, W, A, B):
    return x @ W.T + (x @ A[0].T) @ B[0].T


def _rotate(x, pos, cos, sin, inverse=False):
    c, s = cos[pos.long()][:, None], (-sin if inverse else sin)[pos.long()][:, None]
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _grads(fn, inputs, g):
    with torch.enable_grad():
        t = [z.detach().requires_grad_() for z in inputs]
        return torch.autograd.grad(fn(*t), t, g)


@pytest.fixture
def plain(monkeypatch):
    """One sequence, all keys visible; one request.  Nothing that these compute is seen by autograd."""

    def attention_fwd(q, k, v, *args, need_lse=True, **how):
        return {"out": _attention(q, k, v), "lse": torch.zeros(q.shape[:2])}

    def attention_bwd(dout, q, k, v, *args, **how):
        return dict(zip(("dq", "dk", "dv"), _grads(_attention, (q, k, v), dout)))

    def adapters_fwd(x, W, A, B, *args):
        return {"y": _adapters(x, W, A, B), "h": x}

    def adapters_bwd(dy, x, W, A, B, *args, need_dx=True, need_da=True, need_db=True):
        dx, _, da, db = _grads(_adapters, (x, W, A, B), dy)
        return {"dx": dx if need_dx else None, "da": da if need_da else None,
                "db": db if need_db else None}

    def rotary_apply(q, k, pos, cos, sin, inverse=False):
        return tuple(t if t is None else _rotate(t.detach(), pos, cos, sin, inverse)
                     for t in (q, k))

    for name, fn in (("packed_attention_fwd", attention_fwd), ("packed_attention_bwd", attention_bwd),
                     ("adapter_linear_fwd", adapters_fwd), ("adapter_linear_bwd", adapters_bwd),
                     ("rotary_apply", rotary_apply)):
        monkeypatch.setattr(hpr, name, fn)


def _attention_inputs():
    g = torch.Generator().manual_seed(1)
    return [torch.randn(5, 2, 8, generator=g, dtype=torch.float64) for _ in range(3)]


def _adapter_inputs():
    g = torch.Generator().manual_seed(2)
    return [torch.randn(*s, generator=g, dtype=torch.float64)
            for s in ((5, 8), (6, 8), (1, 3, 8), (1, 6, 3))]


def _calls():
    q, k, v = _attention_inputs()
    x, W, A, B = _adapter_inputs()
    none = torch.zeros(1)
    return {
        "packed_attention": (lambda *t: hpr.packed_attention(*t, None), [q, k, v], _attention),
        "adapter_linear": (lambda x, A, B: hpr.adapter_linear(x, W, A, B, none, none, none),
                           [x, A, B], lambda x, A, B: _adapters(x, W, A, B)),
    }


@pytest.mark.parametrize("name", ["packed_attention", "adapter_linear"])
def test_second_derivatives_raise(plain, name):
    fn, inputs, formula = _calls()[name]
    t = [z.clone().requires_grad_() for z in inputs]
    # the gradient itself is there under create_graph, and says that it depends on the inputs
    y = fn(*t)
    first = torch.autograd.grad(y.sum(), t, create_graph=True)
    for got, want in zip(first, _grads(formula, inputs, torch.ones_like(y))):
        assert torch.allclose(got, want) and got.requires_grad
    with pytest.raises(RuntimeError, match=f"{name} has no second derivatives"):
        (y.sum() + sum((g ** 2).sum() for g in first)).backward()
    # ... so does one with respect to a single input, through a gradient of y that depends on others
    last = inputs[-1].clone().requires_grad_()
    up = torch.ones_like(y).requires_grad_()
    g, = torch.autograd.grad(fn(*inputs[:-1], last), last, up, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivatives"):
        g.sum().backward()


@pytest.mark.parametrize("name", ["packed_attention", "adapter_linear"])
def test_first_derivatives_under_create_graph(plain, name):
    """A backward pass that is recorded and never differentiated again is as any other."""
    fn, inputs, formula = _calls()[name]
    t = [z.clone().requires_grad_() for z in inputs]
    fn(*t).sum().backward(create_graph=True)
    for z, want in zip(t, _grads(formula, inputs, torch.ones_like(fn(*inputs)))):
        assert torch.allclose(z.grad, want)


@pytest.mark.parametrize("which", ["both", "q", "k", "q alone"])
def test_rotary_second_derivatives(plain, which):
    """The gradient is a rotation of the gradient from above, and differentiable as one."""
    g = torch.Generator().manual_seed(3)
    q, k = [torch.randn(5, h, 8, generator=g, dtype=torch.float64) for h in (3, 2)]
    angle = torch.rand(7, 4, generator=g, dtype=torch.float64)
    cos, sin, pos = angle.cos(), angle.sin(), torch.tensor([6, 0, 3, 3, 1])
    q.requires_grad_(which != "k")
    k = k.requires_grad_(which in ("both", "k")) if which != "q alone" else None
    t = [z for z in (q, k) if z is not None and z.requires_grad]

    def second(fn):
        """Gradients of a sum that the first gradients enter as squares."""
        y = [z for z in fn() if z is not None and z.requires_grad]
        first = torch.autograd.grad(sum((z ** 3).sum() for z in y), t, create_graph=True)
        return torch.autograd.grad(sum((z ** 2).sum() for z in first), t)

    got = second(lambda: hpr.rotary(q, k, pos, cos, sin))
    want = second(lambda: [z if z is None else _rotate(z, pos, cos, sin) for z in (q, k)])
    assert all(torch.allclose(a, b) for a, b in zip(got, want))


def test_operands_without_a_gradient_refuse_one(plain):
    q, k, v = _attention_inputs()
    angle = torch.rand(7, 4)
    pos = torch.zeros(5, dtype=torch.int32)
    one = torch.ones(1, requires_grad=True)
    for cos, sin, name in ((angle.cos().requires_grad_(), angle.sin(), "cos"),
                           (angle.cos(), angle.sin().requires_grad_(), "sin")):
        with pytest.raises(ValueError, match=f"{name} is frozen"):
            hpr.rotary(q, k, pos, cos, sin)
    with pytest.raises(ValueError, match="scale is frozen"):
        hpr.packed_attention(q, k, v, None, scale=one)
    x, W, A, B = _adapter_inputs()
    with pytest.raises(ValueError, match="W is frozen"):
        hpr.adapter_linear(x, W.requires_grad_(), A, B, None, None, None)
    with pytest.raises(ValueError, match="scale is frozen"):
        hpr.adapter_linear(x, W.detach(), A, B, one, None, None)
