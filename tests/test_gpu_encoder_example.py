"""The example runs the encoder's operators together: its gradients agree with the same step in plain
fp64 torch, its steps lower the loss, and tokens one at a time give the whole prompt's embeddings."""

import importlib.util
import os

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _example():
    spec = importlib.util.spec_from_file_location("encoder_step",
                                                  os.path.join(ROOT, "examples", "encoder_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _batch(hidden=256):
    g = torch.Generator().manual_seed(1)
    docs = [40, 200, 64, 97, 33, 150]
    x = torch.randn(4 * 16 + sum(docs), hidden, generator=g).to(torch.bfloat16).to(DEV)
    return x, 4, 16, docs, torch.tensor([2, 0, 5, 1], dtype=torch.int32, device=DEV)


def _plain_loss(enc, params, x, n_q, lq, docs, pos, scale, tau):
    """The step in fp64 on the CPU, sequence by sequence."""
    A1, B1, A2, B2 = params
    x, Wq, Wo = x.cpu().double(), enc.w_qkv.cpu().double(), enc.w_out.cpu().double()
    c, s = enc.cos.cpu().double(), enc.sin.cpu().double()
    h, hk, d = enc.heads, enc.kv_heads, enc.dim
    M1, M2 = Wq + 2.0 * B1[0] @ A1[0], Wo + 2.0 * B2[0] @ A2[0]
    emb, t0 = [], 0
    for n in [lq] * n_q + docs:
        qkv = (x[t0:t0 + n] @ M1.T).view(n, -1, d)
        t0 += n

        def turn(z):
            a, b = z[..., :d // 2], z[..., d // 2:]
            cc, ss = c[:n, None], s[:n, None]
            return torch.cat([a * cc - b * ss, b * cc + a * ss], -1)

        q, k, v = turn(qkv[:, :h]), turn(qkv[:, h:h + hk]), qkv[:, h + hk:]
        k, v = k.repeat_interleave(h // hk, 1), v.repeat_interleave(h // hk, 1)
        w = torch.einsum("ihd,jhd->hij", q, k) * d ** -0.5
        w = w.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf")).softmax(-1)
        y = torch.einsum("hij,jhd->ihd", w, v).reshape(n, -1) @ M2.T
        emb.append(y / y.norm(dim=-1, keepdim=True))
    Q, D = torch.stack(emb[:n_q]), emb[n_q:]
    S = torch.stack([torch.stack([(a @ b.T).amax(1).sum() for b in D]) for a in Q]) * scale
    pool_q = torch.nn.functional.normalize(Q.mean(1), dim=-1)
    pool_d = torch.nn.functional.normalize(torch.stack([b.mean(0) for b in D]), dim=-1)
    p = pos.cpu().long()
    li = torch.nn.functional.cross_entropy(S, p)
    lc = torch.nn.functional.cross_entropy(pool_q @ pool_d.T / tau, p)
    return (li + lc) / 2


def test_train_step_against_fp64():
    ex = _example()
    enc = ex.Encoder()
    g = torch.Generator().manual_seed(2)
    with torch.no_grad():  # adapters that have been trained for a while
        for B in (enc.adapters[1], enc.adapters[3]):
            B.copy_(torch.randn(B.shape, generator=g) * 0.2)
    batch = _batch()
    loss, grads = ex.train_step(enc, *batch)
    params = [p.detach().cpu().double().requires_grad_() for p in enc.adapters]
    want = _plain_loss(enc, params, *batch, 1.5625, 0.05)
    want.backward()
    # bf16 embeddings enter the loss: token scores off by 2^-8 each (half from either side), tens of
    # them summed with random signs, times the scale; gradients pass eight roundings of 2^-8
    assert abs(loss.item() - want.item()) < 0.05 * max(1.0, want.item())
    for got, p in zip(grads, params):
        err = (got.cpu().double() - p.grad).norm() / p.grad.norm()
        assert err < 0.1, err


def test_steps_lower_the_loss():
    ex = _example()
    enc = ex.Encoder()
    batch = _batch()
    losses = [ex.train_step(enc, *batch, lr=0.03)[0].item() for _ in range(6)]
    assert losses[-1] < losses[0]


def test_tokens_one_at_a_time_are_the_prompt():
    ex = _example()
    enc = ex.Encoder(n_adapters=3)
    g = torch.Generator().manual_seed(3)
    with torch.no_grad():
        for B in (enc.adapters[1], enc.adapters[3]):
            B.copy_(torch.randn(B.shape, generator=g) * 0.2)
    n_seq, steps = 5, 20
    x = torch.randn(n_seq, steps, 256, generator=g).to(torch.bfloat16).to(DEV)
    adapter = torch.tensor([2, 0, -1, 1, 2], dtype=torch.int32, device=DEV)
    one = ex.answer_tokens(enc, x, adapter, room=24)
    off = torch.arange(n_seq + 1, device=DEV) * steps
    with torch.no_grad():
        whole = enc(x.reshape(n_seq * steps, -1), off, off, adapter).view(one.shape)
    # unit rows whose entries passed the same roundings in another order of sums: a few bf16 units
    assert (one.float() - whole.float()).norm(dim=-1).max() < 0.03
