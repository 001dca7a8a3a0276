"""CPU-only: the encoder operators' argument checks, in the C ABI (before any device call) and in the
binding."""

import ctypes

import pytest
import torch

import paper_2505_04846_amd as hpr

FAKE = 0x10000       # non-NULL, 16-byte aligned, never dereferenced on the host
FAKE_ODD = 0x10008   # misaligned
BIG = 1 << 40


def _desc(**kw):
    a = dict(n_q=100, n_k=100, q_row=1024, q_head=128, k_row=256, k_head=128, v_row=256, v_head=128,
             n_seq=3, heads=8, kv_heads=2, dim=128, dtype=0, causal=1, window=0, scale=0.1)
    a.update(kw)
    return hpr._AttentionDesc(*[a[n] for n, _ in hpr._AttentionDesc._fields_])


def _attn_fwd(desc, q=FAKE, k=FAKE, v=FAKE, q_off=FAKE, k_off=FAKE, k_len=None, out=FAKE, lse=FAKE,
              ws=FAKE, ws_bytes=BIG):
    return hpr.lib().packed_attention_fwd(desc and ctypes.byref(desc), q, k, v, q_off, k_off, k_len,
                                          out, lse, ws, ws_bytes, None)


def _attn_bwd(desc, q=FAKE, k=FAKE, v=FAKE, q_off=FAKE, k_off=FAKE, k_len=None, out=FAKE, lse=FAKE,
              dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, ws_bytes=BIG):
    return hpr.lib().packed_attention_bwd(desc and ctypes.byref(desc), dout, q, k, v, out, lse, q_off,
                                          k_off, k_len, dq, dk, dv, ws, ws_bytes, None)


SHARED = [
    (dict(n_q=-1), {}, 1), (dict(n_k=-1), {}, 1), (dict(n_seq=0), {}, 1), (dict(heads=0), {}, 1),
    (dict(heads=7), {}, 1), (dict(kv_heads=0), {}, 1), (dict(dtype=2), {}, 1), (dict(window=-1), {}, 1),
    (dict(window=5, causal=0), {}, 1), (dict(scale=0.0), {}, 1), (dict(scale=-1.0), {}, 1),
    (dict(scale=float("nan")), {}, 1), (dict(scale=float("inf")), {}, 1), (dict(dim=0), {}, 4),
    (dict(dim=12), {}, 4), (dict(dim=136), {}, 4), (dict(heads=66, kv_heads=2), {}, 4),
    (dict(n_q=1 << 31), {}, 4), (dict(q_row=1020), {}, 4), (dict(k_head=-128), {}, 4),
    (dict(v_row=1 << 22), {}, 4), ({}, dict(q=None), 1), ({}, dict(k=None), 1), ({}, dict(v=None), 1),
    ({}, dict(q_off=None), 1), ({}, dict(k_off=None), 1), ({}, dict(q=FAKE_ODD), 1),
    ({}, dict(out=None), 1), ({}, dict(out=FAKE_ODD), 1), ({}, dict(k_len=FAKE_ODD), 1),
]


@pytest.mark.parametrize("desc,kw,status", SHARED)
def test_attention_rejects(desc, kw, status):
    assert _attn_fwd(_desc(**desc), **kw) == status
    assert hpr.lib().hpr_last_error()
    assert _attn_bwd(_desc(**desc), **kw) == status


def test_attention_rejects_more():
    assert _attn_fwd(None) == 1 and _attn_bwd(None) == 1
    assert _attn_bwd(_desc(), dout=None) == 1 and _attn_bwd(_desc(), lse=None) == 1
    assert _attn_bwd(_desc(), dk=None) == 1 and _attn_bwd(_desc(), dq=FAKE_ODD) == 1
    assert _attn_bwd(_desc(), ws_bytes=0) == 5 and _attn_bwd(_desc(), ws=None) == 5
    split = _desc(n_q=1, n_k=100_000, n_seq=1)  # few rows: the keys are split, and need a workspace
    assert hpr.lib().packed_attention_workspace_size(ctypes.byref(split)) > 0
    assert _attn_fwd(split, ws_bytes=0) == 5 and _attn_fwd(split, ws=None) == 5
    assert hpr.lib().packed_attention_workspace_size(None) == 0
    assert hpr.lib().packed_attention_bwd_workspace_size(ctypes.byref(_desc())) == 100 * 8 * 4 + 128
    # nothing to do
    assert _attn_fwd(_desc(n_q=0, n_k=0, n_seq=0), q=None, k=None, v=None, q_off=None, k_off=None,
                     out=None, ws=None, ws_bytes=0) == 0


def _adapters(call, **kw):
    a = dict(x=FAKE, n=10, k=64, w=FAKE, m=32, a=FAKE, b=FAKE, r=8, n_ad=2, scale=FAKE, off=FAKE,
             adapter=FAKE, n_req=3, dtype=0)
    more = dict(h=FAKE, y=FAKE) if call == "fwd" else dict(dy=FAKE, h=FAKE, dx=FAKE, da=FAKE, db=FAKE,
                                                           ws=FAKE, ws_bytes=BIG)
    a.update(more)
    a.update({n: v for n, v in kw.items() if n in a})
    head = [a[n] for n in ("x", "n", "k", "w", "m", "a", "b", "r", "n_ad", "scale", "off", "adapter",
                           "n_req", "dtype")]
    if call == "fwd":
        return hpr.lib().adapter_linear_fwd(*head, a["h"], a["y"], None)
    return hpr.lib().adapter_linear_bwd(a["dy"], *head, a["h"], a["dx"], a["da"], a["db"], a["ws"],
                                        a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 1), (dict(k=0), 1), (dict(m=0), 1), (dict(r=0), 1), (dict(n_ad=-1), 1),
    (dict(n_req=-1), 1), (dict(dtype=7), 1), (dict(k=60), 4), (dict(m=36), 4), (dict(k=65544), 4),
    (dict(r=129), 4), (dict(n=1 << 31), 4), (dict(n_ad=65536), 4), (dict(x=None), 1), (dict(w=None), 1),
    (dict(a=None), 1), (dict(b=None), 1), (dict(scale=None), 1), (dict(off=None), 1),
    (dict(adapter=None), 1), (dict(x=FAKE_ODD), 1), (dict(w=FAKE_ODD), 1), (dict(h=None), 1),
    (dict(h=FAKE_ODD), 1)])
def test_adapters_reject(kw, status):
    assert _adapters("fwd", **kw) == status
    assert _adapters("bwd", **kw) == status
    assert hpr.lib().hpr_last_error()


def test_adapters_reject_more():
    assert _adapters("fwd", y=None) == 1 and _adapters("bwd", dy=None) == 1
    assert _adapters("bwd", da=FAKE_ODD) == 1
    assert _adapters("bwd", ws_bytes=0) == 5 and _adapters("bwd", ws=None) == 5
    assert _adapters("fwd", n=0, x=None, h=None, y=None) == 0
    assert hpr.lib().adapter_linear_bwd_workspace_size(-1, 64, 32, 8, 2, 3) == 0


def _rotary(**kw):
    a = dict(q=FAKE, q_row=512, q_head=64, q_heads=8, k=FAKE, k_row=128, k_head=64, k_heads=2, n=10,
             dim=64, rot=64, pos=FAKE, cos=FAKE, sin=FAKE, n_pos=100, inverse=0, dtype=0, q_out=FAKE,
             k_out=FAKE)
    a.update(kw)
    return hpr.lib().rotary_apply(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 1), (dict(n=1 << 31), 1), (dict(q_heads=0), 1), (dict(k_heads=-1), 1),
    (dict(n_pos=0), 1), (dict(dtype=3), 1), (dict(dim=60), 4), (dict(dim=1032), 4), (dict(rot=24), 4),
    (dict(rot=80), 4), (dict(rot=0), 4), (dict(q_heads=5000), 4), (dict(q=None), 1), (dict(k=None), 1),
    (dict(pos=None), 1), (dict(cos=None), 1), (dict(q_out=None), 1), (dict(k_out=None), 1),
    (dict(q_row=12), 4), (dict(k_head=-64), 4), (dict(q=FAKE_ODD), 1)])
def test_rotary_rejects(kw, status):
    assert _rotary(**kw) == status
    assert hpr.lib().hpr_last_error()


def test_rotary_nothing_to_do():
    assert _rotary(n=0, q=None, k=None, pos=None, cos=None, sin=None, q_out=None, k_out=None) == 0


def test_binding_rejects_host_tensors_and_other_types():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    off = torch.tensor([0, 4])
    with pytest.raises(ValueError, match="CUDA"):
        hpr.packed_attention_fwd(q, q, q, off)
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        hpr.packed_attention_fwd(q.float(), q, q, off)
    with pytest.raises(TypeError, match="torch.Tensor"):
        hpr.packed_attention_fwd([1], q, q, off)
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        hpr.adapter_linear_fwd(x, x, q, q, torch.ones(2), off, off.int())
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        hpr.adapter_linear_fwd(x.double(), x, q, q, torch.ones(2), off, off.int())
    with pytest.raises(ValueError, match="CUDA"):
        hpr.rotary_apply(q, None, off.int(), torch.ones(2, 32), torch.ones(2, 32))
