"""Python binding of libhiperrag.so: MI355X MaxSim scoring, InfoNCE and exact top-k.

Argument marshalling only.  Every computation runs in the HIP kernels of the shared library;
torch provides device memory (outputs and workspaces) and the current stream.  There is no
fallback: if the library is not built, or a call fails, an exception is raised.

    maxsim_score(Q, D, off)                       -> scores fp32 [nq, n_docs]
    maxsim_score_noalloc(Q, D, off)               -> the same, with no device allocation
    maxsim_topk(Q, D, off, k)                     -> (scores fp32 [nq, k], idx int64 [nq, k])
    coltrast_loss_fwd_bwd(Q, D, off, pos, scale)  -> dict(loss, dq, dd, scores)
    coltrast_loss(Q, D, off, pos, scale)          -> loss with autograd to Q and D
    coltrast_total_loss_fwd_bwd(Q, D, off, pos, scale, tau)
                                                  -> dict(loss [3]: L, L_LI, L_C; dq, dd)
    coltrast_total_loss(Q, D, off, pos, scale, tau) -> L with autograd to Q and D
    dense_ip_topk(Q, X, k)                        -> (scores fp32 [nq, k], idx int64 [nq, k])
    semantic_chunk(E, paper_off, threshold)       -> dict(seg int32 [n], n_segments, cos)
    retrieval_metrics(idx, positive, k)           -> dict(p_at_k, mrr_at_k, ranks) on the device
    csr_validate(off, n_tok)                      -> (status name, first bad document or -1)

The encoder's operators over the same packed sequences, in bf16 or fp16 (attention's q and dout, and the
keys that some query sees, must be finite: what is not stays within its sequence, but need not show in
every output, so look for the overflow of a scaled fp16 loss in out and in dout):

    packed_attention(q, k, v, q_off, ...)         -> out like q, with autograd (once) to q, k and v
    packed_attention_fwd(q, k, v, q_off, ...)     -> dict(out, lse)
    packed_attention_bwd(dout, q, k, v, out, lse, q_off, ...) -> dict(dq, dk, dv)
    adapter_linear(x, W, A, B, scale, off, adapter) -> y [n, m], with autograd (once) to x, A and B
    adapter_linear_fwd(x, W, A, B, scale, off, adapter)       -> dict(y, h)
    adapter_linear_bwd(dy, x, W, A, B, scale, off, adapter, h) -> dict(dx, da, db)
    rotary(q, k, pos, cos, sin)                   -> (q, k) rotated, with autograd to q and k
    rotary_apply(q, k, pos, cos, sin, inverse)    -> (q, k) rotated
    residual_norm(x, b, weight, ...)              -> (r, y): the norm after a block, gate, residual sum and the
                                                     norm before the next, with autograd (once) to everything
    residual_norm_fwd(x, b, weight, ...)          -> dict(r, y)
    residual_norm_bwd(dr, dy, x, b, weight, ...)  -> dict(dx, db, dweight, dbias, dpost_weight, dpost_bias, dgate)
    gated_linear(x, w_gate, w_up, act)            -> h = act(x w_gate^T) * (x w_up^T), with autograd (once)
    gated_linear_fwd(x, w_gate, w_up, act)        -> dict(h)
    gated_linear_bwd(dh, x, w_gate, w_up, act)    -> dict(dx, dw_gate, dw_up)
    checkpoint_pack(x)                            -> Checkpoint: rows in 8 bits, which the two backward passes read
    checkpoint_unpack(c)                          -> the rows that it stands for

Q and D are bf16 CUDA tensors ([nq, lq, dim] and [n_tok, dim]); off is int64 [n_docs + 1];
pos is int32 [nq]; Q and X of dense_ip_topk are fp16 [nq, dim] and [n, dim].  A valid CSR is a
precondition of the MaxSim calls (the library never reads the offsets on the host); with the
environment variable HPR_VALIDATE=1 every MaxSim call first checks it with csr_validate (one
synchronisation) and raises HprError on an invalid one.
"""

import ctypes
import os
from typing import NamedTuple

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libhiperrag.so")

STATUS_NAMES = {
    0: "HPR_OK",
    1: "HPR_ERR_INVALID_ARG",
    2: "HPR_ERR_BAD_CSR",
    3: "HPR_ERR_EMPTY_DOC",
    4: "HPR_ERR_UNSUPPORTED_SHAPE",
    5: "HPR_ERR_WORKSPACE_TOO_SMALL",
    6: "HPR_ERR_CAPACITY",
    7: "HPR_ERR_HIP",
}


class HprError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status
        self.status_name = STATUS_NAMES.get(status, str(status))


_lib = None

_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
_F32 = ctypes.c_float

_SIGNATURES = {
    "maxsim_score": (_I32, [_P, _I32, _I32, _P, _P, _I64, _I64, _I32, _P, _P, _SZ, _P]),
    "maxsim_score_noalloc": (_I32, [_P, _I32, _I32, _P, _P, _I64, _I64, _I32, _P, _P]),
    "maxsim_topk": (_I32, [_P, _I32, _I32, _P, _P, _I64, _I64, _I32, _I32, _P, _P, _P, _SZ, _P]),
    "coltrast_loss_fwd_bwd": (_I32, [_P, _I32, _I32, _P, _P, _I64, _I64, _I32, _P, _F32,
                                     _P, _P, _P, _P, _P, _SZ, _P]),
    "coltrast_total_loss_fwd_bwd": (_I32, [_P, _I32, _I32, _P, _P, _I64, _I64, _I32, _P, _F32,
                                           _F32, _P, _P, _P, _P, _SZ, _P]),
    "dense_ip_topk": (_I32, [_P, _I32, _P, _I64, _I32, _I32, _P, _P, _P, _SZ, _P]),
    "maxsim_score_workspace_size": (_SZ, [_I32, _I32, _I64, _I64, _I32]),
    "maxsim_topk_workspace_size": (_SZ, [_I32, _I32, _I64, _I64, _I32, _I32]),
    "coltrast_loss_workspace_size": (_SZ, [_I32, _I32, _I64, _I64, _I32]),
    "coltrast_total_loss_workspace_size": (_SZ, [_I32, _I32, _I64, _I64, _I32]),
    "dense_ip_topk_workspace_size": (_SZ, [_I32, _I64, _I32, _I32]),
    "semantic_chunk": (_I32, [_P, _I64, _I32, _P, _I64, _F32, _P, _P, _P, _P, _SZ, _P]),
    "semantic_chunk_workspace_size": (_SZ, [_I64, _I32]),
    "retrieval_metrics": (_I32, [_P, _I32, _I32, _I32, _P, _P, _P, _P]),
    "packed_attention_workspace_size": (_SZ, [_P]),
    "packed_attention_bwd_workspace_size": (_SZ, [_P]),
    "packed_attention_fwd": (_I32, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "packed_attention_bwd": (_I32, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "adapter_linear_fwd": (_I32, [_P, _I64, _I32, _P, _I32, _P, _P, _I32, _I32, _P, _P, _P, _I32, _I32,
                                  _P, _P, _P]),
    "adapter_linear_bwd_workspace_size": (_SZ, [_I64, _I32, _I32, _I32, _I32, _I32]),
    "adapter_linear_bwd": (_I32, [_P, _P, _I64, _I32, _P, _I32, _P, _P, _I32, _I32, _P, _P, _P, _I32,
                                  _I32, _P, _P, _P, _P, _P, _SZ, _P]),
    "rotary_apply": (_I32, [_P, _I64, _I64, _I32, _P, _I64, _I64, _I32, _I64, _I32, _I32, _P, _P, _P,
                            _I64, _I32, _I32, _P, _P, _P]),
    "checkpoint_pack": (_I32, [_P, _I64, _I64, _I32, _I32, _P, _P, _P]),
    "checkpoint_unpack": (_I32, [_P, _P, _I64, _I32, _I32, _P, _P]),
    "gated_linear_fwd": (_I32, [_P, _I64, _I64, _I32, _P, _P, _I32, _I32, _I32, _P, _P]),
    "gated_linear_bwd_workspace_size": (_SZ, [_I64, _I32, _I32, _I32, _I32, _I32]),
    "gated_linear_bwd": (_I32, [_P, _P, _P, _I64, _I64, _I32, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _SZ,
                                _P]),
    "residual_norm_fwd": (_I32, [_P] * 11),
    "residual_norm_bwd_workspace_size": (_SZ, [_P]),
    "residual_norm_bwd": (_I32, [_P] * 19 + [_SZ, _P]),
    "hpr_mfma_calibration": (_I32, [_I64, _I32, _P, ctypes.POINTER(ctypes.c_double), _P]),
    "hpr_read_calibration": (_I32, [_P, _I64, _P, _P]),
    "hpr_csr_validate": (_I32, [_P, _I64, _I64, _P, _P, _P]),
    "hpr_scale_f32": (_I32, [_P, _I64, _P, _P]),
    "hpr_scale_grads_bf16": (_I32, [_P, _I64, _P, _P, _I64, _P, _P, _P]),
    "hpr_kernel_timing": (_I32, [_I32]),
    "hpr_kernel_timing_read": (_I32, [ctypes.c_char_p, ctypes.POINTER(ctypes.c_double),
                                      ctypes.POINTER(ctypes.c_int64)]),
    "hpr_status_string": (ctypes.c_char_p, [_I32]),
    "hpr_last_error": (ctypes.c_char_p, []),
    "hpr_abi_version": (_I32, []),
}


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2505_04846_amd.build` "
                "(there is no fallback implementation)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _check(status):
    if status != 0:
        raise HprError(status, lib().hpr_last_error().decode())


def _public_raw_stream(index):
    return torch.cuda.current_stream(index).cuda_stream


# The raw handle of a device's current stream, without the Stream object around it.  torch's accessor
# for it is not public: where it is missing, the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _public_raw_stream)
# The current device's index likewise, without the checks around it (the tensors of a call are on a device
# already).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(device):
    index = device.index
    return _raw_stream(torch.cuda.current_device() if index is None else index)


def _launch(fn, device, *args):
    """fn(*args, stream) with `device` current and its current stream last; raises on a status.
    Entering torch's device guard costs about as much as a kernel launch, so only a call for
    another device than the current one does."""
    index = device.index  # (a tensor's device always has one)
    if _current_device() == index:
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            status = fn(*args, _raw_stream(index))
    if status != 0:
        _check(status)


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _need(t, name, dtype, ndim, device=None):
    if (isinstance(t, torch.Tensor) and t.dtype == dtype and t.dim() == ndim and t.is_cuda
            and (device is None or t.device == device) and t.is_contiguous()):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions, got {t.dim()}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def _given_workspace(ws, nbytes, device):
    """ws where it can serve, or a new one."""
    fits = ws is not None and ws.device == device and ws.is_contiguous() and ws.numel() >= nbytes \
        and ws.data_ptr() % 256 == 0
    return ws if fits else _workspace(nbytes, device)


def _maxsim_inputs(Q, D, off):
    _need(Q, "Q", torch.bfloat16, 3)
    dev = Q.device
    _need(D, "D", torch.bfloat16, 2, dev)
    _need(off, "off", torch.int64, 1, dev)
    nq, lq, dim = Q.shape
    if D.shape[1] != dim:
        raise ValueError(f"D has dim {D.shape[1]}, Q has {dim}")
    if os.environ.get("HPR_VALIDATE") == "1":  # debugging aid: checks the CSR, synchronising
        status, doc = csr_validate(off, D.shape[0])
        if status != "HPR_OK":
            raise HprError({v: k for k, v in STATUS_NAMES.items()}[status],
                           f"invalid CSR offsets (first bad document {doc})")
    return dev, nq, lq, dim, off.numel() - 1, D.shape[0]


def maxsim_score(Q, D, off, ws=None):
    dev, nq, lq, dim, n_docs, n_tok = _maxsim_inputs(Q, D, off)
    L = lib()
    need = L.maxsim_score_workspace_size(nq, lq, n_docs, n_tok, dim)
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    scores = torch.empty((nq, n_docs), dtype=torch.float32, device=dev)
    _launch(L.maxsim_score, dev, _ptr(Q), nq, lq, _ptr(D), _ptr(off), n_docs, n_tok, dim,
            _ptr(scores), _ptr(ws), ws.numel())
    return scores


def maxsim_score_noalloc(Q, D, off, out=None):
    """maxsim_score through the entry point that allocates no device memory (its scratch is a
    static array of the library); `out` may be a preallocated fp32 [nq, n_docs] tensor."""
    dev, nq, lq, dim, n_docs, n_tok = _maxsim_inputs(Q, D, off)
    scores = out if out is not None else torch.empty((nq, n_docs), dtype=torch.float32,
                                                     device=dev)
    _need(scores, "out", torch.float32, 2, dev)
    if tuple(scores.shape) != (nq, n_docs):
        raise ValueError(f"out must be [{nq}, {n_docs}]")
    _launch(lib().maxsim_score_noalloc, dev, _ptr(Q), nq, lq, _ptr(D), _ptr(off), n_docs, n_tok,
            dim, _ptr(scores))
    return scores


def maxsim_topk(Q, D, off, k, ws=None):
    dev, nq, lq, dim, n_docs, n_tok = _maxsim_inputs(Q, D, off)
    L = lib()
    need = L.maxsim_topk_workspace_size(nq, lq, n_docs, n_tok, dim, k)
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    out_s = torch.empty((nq, k), dtype=torch.float32, device=dev)
    out_i = torch.empty((nq, k), dtype=torch.int64, device=dev)
    _launch(L.maxsim_topk, dev, _ptr(Q), nq, lq, _ptr(D), _ptr(off), n_docs, n_tok, dim, int(k),
            _ptr(out_s), _ptr(out_i), _ptr(ws), ws.numel())
    return out_s, out_i


def coltrast_workspace(Q, D, off):
    dev, nq, lq, dim, n_docs, n_tok = _maxsim_inputs(Q, D, off)
    return _workspace(lib().coltrast_loss_workspace_size(nq, lq, n_docs, n_tok, dim), dev)


def coltrast_loss_fwd_bwd(Q, D, off, pos, logit_scale, need_dq=True, need_dd=True,
                          return_scores=False, ws=None, out=None):
    """Loss (fp32 [1]), dQ (fp32 like Q or None), dD (fp32 like D or None), scores or None.

    `out` may hold preallocated outputs {"loss", "dq", "dd", "scores"} (reused as given).
    """
    dev, nq, lq, dim, n_docs, n_tok = _maxsim_inputs(Q, D, off)
    _need(pos, "pos", torch.int32, 1, dev)
    if pos.numel() != nq:
        raise ValueError("pos must hold one positive per query")
    L = lib()
    need = L.coltrast_loss_workspace_size(nq, lq, n_docs, n_tok, dim)
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    out = {} if out is None else out
    loss = out.get("loss")
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=dev)
    dq = out.get("dq") if need_dq else None
    if need_dq and dq is None:
        dq = torch.empty(Q.shape, dtype=torch.float32, device=dev)
    dd = out.get("dd") if need_dd else None
    if need_dd and dd is None:
        dd = torch.empty(D.shape, dtype=torch.float32, device=dev)
    scores = out.get("scores") if return_scores else None
    if return_scores and scores is None:
        scores = torch.empty((nq, n_docs), dtype=torch.float32, device=dev)
    _launch(L.coltrast_loss_fwd_bwd, dev, _ptr(Q), nq, lq, _ptr(D), _ptr(off), n_docs, n_tok, dim,
            _ptr(pos), float(logit_scale), _ptr(loss), _ptr(dq), _ptr(dd), _ptr(scores), _ptr(ws),
            ws.numel())
    return {"loss": loss, "dq": dq, "dd": dd, "scores": scores}


def coltrast_total_workspace(Q, D, off):
    dev, nq, lq, dim, n_docs, n_tok = _maxsim_inputs(Q, D, off)
    return _workspace(lib().coltrast_total_loss_workspace_size(nq, lq, n_docs, n_tok, dim), dev)


def coltrast_total_loss_fwd_bwd(Q, D, off, pos, logit_scale, temperature, need_dq=True,
                                need_dd=True, ws=None, out=None):
    """Loss (fp32 [3]: L, L_LI, L_C), dQ (fp32 like Q or None), dD (fp32 like D or None).

    `out` may hold preallocated outputs {"loss", "dq", "dd"} (reused as given).
    """
    dev, nq, lq, dim, n_docs, n_tok = _maxsim_inputs(Q, D, off)
    _need(pos, "pos", torch.int32, 1, dev)
    if pos.numel() != nq:
        raise ValueError("pos must hold one positive per query")
    L = lib()
    need = L.coltrast_total_loss_workspace_size(nq, lq, n_docs, n_tok, dim)
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    out = {} if out is None else out
    loss = out.get("loss")
    if loss is None:
        loss = torch.empty(3, dtype=torch.float32, device=dev)
    dq = out.get("dq") if need_dq else None
    if need_dq and dq is None:
        dq = torch.empty(Q.shape, dtype=torch.float32, device=dev)
    dd = out.get("dd") if need_dd else None
    if need_dd and dd is None:
        dd = torch.empty(D.shape, dtype=torch.float32, device=dev)
    _launch(L.coltrast_total_loss_fwd_bwd, dev, _ptr(Q), nq, lq, _ptr(D), _ptr(off), n_docs, n_tok,
            dim, _ptr(pos), float(logit_scale), float(temperature), _ptr(loss), _ptr(dq), _ptr(dd),
            _ptr(ws), ws.numel())
    return {"loss": loss, "dq": dq, "dd": dd}


def scale_(x, scale):
    """x *= scale in place (x fp32 contiguous CUDA tensor, scale a 1-element fp32 CUDA tensor)."""
    _launch(lib().hpr_scale_f32, x.device, _ptr(x), x.numel(), _ptr(scale))
    return x


def _scaled_grads(dq, dd, scale):
    """bf16(dq * scale) and bf16(dd * scale) (either may be None) in one launch; dq and dd stay
    as they are.  The inputs of the losses are bf16, so this is what autograd hands on."""
    device = (dq if dq is not None else dd).device
    # (a saved-tensor hook may hand back another type or layout than it was given)
    src = [t if t is None or (t.dtype == torch.float32 and t.is_contiguous())
           else t.to(torch.float32).contiguous() for t in (dq, dd)]
    out = [None if t is None else torch.empty(t.shape, dtype=torch.bfloat16, device=device)
           for t in src]
    q, d = [0 if t is None else t.numel() for t in src]
    _launch(lib().hpr_scale_grads_bf16, device, _ptr(src[0]), q, _ptr(out[0]), _ptr(src[1]), d,
            _ptr(out[1]), _ptr(scale))
    return out


class _ColTrastLI(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, D, off, pos, logit_scale):
        r = coltrast_loss_fwd_bwd(Q.detach(), D.detach(), off, pos, logit_scale,
                                  need_dq=ctx.needs_input_grad[0],
                                  need_dd=ctx.needs_input_grad[1])
        ctx.save_for_backward(*(t for t in (r["dq"], r["dd"]) if t is not None))
        ctx.has = (r["dq"] is not None, r["dd"] is not None)
        return r["loss"][0]

    @staticmethod
    def backward(ctx, grad_out):
        saved = list(ctx.saved_tensors)
        g = grad_out.to(torch.float32)  # a scalar: 0-dimensional
        dq = saved.pop(0) if ctx.has[0] else None
        dd = saved.pop(0) if ctx.has[1] else None
        # the saved gradients stay as the forward left them, so a second backward over a retained
        # graph scales them afresh
        if dq is not None or dd is not None:
            dq, dd = _scaled_grads(dq, dd, g)
        return dq, dd, None, None, None


def coltrast_loss(Q, D, off, pos, logit_scale):
    """L_LI as a differentiable scalar (gradients reach Q and D)."""
    return _ColTrastLI.apply(Q, D, off, pos, float(logit_scale))


class _ColTrastTotal(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, D, off, pos, logit_scale, temperature):
        r = coltrast_total_loss_fwd_bwd(Q.detach(), D.detach(), off, pos, logit_scale,
                                        temperature, need_dq=ctx.needs_input_grad[0],
                                        need_dd=ctx.needs_input_grad[1])
        ctx.save_for_backward(*(t for t in (r["dq"], r["dd"]) if t is not None))
        ctx.has = (r["dq"] is not None, r["dd"] is not None)
        return r["loss"][0]

    @staticmethod
    def backward(ctx, grad_out):
        dq, dd = _ColTrastLI.backward(ctx, grad_out)[:2]
        return dq, dd, None, None, None, None


def coltrast_total_loss(Q, D, off, pos, logit_scale, temperature):
    """The ColTrast loss (L_LI + L_C) / 2 as a differentiable scalar."""
    return _ColTrastTotal.apply(Q, D, off, pos, float(logit_scale), float(temperature))


def dense_ip_topk(Q, X, k, ws=None):
    _need(Q, "Q", torch.float16, 2)
    dev = Q.device
    _need(X, "X", torch.float16, 2, dev)
    nq, dim = Q.shape
    n = X.shape[0]
    if X.shape[1] != dim:
        raise ValueError(f"X has dim {X.shape[1]}, Q has {dim}")
    L = lib()
    need = L.dense_ip_topk_workspace_size(nq, n, dim, k)
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    out_s = torch.empty((nq, k), dtype=torch.float32, device=dev)
    out_i = torch.empty((nq, k), dtype=torch.int64, device=dev)
    _launch(L.dense_ip_topk, dev, _ptr(Q), nq, _ptr(X), n, dim, int(k), _ptr(out_s), _ptr(out_i),
            _ptr(ws), ws.numel())
    return out_s, out_i


def dense_workspace(Q, X, k):
    return _workspace(lib().dense_ip_topk_workspace_size(Q.shape[0], X.shape[0], Q.shape[1], k),
                      Q.device)


def semantic_chunk(E, paper_off, threshold, return_cos=False, ws=None, out=None):
    """Segment ids of fp16 sentence embeddings E [n, dim] (paper_off int64 [n_papers + 1] or
    None for one paper).  Returns dict(seg int32 [n], n_segments int64 [1], cos fp32 [n] or None),
    all on the device.  `out` may hold preallocated {"seg", "n_segments", "cos"}."""
    _need(E, "E", torch.float16, 2)
    dev = E.device
    n, dim = E.shape
    n_papers = 0
    if paper_off is not None:
        _need(paper_off, "paper_off", torch.int64, 1, dev)
        n_papers = paper_off.numel() - 1
    L = lib()
    need = L.semantic_chunk_workspace_size(n, dim)
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    out = {} if out is None else out
    seg = out.get("seg")
    if seg is None:
        seg = torch.empty(n, dtype=torch.int32, device=dev)
    n_seg = out.get("n_segments")
    if n_seg is None:
        n_seg = torch.empty(1, dtype=torch.int64, device=dev)
    cos = out.get("cos") if return_cos else None
    if return_cos and cos is None:
        cos = torch.empty(n, dtype=torch.float32, device=dev)
    _launch(L.semantic_chunk, dev, _ptr(E), n, dim, _ptr(paper_off), n_papers, float(threshold),
            _ptr(cos), _ptr(seg), _ptr(n_seg), _ptr(ws), ws.numel())
    return {"seg": seg, "n_segments": n_seg, "cos": cos}


def semantic_chunk_workspace(E):
    return _workspace(lib().semantic_chunk_workspace_size(E.shape[0], E.shape[1]), E.device)


def retrieval_metrics(idx, positive, k=None):
    """P@k and MRR@k of index lists idx int64 [nq, ld] against positive int64 [nq].  Returns
    dict(metrics fp64 [2] = (P@k, MRR@k), ranks int32 [nq]) on the device."""
    _need(idx, "idx", torch.int64, 2)
    dev = idx.device
    _need(positive, "positive", torch.int64, 1, dev)
    nq, ld = idx.shape
    k = ld if k is None else int(k)
    if positive.numel() != nq:
        raise ValueError("positive must hold one index per query")
    metrics = torch.empty(2, dtype=torch.float64, device=dev)
    ranks = torch.empty(nq, dtype=torch.int32, device=dev)
    _launch(lib().retrieval_metrics, dev, _ptr(idx), nq, ld, k, _ptr(positive), _ptr(ranks),
            _ptr(metrics))
    return {"metrics": metrics, "ranks": ranks}


# ---- the encoder's operators --------------------------------------------------------------

_HALF_TYPES = {torch.bfloat16: 0, torch.float16: 1}


class _AttentionDesc(ctypes.Structure):
    _fields_ = [(n, _I64) for n in ("n_q", "n_k", "q_row", "q_head", "k_row", "k_head", "v_row",
                                    "v_head")] + \
               [(n, _I32) for n in ("n_seq", "heads", "kv_heads", "dim", "dtype", "causal",
                                    "window")] + [("scale", _F32)]


def _need_heads(t, name, dtype, device):
    """Row and head strides of t [rows, heads, dim], with contiguous values and 16-byte aligned rows
    and heads (views of a projection's output are fine).  A dimension of one row or head is never
    stepped over: its stride counts as 0."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.dim() == 3 and t.is_cuda
            and t.device == device):
        row, head, one = t.stride()
        n, heads, _ = t.shape
        if n < 2:
            row = 0
        if heads < 2:
            head = 0
        if one == 1 and not (row | head) & 7 and not t.data_ptr() & 15 and dtype in _HALF_TYPES:
            return row, head
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype or dtype not in _HALF_TYPES:
        raise TypeError(f"{name} must be bfloat16 or float16, the same for every tensor, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must have 3 dimensions, got {t.dim()}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    row = t.stride(0) if t.shape[0] > 1 else 0
    head = t.stride(1) if t.shape[1] > 1 else 0
    if t.numel() and ((t.stride(2) != 1 and t.shape[2] > 1) or row % 8 or head % 8
                      or t.data_ptr() % 16):
        raise ValueError(f"{name} must have contiguous values, and rows and heads aligned to 16 bytes")
    return (row, head) if t.numel() else (0, 0)


def _attention_desc(q, k, v, q_off, k_off, k_len, causal, window, scale):
    dtype = getattr(q, "dtype", None)
    dev = getattr(q, "device", None)
    q_row, q_head = _need_heads(q, "q", dtype, dev)
    k_row, k_head = _need_heads(k, "k", dtype, dev)
    v_row, v_head = _need_heads(v, "v", dtype, dev)
    if k.shape != v.shape:
        raise ValueError(f"k and v differ in shape: {tuple(k.shape)}, {tuple(v.shape)}")
    n_q, heads, dim = q.shape
    n_k, kv_heads, k_dim = k.shape
    if dim != k_dim:
        raise ValueError(f"k has dim {k_dim}, q has {dim}")
    _need(q_off, "q_off", torch.int64, 1, dev)
    if q_off.numel() < 1:
        raise ValueError("q_off must hold n_seq + 1 offsets")
    if k_off is None:
        k_off = q_off
        if n_k != n_q:
            raise ValueError(f"k has {n_k} rows, q has {n_q}: pass k_off")
    elif k_off is not q_off:
        _need(k_off, "k_off", torch.int64, 1, dev)
        if k_off.numel() != q_off.numel():
            raise ValueError("k_off must hold as many offsets as q_off")
    n_seq = q_off.numel() - 1
    if k_len is not None:
        _need(k_len, "k_len", torch.int64, 1, dev)
        if k_len.numel() != n_seq:
            raise ValueError("k_len must hold one length per sequence")
    scale = dim ** -0.5 if scale is None and dim else scale
    d = _AttentionDesc(n_q, n_k, q_row, q_head, k_row, k_head, v_row, v_head, n_seq, heads, kv_heads,
                       dim, _HALF_TYPES[dtype], bool(causal), int(window), float(scale or 0.0))
    return dev, d, k_off


def packed_attention_fwd(q, k, v, q_off, k_off=None, k_len=None, causal=True, window=0, scale=None,
                         need_lse=True, out=None, ws=None):
    """Attention over packed sequences: dict(out [n_q, heads, dim], lse fp32 [n_q, heads] or None).

    q [n_q, heads, dim], k and v [n_k, kv_heads, dim], bf16 or fp16; sequence s has query rows
    q_off[s]..q_off[s+1] and key rows k_off[s]..k_off[s+1] (int64; None: q_off), of which the first
    k_len[s] count (int64 [n_seq]; None: all).  causal aligns the last query with the last key;
    window > 0 also hides keys more than window - 1 before it.  scale defaults to dim ** -0.5.  A ws that
    is too small is not used; the size a call needs is not monotone in its sizes.
    """
    dev, d, k_off = _attention_desc(q, k, v, q_off, k_off, k_len, causal, window, scale)
    L = lib()
    need = L.packed_attention_workspace_size(ctypes.byref(d))
    if need and (ws is None or ws.numel() < need):
        ws = _workspace(need, dev)
    if out is None:
        out = torch.empty((d.n_q, d.heads, d.dim), dtype=q.dtype, device=dev)
    else:
        _need(out, "out", q.dtype, 3, dev)
        if out.shape != q.shape:
            raise ValueError(f"out must be {tuple(q.shape)}")
    lse = torch.empty((d.n_q, d.heads), dtype=torch.float32, device=dev) if need_lse else None
    _launch(L.packed_attention_fwd, dev, ctypes.byref(d), _ptr(q), _ptr(k), _ptr(v), _ptr(q_off),
            _ptr(k_off), _ptr(k_len), _ptr(out), _ptr(lse), _ptr(ws) if need else None,
            ws.numel() if need else 0)
    return {"out": out, "lse": lse}


def packed_attention_bwd(dout, q, k, v, out, lse, q_off, k_off=None, k_len=None, causal=True, window=0,
                         scale=None, need_dq=True, need_dkv=True, ws=None):
    """Gradients of packed_attention_fwd: dict(dq, dk, dv), dense and of the inputs' type; dq, or dk
    and dv together, None where not needed.  out and lse are the forward's."""
    dev, d, k_off = _attention_desc(q, k, v, q_off, k_off, k_len, causal, window, scale)
    for t, name in ((dout, "dout"), (out, "out")):
        _need(t, name, q.dtype, 3, dev)
        if t.shape != q.shape:
            raise ValueError(f"{name} must be {tuple(q.shape)}")
    _need(lse, "lse", torch.float32, 2, dev)
    if lse.shape != q.shape[:2]:
        raise ValueError(f"lse must be {tuple(q.shape[:2])}")
    L = lib()
    need = L.packed_attention_bwd_workspace_size(ctypes.byref(d))
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    dq = torch.empty(q.shape, dtype=q.dtype, device=dev) if need_dq else None
    dk = torch.empty(k.shape, dtype=q.dtype, device=dev) if need_dkv else None
    dv = torch.empty(k.shape, dtype=q.dtype, device=dev) if need_dkv else None
    _launch(L.packed_attention_bwd, dev, ctypes.byref(d), _ptr(dout), _ptr(q), _ptr(k), _ptr(v),
            _ptr(out), _ptr(lse), _ptr(q_off), _ptr(k_off), _ptr(k_len), _ptr(dq), _ptr(dk), _ptr(dv),
            _ptr(ws), ws.numel())
    return {"dq": dq, "dk": dk, "dv": dv}


class _FirstOrder(torch.autograd.Function):
    """Gradients as they are, as functions of the tensors after them that has no derivative."""

    @staticmethod
    def forward(ctx, name, count, *tensors):
        ctx.name = name
        return tuple(t.detach() for t in tensors[:count])

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(f"{ctx.name} has no second derivatives")


def _frozen(**operands):
    """Raises where an operand that no gradient reaches asks for one."""
    for name, t in operands.items():
        if isinstance(t, torch.Tensor) and t.requires_grad:
            raise ValueError(f"{name} is frozen: it must not require a gradient")


def _first_order(name, grads, *of):
    """grads (some None) of a backward pass that autograd does not see into.  While it records one
    (create_graph), they are tied to the tensors `of` that they depend on: a second derivative raises
    instead of leaving their terms out."""
    if not torch.is_grad_enabled():
        return grads
    of = [t for t in of if t.requires_grad]
    some = [g for g in grads if g is not None]
    if not of or not some:
        return grads
    tied = iter(_FirstOrder.apply(name, len(some), *some, *of))
    return [g if g is None else next(tied) for g in grads]


def _dense(grad):
    """A gradient as the library reads it: dense, at a multiple of 16 bytes.  autograd may hand over a part of a larger
    buffer (the backward pass of torch.cat), which can begin anywhere."""
    grad = grad.contiguous()
    return grad if grad.data_ptr() % 16 == 0 else grad.clone()


class _PackedAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_off, k_off, k_len, causal, window, scale):
        ctx.how = (causal, window, scale)
        train = any(ctx.needs_input_grad[:3])
        r = packed_attention_fwd(q.detach(), k.detach(), v.detach(), q_off, k_off, k_len, causal,
                                 window, scale, need_lse=train)
        if train:
            ctx.save_for_backward(q, k, v, r["out"], r["lse"], q_off, k_off, k_len)
        return r["out"]

    @staticmethod
    def backward(ctx, grad_out):
        q, k, v, out, lse, q_off, k_off, k_len = ctx.saved_tensors
        need = ctx.needs_input_grad
        g = packed_attention_bwd(_dense(grad_out), q, k, v, out, lse, q_off, k_off, k_len,
                                 *ctx.how, need_dq=need[0], need_dkv=need[1] or need[2])
        dq, dk, dv = _first_order("packed_attention", [g["dq"], g["dk"] if need[1] else None,
                                                       g["dv"] if need[2] else None],
                                  grad_out, q, k, v)
        return dq, dk, dv, None, None, None, None, None, None


def packed_attention(q, k, v, q_off, k_off=None, k_len=None, causal=True, window=0, scale=None):
    """packed_attention_fwd's out, differentiable once (gradients reach q, k and v; scale is frozen)."""
    _frozen(scale=scale)
    return _PackedAttention.apply(q, k, v, q_off, k_off, k_len, causal, window, scale)


def _adapter_inputs(x, W, A, B, scale, off, adapter):
    dtype = getattr(x, "dtype", None)
    if dtype not in _HALF_TYPES:
        raise TypeError(f"x must be a bfloat16 or float16 tensor, got {dtype or type(x).__name__}")
    _need(x, "x", dtype, 2)
    dev = x.device
    _need(W, "W", dtype, 2, dev)
    _need(A, "A", dtype, 3, dev)
    _need(B, "B", dtype, 3, dev)
    _need(scale, "scale", torch.float32, 1, dev)
    _need(off, "off", torch.int64, 1, dev)
    _need(adapter, "adapter", torch.int32, 1, dev)
    n, k = x.shape
    m = W.shape[0]
    n_ad, r = A.shape[:2]
    if W.shape[1] != k or A.shape[2] != k:
        raise ValueError(f"x has {k} columns, W {W.shape[1]} and A {A.shape[2]}")
    if B.shape != (n_ad, m, r):
        raise ValueError(f"B must be {(n_ad, m, r)}, got {tuple(B.shape)}")
    if scale.numel() != n_ad:
        raise ValueError("scale must hold one factor per adapter")
    if off.numel() != adapter.numel() + 1:
        raise ValueError("off must hold one offset per request and one more")
    return dev, n, k, m, r, n_ad, adapter.numel(), _HALF_TYPES[dtype]


def adapter_linear_fwd(x, W, A, B, scale, off, adapter, out=None):
    """A shared projection with a low-rank adapter per request beside it: dict(y [n, m], h).

    x [n, k], W [m, k], A [n_ad, r, k], B [n_ad, m, r], bf16 or fp16; scale fp32 [n_ad].  Request s
    has rows off[s]..off[s+1] (int64 [n_req + 1]) and adapter[s] (int32 [n_req], negative: none):
    h_t = scale A x_t, y_t = W x_t + B h_t.  h [n, r rounded up to 16] is what the gradients read.
    """
    dev, n, k, m, r, n_ad, n_req, code = _adapter_inputs(x, W, A, B, scale, off, adapter)
    h = torch.empty((n, (r + 15) // 16 * 16), dtype=x.dtype, device=dev)
    if out is None:
        out = torch.empty((n, m), dtype=x.dtype, device=dev)
    else:
        _need(out, "out", x.dtype, 2, dev)
        if out.shape != (n, m):
            raise ValueError(f"out must be {(n, m)}")
    _launch(lib().adapter_linear_fwd, dev, _ptr(x), n, k, _ptr(W), m, _ptr(A), _ptr(B), r, n_ad,
            _ptr(scale), _ptr(off), _ptr(adapter), n_req, code, _ptr(h), _ptr(out))
    return {"y": out, "h": h}


def adapter_linear_bwd(dy, x, W, A, B, scale, off, adapter, h, need_dx=True, need_da=True, need_db=True,
                       ws=None):
    """Gradients of adapter_linear_fwd's y: dict(dx, da, db), of the inputs' type, None where not
    needed.  W and scale are frozen.  A ws that is too small is not used; the size a call needs is not
    monotone in its sizes."""
    dev, n, k, m, r, n_ad, n_req, code = _adapter_inputs(x, W, A, B, scale, off, adapter)
    _need(dy, "dy", x.dtype, 2, dev)
    if dy.shape != (n, m):
        raise ValueError(f"dy must be {(n, m)}")
    _need(h, "h", x.dtype, 2, dev)
    if h.shape != (n, (r + 15) // 16 * 16):
        raise ValueError("h must be the forward's")
    L = lib()
    need = L.adapter_linear_bwd_workspace_size(n, k, m, r, n_ad, n_req)
    ws = ws if ws is not None and ws.numel() >= need else _workspace(need, dev)
    dx = torch.empty_like(x) if need_dx else None
    da = torch.empty_like(A) if need_da else None
    db = torch.empty_like(B) if need_db else None
    _launch(L.adapter_linear_bwd, dev, _ptr(dy), _ptr(x), n, k, _ptr(W), m, _ptr(A), _ptr(B), r, n_ad,
            _ptr(scale), _ptr(off), _ptr(adapter), n_req, code, _ptr(h), _ptr(dx), _ptr(da), _ptr(db),
            _ptr(ws), ws.numel())
    return {"dx": dx, "da": da, "db": db}


class _AdapterLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, A, B, scale, off, adapter):
        r = adapter_linear_fwd(x.detach(), W.detach(), A.detach(), B.detach(), scale, off, adapter)
        ctx.save_for_backward(x, W, A, B, scale, off, adapter, r["h"])
        return r["y"]

    @staticmethod
    def backward(ctx, grad_y):
        need = ctx.needs_input_grad
        saved = ctx.saved_tensors
        g = adapter_linear_bwd(_dense(grad_y), *saved, need_dx=need[0], need_da=need[2],
                               need_db=need[3])
        x, _, A, B = saved[:4]
        dx, da, db = _first_order("adapter_linear", [g["dx"], g["da"], g["db"]], grad_y, x, A, B)
        return dx, None, da, db, None, None, None


def adapter_linear(x, W, A, B, scale, off, adapter):
    """adapter_linear_fwd's y, differentiable once (gradients reach x, A and B; W and scale are frozen)."""
    _frozen(W=W, scale=scale)
    return _AdapterLinear.apply(x, W, A, B, scale, off, adapter)


def rotary_apply(q, k, pos, cos, sin, inverse=False):
    """q [n, heads, dim] and k [n, kv_heads, dim] (or None) rotated by their rows' positions.

    pos int32 [n]; cos and sin fp32 [n_pos, rot / 2]: values j and j + rot / 2 of every head turn by
    the position's angle j, values past rot are copied.  inverse turns back (the gradient).
    """
    dtype = getattr(q, "dtype", None)
    dev = getattr(q, "device", None)
    q_row, q_head = _need_heads(q, "q", dtype, dev)
    n, heads, dim = q.shape
    k_row = k_head = kv_heads = 0
    if k is not None:
        k_row, k_head = _need_heads(k, "k", dtype, dev)
        rows, kv_heads, k_dim = k.shape
        if rows != n or k_dim != dim:
            raise ValueError(f"k must be [{n}, kv_heads, {dim}], got {tuple(k.shape)}")
    _need(pos, "pos", torch.int32, 1, dev)
    if pos.numel() != n:
        raise ValueError("pos must hold one position per row")
    _need(cos, "cos", torch.float32, 2, dev)
    _need(sin, "sin", torch.float32, 2, dev)
    if cos.shape != sin.shape:
        raise ValueError("cos and sin differ in shape")
    q_out = torch.empty((n, heads, dim), dtype=dtype, device=dev)
    k_out = torch.empty((n, kv_heads, dim), dtype=dtype, device=dev) if k is not None else None
    n_pos, half = cos.shape
    _launch(lib().rotary_apply, dev, q.data_ptr(), q_row, q_head, heads, _ptr(k), k_row, k_head, kv_heads,
            n, dim, 2 * half, pos.data_ptr(), cos.data_ptr(), sin.data_ptr(), n_pos, bool(inverse),
            _HALF_TYPES[dtype], q_out.data_ptr(), _ptr(k_out))
    return q_out, k_out


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, pos, cos, sin, inverse):
        ctx.save_for_backward(pos, cos, sin)
        ctx.inverse = inverse
        return rotary_apply(q.detach(), k.detach() if k is not None else None, pos, cos, sin, inverse)

    @staticmethod
    def backward(ctx, gq, gk):
        need_q, need_k = ctx.needs_input_grad[:2]
        a, b = [_dense(g) if g is not None and need else None
                for g, need in ((gq, need_q), (gk, need_k))]
        back = (*ctx.saved_tensors, not ctx.inverse)
        # (a rotation too, and differentiable as one)
        if a is not None:
            a, b = _Rotary.apply(a, b, *back)
        elif b is not None:
            b, _ = _Rotary.apply(b, None, *back)
        return a, b, None, None, None, None


def rotary(q, k, pos, cos, sin):
    """rotary_apply, differentiable (gradients reach q and k, by the rotation back; cos and sin are
    frozen)."""
    _frozen(cos=cos, sin=sin)
    return _Rotary.apply(q, k, pos, cos, sin, False)


def _need_rows(t, name, dtype, device):
    """Row stride of t [rows, values], with contiguous values and 16-byte aligned rows (columns of a wider
    tensor are fine).  One row is never stepped over: its stride counts as 0."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and dtype in _HALF_TYPES and t.device == device and t.is_cuda
            and t.is_contiguous()):
        shape = t.shape
        if len(shape) == 2 and not (shape[1] & 7 or t.data_ptr() & 15):
            return shape[1]
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype or dtype not in _HALF_TYPES:
        raise TypeError(f"{name} must be bfloat16 or float16, the same for every tensor, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name} must have 2 dimensions, got {t.dim()}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    row = t.stride(0) if t.shape[0] > 1 else 0
    if t.numel() and ((t.stride(1) != 1 and t.shape[1] > 1) or row % 8 or t.data_ptr() % 16):
        raise ValueError(f"{name} must have contiguous values, and rows aligned to 16 bytes")
    return row if t.numel() else 0


class Checkpoint(NamedTuple):
    """Rows in 8 bits (checkpoint_pack): codes int8 [n, dim], exps uint8 [n, ceil(dim / 32)], and the rows' type."""

    codes: torch.Tensor
    exps: torch.Tensor
    dtype: torch.dtype


def _need_checkpoint(c, name, dtype=None, device=None):
    if c.dtype not in _HALF_TYPES or (dtype is not None and c.dtype != dtype):
        raise TypeError(f"{name} must stand for {dtype or 'bfloat16 or float16'}, got {c.dtype}")
    _need(c.codes, f"{name}.codes", torch.int8, 2, device)
    _need(c.exps, f"{name}.exps", torch.uint8, 2, c.codes.device)
    n, dim = c.codes.shape
    if tuple(c.exps.shape) != (n, (dim + 31) // 32):
        raise ValueError(f"{name}.exps must be {(n, (dim + 31) // 32)}, got {tuple(c.exps.shape)}")


def _rows_or_checkpoint(t, name, dtype, device):
    """(pointer, exps pointer, row stride, shape) of 16-bit rows or of a checkpoint of them."""
    if isinstance(t, Checkpoint):
        _need_checkpoint(t, name, dtype, device)
        return t.codes.data_ptr(), t.exps.data_ptr(), 0, t.codes.shape
    row = _need_rows(t, name, dtype, device)
    return t.data_ptr(), None, row, t.shape


def _need_vector(t, name, dtype, dim, device):
    """Pointer of t [dim], None for None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device and t.is_cuda
            and t.shape == (dim,) and t.is_contiguous()):
        _need(t, name, dtype, 1, device)
        if t.numel() != dim:
            raise ValueError(f"{name} must hold {dim} values, got {t.numel()}")
    return t.data_ptr()


def checkpoint_pack(x):
    """x [n, dim], bf16 or fp16 (rows may be strided), in 8 bits: for every 32 values of a row a power of two
    2^e, e = floor(log2 max|x|) - 6, and whole numbers of at most 127 times it.  A block that holds a value that
    is not finite reads back as NaN."""
    dtype = getattr(x, "dtype", None)
    dev = getattr(x, "device", None)
    row = _need_rows(x, "x", dtype, dev)
    n, dim = x.shape
    codes = torch.empty(n, dim, dtype=torch.int8, device=dev)
    exps = torch.empty(n, (dim + 31) // 32, dtype=torch.uint8, device=dev)
    _launch(lib().checkpoint_pack, dev, x.data_ptr(), row, n, dim, _HALF_TYPES[dtype], codes.data_ptr(),
            exps.data_ptr())
    return Checkpoint(codes, exps, dtype)


def checkpoint_unpack(c, out=None):
    """The rows [n, dim] that a checkpoint stands for, in its type (exactly)."""
    if not isinstance(c, Checkpoint):
        raise TypeError("c must be a Checkpoint")
    _need_checkpoint(c, "c")
    dev = c.codes.device
    n, dim = c.codes.shape
    if out is None:
        out = torch.empty(n, dim, dtype=c.dtype, device=dev)
    else:
        _need(out, "out", c.dtype, 2, dev)
        if out.shape != (n, dim):
            raise ValueError(f"out must be {(n, dim)}")
    _launch(lib().checkpoint_unpack, dev, _ptr(c.codes), _ptr(c.exps), n, dim, _HALF_TYPES[c.dtype], _ptr(out))
    return out


_ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


def _gated_weights(w_gate, w_up, act):
    dtype = getattr(w_gate, "dtype", None)
    if dtype not in _HALF_TYPES:
        raise TypeError(f"w_gate must be a bfloat16 or float16 tensor, got {dtype or type(w_gate).__name__}")
    _need(w_gate, "w_gate", dtype, 2)
    dev = w_gate.device
    _need(w_up, "w_up", dtype, 2, dev)
    shape = w_gate.shape
    if shape != w_up.shape:
        raise ValueError(f"w_gate and w_up differ in shape: {tuple(shape)}, {tuple(w_up.shape)}")
    if act not in _ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(_ACTIVATIONS)}, got {act!r}")
    return dev, dtype, *shape


def gated_linear_fwd(x, w_gate, w_up, act="silu", out=None):
    """The gated feed-forward projections: dict(h [n, f]), h = act(x w_gate^T) * (x w_up^T).

    x [n, k] (rows may be strided), w_gate and w_up [f, k], bf16 or fp16; act "silu", "gelu" or "gelu_tanh".
    """
    dev, dtype, f, k = _gated_weights(w_gate, w_up, act)
    row = _need_rows(x, "x", dtype, dev)
    n, cols = x.shape
    if cols != k:
        raise ValueError(f"x has {cols} columns, w_gate {k}")
    if out is None:
        out = x.new_empty(n, f)
    else:
        _need(out, "out", dtype, 2, dev)
        if out.shape != (n, f):
            raise ValueError(f"out must be {(n, f)}")
    _launch(lib().gated_linear_fwd, dev, x.data_ptr(), row, n, k, w_gate.data_ptr(), w_up.data_ptr(), f,
            _ACTIVATIONS[act], _HALF_TYPES[dtype], out.data_ptr())
    return {"h": out}


def gated_linear_bwd(dh, x, w_gate, w_up, act="silu", need_dx=True, need_dw=True, ws=None):
    """Gradients of gated_linear_fwd's h: dict(dx, dw_gate, dw_up), dense and of the inputs' type, None where
    not needed.  x: the forward's, or a Checkpoint of it (the gradients are those at the values that it stands
    for).  The gradients of the two projections, dh u act'(g) and dh act(g), are rounded once to the type, as the
    products' operands; in fp16 times powers of two that hold them for every g and u that are numbers of it (from
    131,040 on, act(g) and u act'(g) overflow; below 2^-12 they lose bits).  A ws that is too small, not aligned or not
    dense on x's device is not used."""
    dev, dtype, f, k = _gated_weights(w_gate, w_up, act)
    x_ptr, exps, row, shape = _rows_or_checkpoint(x, "x", dtype, dev)
    n = shape[0]
    if shape[1] != k:
        raise ValueError(f"x has {shape[1]} columns, w_gate {k}")
    _need(dh, "dh", dtype, 2, dev)
    if dh.shape != (n, f):
        raise ValueError(f"dh must be {(n, f)}")
    L = lib()
    need = L.gated_linear_bwd_workspace_size(n, k, f, exps is not None, bool(need_dx), bool(need_dw))
    ws = _given_workspace(ws, need, dev)
    dx = torch.empty((n, k), dtype=dtype, device=dev) if need_dx else None
    dw = [torch.empty((f, k), dtype=dtype, device=dev) if need_dw else None for _ in range(2)]
    _launch(L.gated_linear_bwd, dev, _ptr(dh), x_ptr, exps, row, n, k, _ptr(w_gate), _ptr(w_up), f,
            _ACTIVATIONS[act], _HALF_TYPES[dtype], _ptr(dx), _ptr(dw[0]), _ptr(dw[1]), _ptr(ws), ws.numel())
    return {"dx": dx, "dw_gate": dw[0], "dw_up": dw[1]}


def _no_second(name):
    """A backward pass that reads a checkpoint has not its inputs to tie a second derivative to."""
    if torch.is_grad_enabled():
        raise RuntimeError(f"{name} from a checkpoint has no second derivatives (create_graph)")


class _GatedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, act, checkpoint):
        h = gated_linear_fwd(x.detach(), w_gate.detach(), w_up.detach(), act)["h"]
        ctx.act, ctx.packed = act, None
        if checkpoint and any(ctx.needs_input_grad[:3]):
            c = checkpoint_pack(x.detach())
            ctx.packed = c.dtype
            ctx.save_for_backward(w_gate, w_up, c.codes, c.exps)
        else:
            ctx.save_for_backward(w_gate, w_up, x)
        return h

    @staticmethod
    def backward(ctx, grad_h):
        w_gate, w_up, *x = ctx.saved_tensors
        if ctx.packed is not None:
            _no_second("gated_linear")
        need = ctx.needs_input_grad
        of = x[0].detach() if ctx.packed is None else Checkpoint(*x, ctx.packed)
        g = gated_linear_bwd(_dense(grad_h), of, w_gate.detach(), w_up.detach(), ctx.act, need_dx=need[0],
                             need_dw=need[1] or need[2])
        dx, dg, du = _first_order("gated_linear", [g["dx"], g["dw_gate"] if need[1] else None,
                                                   g["dw_up"] if need[2] else None],
                                  grad_h, w_gate, w_up, *([] if ctx.packed else x))
        return dx, dg, du, None, None


def gated_linear(x, w_gate, w_up, act="silu", checkpoint=False):
    """gated_linear_fwd's h, differentiable once (gradients reach x, w_gate and w_up).  Of the forward it keeps
    x alone, with checkpoint in 8 bits."""
    return _GatedLinear.apply(x, w_gate, w_up, act, bool(checkpoint))


_NORMS = {"rms": 0, "layer": 1}


class _NormDesc(ctypes.Structure):
    _fields_ = [(n, _I64) for n in ("n", "x_row", "b_row")] + \
               [(n, _I32) for n in ("dim", "dtype", "kind", "gate_rows")] + [("scale", _F32), ("eps", _F32)]


def _norm_inputs(x, b, weight, bias, post_weight, post_bias, gate, scale, eps, kind):
    """Device, type, description, the pointers of x, its exps, b and its exps, and those of the vectors and gate."""
    dtype = getattr(x, "dtype", None)
    dev = x.codes.device if isinstance(x, Checkpoint) else getattr(x, "device", None)
    if kind not in _NORMS:
        raise ValueError(f"kind must be one of {', '.join(_NORMS)}, got {kind!r}")
    if b is not None and isinstance(x, Checkpoint) != isinstance(b, Checkpoint):
        raise TypeError("x and b must both be tensors or both be Checkpoints")
    x_ptr, x_exps, x_row, shape = _rows_or_checkpoint(x, "x", dtype, dev)
    n, dim = shape
    b_ptr = b_exps = None
    b_row = 0
    if b is not None:
        b_ptr, b_exps, b_row, b_shape = _rows_or_checkpoint(b, "b", dtype, dev)
        if b_shape != shape:
            raise ValueError(f"b must be {tuple(shape)}, got {tuple(b_shape)}")
    elif post_weight is not None or post_bias is not None or gate is not None:
        raise ValueError("post_weight, post_bias and gate need b")
    vectors = (_need_vector(weight, "weight", dtype, dim, dev), _need_vector(bias, "bias", dtype, dim, dev),
               _need_vector(post_weight, "post_weight", dtype, dim, dev),
               _need_vector(post_bias, "post_bias", dtype, dim, dev))
    if kind != "layer" and (bias is not None or post_bias is not None):
        raise ValueError("a bias needs kind \"layer\"")
    if (bias is not None and weight is None) or (post_bias is not None and post_weight is None):
        raise ValueError("a bias needs its weight")
    gate_rows = 0
    gate_ptr = None
    if isinstance(gate, torch.Tensor) and gate.dim() == 2:
        gate_rows = 1
        _need(gate, "gate", dtype, 2, dev)
        if gate.shape != shape:
            raise ValueError(f"gate must be {(dim,)} or {tuple(shape)}, got {tuple(gate.shape)}")
        gate_ptr = gate.data_ptr()
    else:
        gate_ptr = _need_vector(gate, "gate", dtype, dim, dev)
    d = _NormDesc(n, x_row, b_row, dim, _HALF_TYPES[dtype], _NORMS[kind], gate_rows, float(scale), float(eps))
    return dev, dtype, d, (x_ptr, x_exps, b_ptr, b_exps), (*vectors, gate_ptr)


def residual_norm_fwd(x, b=None, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, scale=1.0,
                      eps=1e-6, kind="rms"):
    """The norm after a block, its gate and residual scale, the residual sum and the norm before the next block:

        p = N(b; post_weight, post_bias)   (b itself without post_weight)
        r = x + scale * gate * p           (x itself without b)
        y = N(r; weight, bias)             (None without weight)

    dict(r, y).  x (the residual stream) and b (the block's output) [n, dim], rows may be strided; weights and
    biases [dim]; gate [dim] or [n, dim] or None; kind "rms" or "layer" (biases are the latter's).
    """
    dev, _, d, (x_ptr, x_exps, b_ptr, _), vectors = _norm_inputs(x, b, weight, bias, post_weight, post_bias, gate,
                                                                 scale, eps, kind)
    if isinstance(x, Checkpoint):
        raise TypeError("x and b must be tensors")
    n, dim = x.shape
    r = x.new_empty(n, dim) if b is not None else None
    y = x.new_empty(n, dim) if weight is not None else None
    _launch(lib().residual_norm_fwd, dev, ctypes.byref(d), x_ptr, b_ptr, *vectors, _ptr(r), _ptr(y))
    return {"r": x if b is None else r, "y": y}


def residual_norm_bwd(dr, dy, x, b=None, weight=None, bias=None, post_weight=None, post_bias=None, gate=None,
                      scale=1.0, eps=1e-6, kind="rms", need_dx=True, need_db=True, need_dw=True, need_dgate=True,
                      ws=None):
    """Gradients of residual_norm_fwd's r and y: dict(dx, db, dweight, dbias, dpost_weight, dpost_bias, dgate),
    dense and of the inputs' type, None where there is nothing that they are the gradient of or where not needed
    (need_dw: the weights' and biases').  dr and dy [n, dim], either may be None.  x and b: the forward's, or
    Checkpoints of them (the gradients are those at the values that they stand for)."""
    dev, dtype, d, (x_ptr, x_exps, b_ptr, b_exps), (w_ptr, _, pw_ptr, pc_ptr, g_ptr) = _norm_inputs(
        x, b, weight, bias, post_weight, post_bias, gate, scale, eps, kind)
    for t, name in ((dr, "dr"), (dy, "dy")):
        if t is None:
            continue
        _need(t, name, dtype, 2, dev)
        if t.shape != (d.n, d.dim):
            raise ValueError(f"{name} must be {(d.n, d.dim)}")
    if dy is not None and weight is None:
        raise ValueError("dy needs weight")

    def like(t, need):
        return torch.empty(t.shape, dtype=dtype, device=dev) if need and t is not None else None

    rows = (d.n, d.dim)
    dx = torch.empty(rows, dtype=dtype, device=dev) if need_dx else None
    db = torch.empty(rows, dtype=dtype, device=dev) if need_db and b is not None else None
    dw, dc, dpw, dpc = [like(t, need_dw) for t in (weight, bias, post_weight, post_bias)]
    dgate = like(gate, need_dgate)
    L = lib()
    need = L.residual_norm_bwd_workspace_size(ctypes.byref(d))
    ws = _given_workspace(ws, need, dev)
    _launch(L.residual_norm_bwd, dev, ctypes.byref(d), _ptr(dr), _ptr(dy), x_ptr, x_exps, b_ptr, b_exps,
            w_ptr, pw_ptr, pc_ptr, g_ptr, _ptr(dx), _ptr(db), _ptr(dw), _ptr(dc),
            _ptr(dpw), _ptr(dpc), _ptr(dgate), _ptr(ws), ws.numel())
    return {"dx": dx, "db": db, "dweight": dw, "dbias": dc, "dpost_weight": dpw, "dpost_bias": dpc, "dgate": dgate}


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, b, weight, bias, post_weight, post_bias, gate, scale, eps, kind, checkpoint):
        of = [None if t is None else t.detach() for t in (x, b, weight, bias, post_weight, post_bias, gate)]
        r = residual_norm_fwd(*of, scale=scale, eps=eps, kind=kind)
        ctx.how = dict(scale=scale, eps=eps, kind=kind)
        ctx.packed, ctx.has_b = None, b is not None
        ctx.set_materialize_grads(False)
        if checkpoint and any(ctx.needs_input_grad[:7]):
            c = [checkpoint_pack(t) for t in of[:2] if t is not None]
            ctx.packed = c[0].dtype
            ctx.save_for_backward(weight, bias, post_weight, post_bias, gate, *(t for p in c for t in p[:2]))
        else:
            ctx.save_for_backward(weight, bias, post_weight, post_bias, gate, x, b)
        # (without a block r is x, which the caller has)
        return r["r"] if ctx.has_b else None, r["y"]

    @staticmethod
    def backward(ctx, grad_r, grad_y):
        weight, bias, post_weight, post_bias, gate, *rows = ctx.saved_tensors
        if ctx.packed is not None:
            _no_second("residual_norm")
        if grad_r is None and grad_y is None:
            return (None,) * 11
        need = ctx.needs_input_grad
        if ctx.packed is None:
            x, b = [None if t is None else t.detach() for t in rows]
            inputs = [t for t in rows if t is not None]
        else:
            x, *b = [Checkpoint(*rows[i:i + 2], ctx.packed) for i in range(0, len(rows), 2)]
            b, inputs = (b[0] if b else None), []
        vectors = [None if t is None else t.detach() for t in (weight, bias, post_weight, post_bias, gate)]
        g = residual_norm_bwd(*(None if t is None else _dense(t) for t in (grad_r, grad_y)), x, b, *vectors,
                              **ctx.how, need_dx=need[0], need_db=need[1], need_dw=any(need[2:6]),
                              need_dgate=need[6])
        names = ("dx", "db", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate")
        of = [t for t in (grad_r, grad_y, *inputs, weight, bias, post_weight, post_bias, gate) if t is not None]
        grads = _first_order("residual_norm", [g[t] if wanted else None for t, wanted in zip(names, need)], *of)
        return (*grads, None, None, None, None)


def residual_norm(x, b=None, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, scale=1.0,
                  eps=1e-6, kind="rms", checkpoint=False):
    """residual_norm_fwd's (r, y), differentiable once (gradients reach every tensor; scale and eps are frozen).
    Of the forward it keeps x and b alone, with checkpoint in 8 bits."""
    _frozen(scale=scale, eps=eps)
    if b is None and weight is None:
        raise ValueError("there is nothing to do without b and without weight")
    r, y = _ResidualNorm.apply(x, b, weight, bias, post_weight, post_bias, gate, float(scale), float(eps), kind,
                               bool(checkpoint))
    return (x if b is None else r), y


def calibrate(device="cuda:0", mfma_iters=20000, read_bytes=16 << 30, reps=3):
    """Measured ceilings of this device: bf16 MFMA TFLOP/s on a fixed low-entropy operand
    pattern and on random embedding-sized operands, and the HBM read rate in GB/s; each the
    best of `reps` timed launches of the library's calibration kernels on the current stream."""
    dev = torch.device(device)
    L = lib()
    sink_f = torch.empty(4096, dtype=torch.float32, device=dev)
    sink_u = torch.empty(16384, dtype=torch.int32, device=dev)
    buf = torch.ones(read_bytes // 4, dtype=torch.float32, device=dev)
    flops = ctypes.c_double(0.0)
    best = [0.0, 0.0, 0.0]
    with torch.cuda.device(dev):
        s = _stream(dev)

        def timed(launch):
            a = torch.cuda.Event(enable_timing=True)
            b = torch.cuda.Event(enable_timing=True)
            a.record()
            launch()
            b.record()
            b.synchronize()
            return a.elapsed_time(b) * 1e-3

        for rep in range(reps + 1):  # the first of each is a warm-up
            for operands in (0, 1):
                t = timed(lambda: _check(L.hpr_mfma_calibration(
                    mfma_iters, operands, _ptr(sink_f), ctypes.byref(flops), s)))
                if rep:
                    best[operands] = max(best[operands], flops.value / t / 1e12)
            t = timed(lambda: _check(L.hpr_read_calibration(_ptr(buf), buf.numel() * 4,
                                                            _ptr(sink_u), s)))
            if rep:
                best[2] = max(best[2], buf.numel() * 4 / t / 1e9)
    del buf
    return tuple(best)


def kernel_timing(enable):
    """Turns per-kernel HIP-event timing inside the library on or off."""
    _check(lib().hpr_kernel_timing(1 if enable else 0))


def kernel_timing_read(name):
    """(total milliseconds, launches) recorded for kernel `name` since the last read."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(lib().hpr_kernel_timing_read(name.encode(), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def csr_validate(off, n_tok):
    """Checks CSR offsets on the device (synchronises).  Returns (status name, first bad doc)."""
    _need(off, "off", torch.int64, 1)
    ws = _workspace(16, off.device)
    bad = ctypes.c_int64(-1)
    with torch.cuda.device(off.device):
        st = lib().hpr_csr_validate(_ptr(off), off.numel() - 1, int(n_tok), _ptr(ws),
                                    _stream(off.device), ctypes.byref(bad))
    if st not in (0, 2, 3):
        _check(st)
    return STATUS_NAMES[st], bad.value
