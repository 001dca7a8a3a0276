"""The rest of the encoder's block in fp64: the gated feed-forward projections, the norms around a block with its
gate and residual scale, and activations in 8 bits, the first two with their gradients from the formulas.

`gated_linear` and `residual_norm` also return, entry by entry, how far a computation that rounds its operands
and outputs to a type of unit roundoff `u` (off by `tiny` below its normal range) and computes in fp32 may be from
the exact value: `bound` in each result, which the tests hold the GPU to.
"""

import math

import numpy as np

F32 = 2.0 ** -24     # unit roundoff of fp32
LEAST = 2.0 ** -126  # its least normal number
_erfc = np.vectorize(math.erfc, otypes=[float])


# ---- activations in 8 bits --------------------------------------------------------------------


def checkpoint_pack(x, least):
    """codes int8 and exps uint8 of x [n, d] (fp64); least: the lowest power of two (-24 fp16, -126 bf16)."""
    n, d = x.shape
    blocks = -(-d // 32)
    v = np.zeros((n, blocks * 32))
    v[:, :d] = x
    v = v.reshape(n, blocks, 32)
    fine = np.isfinite(v).all(-1)
    v = np.where(fine[..., None], v, 0.0)
    top = np.abs(v).max(-1)
    e = np.frexp(top)[1] - 1 - 6  # floor(log2 top) - 6
    e = np.maximum(np.where(top > 0, e, least), least)
    code = np.clip(np.rint(np.ldexp(v, -e[..., None])), -127, 127)
    exps = np.where(fine, e + 127, 255).astype(np.uint8)
    return code.astype(np.int8).reshape(n, blocks * 32)[:, :d], exps


def checkpoint_values(codes, exps):
    """The values that they stand for."""
    d = codes.shape[1]
    e = np.repeat(exps.astype(int), 32, axis=1)[:, :d]
    return np.where(e == 255, np.nan, np.ldexp(codes.astype(float), e - 127))


# ---- the gated projections --------------------------------------------------------------------


def activation(name, g):
    """Value, derivative, the sum of the derivative's terms' magnitudes, and how many times its fp32 rounding an
    exponential in it may be off (the size of its exponent)."""
    if name == "silu":
        s = np.where(g > 0, 1 / (1 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1 + np.exp(-np.abs(g))))
        return g * s, s * (1 + g * (1 - s)), s * (1 + np.abs(g) * (1 - s)), np.abs(g)
    if name == "gelu":
        c = 0.5 * _erfc(-g / math.sqrt(2))
        d = np.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        return g * c, c + g * d, c + np.abs(g) * d, g * g
    z = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    s = 0.5 * (1 + np.tanh(z))
    slope = math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)
    d = 0.5 * slope * np.where(np.abs(z) < 300, np.cosh(np.minimum(np.abs(z), 300.0)) ** -2.0, 0.0)
    return g * s, s + g * d, s + np.abs(g) * d, 2 * np.abs(z)


def _power(top):
    """The power of two of top, 1 where it is zero."""
    return np.where(top > 0, 2.0 ** (np.frexp(top)[1] - 1), 1.0)


def gated_linear(x, w_gate, w_up, act, dh=None, u=0.0, tiny=0.0):
    """x [n, k], w_gate and w_up [f, k] (fp64).  dict(h[, dx, dw_gate, dw_up], bound)."""
    n, k = x.shape
    f = w_gate.shape[0]
    ax, ag, au = np.abs(x), np.abs(w_gate), np.abs(w_up)
    g, v = x @ w_gate.T, x @ w_up.T
    eg, ev = k * F32 * (ax @ ag.T), k * F32 * (ax @ au.T)
    a, slope, size, reach = activation(act, g)
    rel = F32 * (16 + 4 * reach)
    # neither an activation's slope nor that slope's passes 1.2 in magnitude
    ea = 1.2 * eg + rel * np.abs(a) + LEAST
    es = 1.2 * eg + rel * size + LEAST
    h = a * v
    r = {"h": h}
    b = {"h": 1.01 * (ea * (np.abs(v) + ev) + np.abs(a) * ev + 2 * F32 * np.abs(h))}
    if dh is not None:
        adh = np.abs(dh)
        dg, du = dh * v * slope, dh * a
        # (as operands: rounded to u, in fp16 below the normal range at the size of the row or column: they are
        # multiplied by the power of two that brings its largest |dh| to [1/4, 1/2), rounded to within `tiny` there,
        # and divided by it again, which makes it 4 tiny times the power of two of that |dh|)
        e_g = adh * (np.abs(slope) * ev + es * (np.abs(v) + ev)) + (3 * F32 + u) * np.abs(dg) + LEAST
        e_u = adh * ea + (2 * F32 + u) * np.abs(du) + LEAST
        row = 4 * tiny * _power(adh.max(1, initial=0.0))[:, None]
        col = 4 * tiny * _power(adh.max(0, initial=0.0))[None]
        r.update(dx=dg @ w_gate + du @ w_up, dw_gate=dg.T @ x, dw_up=du.T @ x)
        b["dx"] = 1.01 * ((e_g + row) @ ag + (e_u + row) @ au
                          + 2 * f * F32 * (np.abs(dg) @ ag + np.abs(du) @ au))
        b["dw_gate"] = 1.01 * ((e_g + col).T @ ax + (n + 8) * F32 * (np.abs(dg).T @ ax))
        b["dw_up"] = 1.01 * ((e_u + col).T @ ax + (n + 8) * F32 * (np.abs(du).T @ ax))
    for name in r:
        b[name] = b[name] + u * np.abs(r[name]) + max(tiny, LEAST)
    r["bound"] = b
    return r


# ---- norms around a block ---------------------------------------------------------------------

# An fp32 sum over a row: at most 32 values one after another in a lane, then 9 steps over lanes and waves, and the
# roundings of its terms.
ROW = 48 * F32


class _Norm:
    """Rows v with entrywise errors ev: hat (normalised), rs (1 / sigma), and their errors (of rs: relative)."""

    def __init__(self, v, ev, eps, layer):
        mean = v.mean(1, keepdims=True) if layer else 0.0
        em = (ev + ROW * np.abs(v)).mean(1, keepdims=True) if layer else 0.0
        q = v - mean
        eq = ev + em + F32 * np.abs(q)
        self.rs = 1 / np.sqrt((q * q).mean(1, keepdims=True) + eps)
        self.ers = 0.5 * self.rs ** 2 * (2 * np.abs(q) * eq + eq * eq + ROW * q * q).mean(1, keepdims=True) + 6 * F32
        self.hat = q * self.rs
        self.ehat = self.rs * eq + np.abs(self.hat) * (self.ers + 2 * F32)
        self.layer = layer

    def back(self, e, ee):
        """The gradient with respect to v from e with respect to hat, and its error."""
        along = (e * self.hat).mean(1, keepdims=True)
        ealong = (ee * np.abs(self.hat) + np.abs(e) * self.ehat + 1.5 * ROW * np.abs(e * self.hat)).mean(
            1, keepdims=True)
        base, ebase = 0.0, 0.0
        if self.layer:
            base = e.mean(1, keepdims=True)
            ebase = (ee + 1.5 * ROW * np.abs(e)).mean(1, keepdims=True)
        r = (e - base - self.hat * along) * self.rs
        size = np.abs(e) + np.abs(base) + np.abs(self.hat * along)
        return r, self.rs * (ee + ebase + self.ehat * np.abs(along) + np.abs(self.hat) * ealong
                             + 4 * F32 * size) + np.abs(r) * self.ers


def residual_norm(x, b=None, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, scale=1.0,
                  eps=1e-6, kind="rms", dr=None, dy=None, u=0.0, tiny=0.0):
    """x and b [n, d], weights and biases [d], gate [d] or [n, d] (fp64).  dict of r and y and, with dr or dy,
    the gradients of everything that is there, and bound."""
    n, d = x.shape
    layer = kind == "layer"
    out, err = {}, {}
    zero = np.zeros((n, d))
    r, er = x, zero
    if b is not None:
        g = 1.0 if gate is None else gate
        norm = None
        hat, ehat, w, o = b, zero, 1.0, 0.0
        if post_weight is not None:
            norm = _Norm(b, zero, eps, layer)
            hat, ehat, w = norm.hat, norm.ehat, post_weight
            o = 0.0 if post_bias is None else post_bias
        p = hat * w + o
        ep = ehat * np.abs(w) + 2 * F32 * (np.abs(hat * w) + np.abs(o))
        r = x + scale * g * p
        er = np.abs(scale * g) * (ep + 3 * F32 * np.abs(p)) + F32 * np.abs(r)
        out["r"], err["r"] = r, er
    if weight is not None:
        pre = _Norm(r, er, eps, layer)
        c = 0.0 if bias is None else bias
        out["y"] = pre.hat * weight + c
        err["y"] = pre.ehat * np.abs(weight) + 2 * F32 * (np.abs(pre.hat * weight) + np.abs(c))
    if dr is not None or dy is not None:
        dx, edx = (zero if dr is None else dr), zero
        total = 8 * F32 * max(1, n)  # of a sum over rows, relative to the terms' magnitudes
        if dy is not None:
            e = dy * weight
            back, eback = pre.back(e, F32 * np.abs(e))
            dx = dx + back
            edx = eback + F32 * (np.abs(dx) + np.abs(back))
        out["dx"], err["dx"] = dx, edx

        def column(name, terms, errors):
            out[name] = terms.sum(0)
            err[name] = (errors + total * np.abs(terms)).sum(0)

        if weight is not None:
            y = zero if dy is None else dy
            column("dweight", y * pre.hat, np.abs(y) * pre.ehat)
            if bias is not None:
                column("dbias", y, zero)
        if b is not None:
            dp = scale * g * dx
            edp = np.abs(scale * g) * edx + 3 * F32 * np.abs(dp)
            out["db"], err["db"] = dp, edp
            if norm is not None:
                f = dp * w
                out["db"], err["db"] = norm.back(f, edp * np.abs(w) + F32 * np.abs(f))
                column("dpost_weight", dp * hat, edp * np.abs(hat) + np.abs(dp) * ehat + 4 * F32 * np.abs(dp * hat))
                if post_bias is not None:
                    column("dpost_bias", dp, edp)
            if gate is not None:
                dgate = scale * dx * p
                size = np.abs(scale * dx) * (np.abs(hat * w) + np.abs(o))
                edgate = abs(scale) * (edx * np.abs(p) + np.abs(dx) * ep) + 6 * F32 * size
                if gate.ndim == 2:
                    out["dgate"], err["dgate"] = dgate, edgate
                else:  # (its two sums, times post_weight and post_bias, may cancel)
                    column("dgate", dgate, edgate + total * size)
    out["bound"] = {t: 1.02 * err[t] + u * np.abs(out[t]) + max(tiny, LEAST) for t in err}
    return out
