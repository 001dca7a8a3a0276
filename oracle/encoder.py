"""The encoder's operators in fp64: attention over packed sequences, a projection with low-rank
adapters, and rotation by position, each with its gradients from the formulas.

The attention and adapter functions also return, entry by entry, how far a computation that rounds
its intermediate operands to a type of unit roundoff `u` (off by `tiny` below its normal range) and
sums in fp32 may be from the exact value: `bound` in each result, which the tests hold the GPU to.
Numbers below fp32's normal range (2^-126) may come out as zero, entry by entry.
"""

import numpy as np

F32 = 2.0 ** -24  # unit roundoff of fp32
LEAST = 2.0 ** -126  # its least normal number


def visible(lq, lk, causal, window):
    """Boolean [lq, lk]: query i sees key j."""
    i = np.arange(lq)[:, None] + (lk - lq)
    j = np.arange(lk)[None]
    see = np.ones((lq, lk), bool)
    if causal:
        see &= j <= i
        if window:
            see &= j > i - window
    return see


def packed_attention(q, k, v, q_off, k_off, k_len, causal, window, scale, dout=None, u=0.0,
                     tiny=0.0):
    """q [n_q, H, D], k and v [n_k, Hk, D] (fp64).  dict(out, lse[, dq, dk, dv], bound), bound a
    dict of the same names (lse's too)."""
    tiny = max(tiny, LEAST)
    n_q, H, D = q.shape
    Hk = k.shape[1]
    G = H // Hk
    names = ["out", "lse"] + (["dq", "dk", "dv"] if dout is not None else [])
    shape = {"out": q.shape, "lse": q.shape[:2], "dq": q.shape, "dk": k.shape, "dv": k.shape}
    r = {n: np.zeros(shape[n]) for n in names}
    b = {n: np.zeros(shape[n]) for n in names}
    r["lse"][:] = -np.inf
    for s in range(len(q_off) - 1):
        q0, q1 = int(q_off[s]), int(q_off[s + 1])
        k0, k1 = int(k_off[s]), int(k_off[s + 1])
        if k_len is not None:
            k1 = min(k1, k0 + int(k_len[s]))
        if q1 <= q0 or k1 <= k0:
            continue
        see = visible(q1 - q0, k1 - k0, causal, window)
        for h in range(H):
            Q, K, V = q[q0:q1, h], k[k0:k1, h // G], v[k0:k1, h // G]
            x = scale * (Q @ K.T)
            size = scale * (np.abs(Q) @ np.abs(K).T)
            x = np.where(see, x, -np.inf)
            top = x.max(1, keepdims=True)
            some = np.isfinite(top)
            top = np.where(some, top, 0.0)
            e = np.where(see, np.exp(x - top), 0.0)
            total = e.sum(1, keepdims=True)
            p = e / np.where(total == 0, 1.0, total)
            o = p @ V
            r["out"][q0:q1, h] = o
            with np.errstate(divide="ignore"):
                lse = np.where(some, top + np.log(np.where(total == 0, 1.0, total)), -np.inf)
            r["lse"][q0:q1, h] = lse[:, 0]
            # relative error of a computed exponential and of its row's total: the product's fp32
            # sum, the scaling and the subtraction of the maximum (in powers of two), and exp2 and
            # log2 themselves, each a few units
            size = np.where(see, size, 0.0)
            reach = size.max(1, keepdims=True)
            rel = 2.0 * F32 * ((D + 4) * reach + 4 * (np.abs(top) + reach) + 16 + (k1 - k0) ** 0.5)
            av = p @ np.abs(V)
            out_err = (u + rel) * av * 1.01 + (k1 - k0) * F32 * av + u * np.abs(o)
            out_err += tiny * (1 + see @ np.abs(V))
            b["out"][q0:q1, h] = out_err
            b["lse"][q0:q1, h] = (rel + 4 * F32 * (1 + np.abs(np.where(some, lse, 0.0))))[:, 0]
            if dout is None:
                continue
            g = dout[q0:q1, h]
            dp = g @ V.T
            adp = np.abs(g) @ np.abs(V).T
            delta = (g * o).sum(1, keepdims=True)
            ds = p * (dp - delta)
            r["dv"][k0:k1, h // G] += p.T @ g
            r["dq"][q0:q1, h] = scale * (ds @ K)
            r["dk"][k0:k1, h // G] += scale * (ds.T @ Q)
            rel = rel + 4 * F32 * (1 + np.abs(np.where(some, lse, 0.0)))  # p again, from lse
            n_i, n_j = G * (q1 - q0), k1 - k0
            b["dv"][k0:k1, h // G] += 1.01 * ((u + rel).T * p.T + n_i * F32 * p.T + tiny * see.T) @ np.abs(
                g)
            # delta is of the rounded output; dp - delta is formed in fp32
            d_err = (np.abs(g) * out_err).sum(1, keepdims=True) + D * F32 * (np.abs(g) * np.abs(o)).sum(
                1, keepdims=True)
            ds_err = (u + rel) * np.abs(ds) + p * (d_err + (D + 2) * F32 * adp + F32 * np.abs(delta))
            ds_err += tiny * see
            b["dq"][q0:q1, h] = 1.01 * scale * (ds_err + n_j * F32 * np.abs(ds)) @ np.abs(K)
            b["dk"][k0:k1, h // G] += 1.01 * scale * (ds_err + n_i * F32 * np.abs(ds)).T @ np.abs(Q)
    for n in ("dq", "dk", "dv"):
        if n in r:
            b[n] += u * np.abs(r[n]) + tiny
    r["bound"] = b
    return r


def adapter_linear(x, W, A, B, scale, off, adapter, dy=None, u=0.0, tiny=0.0):
    """x [n, k], W [m, k], A [n_ad, r, k], B [n_ad, m, r] (fp64).  dict(y[, dx, da, db], bound)."""
    tiny = max(tiny, LEAST)
    n, k = x.shape
    m = W.shape[0]
    y = x @ W.T
    by = k * F32 * (np.abs(x) @ np.abs(W).T)
    r = {"y": y}
    bound = {"y": by}
    if dy is not None:
        r.update(dx=dy @ W, da=np.zeros_like(A), db=np.zeros_like(B))
        bound.update(dx=m * F32 * (np.abs(dy) @ np.abs(W)), da=np.zeros_like(A), db=np.zeros_like(B))
    for s, a in enumerate(adapter):
        t = slice(int(off[s]), int(off[s + 1]))
        rows = t.stop - t.start
        if a < 0 or a >= len(A) or rows <= 0:
            continue
        h = scale[a] * (x[t] @ A[a].T)
        eh = tiny + u * np.abs(h) + (k + 2) * F32 * abs(scale[a]) * (np.abs(x[t]) @ np.abs(A[a]).T)
        rank = A.shape[1]
        y[t] += h @ B[a].T
        by[t] += (1.01 * eh + (rank + 1) * F32 * np.abs(h)) @ np.abs(B[a]).T
        if dy is None:
            continue
        g = scale[a] * (dy[t] @ B[a])
        eg = tiny + u * np.abs(g) + (m + 2) * F32 * abs(scale[a]) * (np.abs(dy[t]) @ np.abs(B[a]))
        r["dx"][t] += g @ A[a]
        bound["dx"][t] += (1.01 * eg + (rank + 1) * F32 * np.abs(g)) @ np.abs(A[a])
        r["da"][a] += g.T @ x[t]
        bound["da"][a] += (1.01 * eg + n * F32 * np.abs(g)).T @ np.abs(x[t])
        r["db"][a] += dy[t].T @ h
        bound["db"][a] += np.abs(dy[t]).T @ (1.01 * eh + n * F32 * np.abs(h))
    for name in bound:
        bound[name] = bound[name] + u * np.abs(r[name]) + tiny
    r["bound"] = bound
    return r


def rotary(x, pos, cos, sin, inverse=False):
    """x [n, heads, dim] (fp64) rotated by its rows' positions."""
    half = cos.shape[1]
    c, s = cos[pos][:, None], (-sin if inverse else sin)[pos][:, None]
    a, b = x[..., :half], x[..., half:2 * half]
    return np.concatenate([a * c - b * s, b * c + a * s, x[..., 2 * half:]], -1)
