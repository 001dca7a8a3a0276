"""The rest of the encoder's block beside attention, as cases that can be timed and compared.

A case is a dict of plain values; its "op" says which operator one pass goes through:

  gated       the gated feed-forward projections and their product, h = act(x Wg^T) * (x Wu^T):
              "forward", or with its gradients ("train"), of the rows and the weights or, with the
              weights frozen, of the rows alone; with "packed" the backward pass reads x from a
              checkpoint in 8 bits that the pass makes
  norm        the norm after a block, its gate and residual scale, the residual sum and the norm
              before the next block, in one operator: "forward", or with its gradients ("train");
              with "packed" the backward pass reads the residual and the block's output from
              checkpoints in 8 bits that the pass makes
  checkpoint  rows packed into 8 bits with an exponent for every 32 values, and read back

`run` goes through the framework's entry points where `own` is true, and through elementary torch
operations in 32 bits, rounded once at the end, where it is false.
"""

import math
import random

import torch

DEV = "cuda:0"
own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_EPS = {"rms": 1e-6, "layer": 1e-5}


def listed():
    return [
        # One short question in the smaller encoder (latency).
        {"name": "gated_question", "op": "gated", "dir": "forward", "rows": 7, "cols": 768,
         "width": 2304, "act": "gelu", "dtype": "f16", "frozen": True, "packed": False},
        # One token of each of 32 answers: all of the weights are read for 32 rows.
        {"name": "gated_token", "op": "gated", "dir": "forward", "rows": 32, "cols": 4096,
         "width": 14336, "act": "silu", "dtype": "bf16", "frozen": True, "packed": False},
        # Encoding a store: the rows of 64 chunks of 32 to 384 tokens.
        {"name": "gated_chunks", "op": "gated", "dir": "forward", "rows": 13063, "cols": 4096,
         "width": 14336, "act": "silu", "dtype": "bf16", "frozen": True, "packed": False},
        # Fine-tuning every weight: a batch of 24 questions and 24 chunks.
        {"name": "gated_train", "op": "gated", "dir": "train", "rows": 6529, "cols": 4096,
         "width": 14336, "act": "silu", "dtype": "bf16", "frozen": False, "packed": False},
        # Fine-tuning adapters beside frozen weights, the rows kept in 8 bits for the backward pass.
        {"name": "gated_train_packed", "op": "gated", "dir": "train", "rows": 4001, "cols": 4096,
         "width": 14336, "act": "silu", "dtype": "bf16", "frozen": True, "packed": True},
        # The smaller encoder's batch of a few short requests in fp16, with all gradients.
        {"name": "gated_train_small", "op": "gated", "dir": "train", "rows": 764, "cols": 768,
         "width": 2304, "act": "gelu", "dtype": "f16", "frozen": False, "packed": False},
        # One token of each of 64 answers (latency).
        {"name": "norm_token", "op": "norm", "dir": "forward", "rows": 64, "cols": 4096,
         "kind": "rms", "post": True, "gate": "vector", "scale": 0.5, "dtype": "bf16",
         "packed": False},
        # A store's batch with its gradients, norms on both sides of the block and a learned gate.
        {"name": "norm_train", "op": "norm", "dir": "train", "rows": 53248, "cols": 4096,
         "kind": "rms", "post": True, "gate": "vector", "scale": 0.5, "dtype": "bf16",
         "packed": False},
        # The bidirectional encoder: residual sum and layer norm with biases, fp16.
        {"name": "norm_train_layer", "op": "norm", "dir": "train", "rows": 32749, "cols": 768,
         "kind": "layer", "post": False, "gate": "none", "scale": 1.0, "dtype": "f16",
         "packed": False},
        # A fine-tuning batch, residual and block output kept in 8 bits for the backward pass.
        {"name": "norm_train_packed", "op": "norm", "dir": "train", "rows": 13057, "cols": 4096,
         "kind": "rms", "post": True, "gate": "rows", "scale": 1.0, "dtype": "bf16",
         "packed": True},
        # The activations of a store's batch, kept and read back.
        {"name": "checkpoint_chunks", "op": "checkpoint", "rows": 53248, "cols": 4096,
         "dtype": "bf16"},
        # The smaller encoder's few rows (latency).
        {"name": "checkpoint_small", "op": "checkpoint", "rows": 764, "cols": 768, "dtype": "f16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated", "gated", "gated", "norm", "norm", "checkpoint"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "checkpoint":
        return {"op": op, "rows": _log_int(rng, 1, 53248),
                "cols": rng.choice([128, 768, 1000, 2048, 4096]), "dtype": dtype}
    way = rng.choice(["forward", "train", "train"])
    if op == "norm":
        c = {"op": op, "dir": way, "rows": _log_int(rng, 1, 53248),
             "cols": rng.choice([256, 768, 1000, 1024, 2048, 4096, 4096, 8192]),
             "kind": rng.choice(["rms", "rms", "layer"]), "post": rng.random() < 0.6,
             "gate": rng.choice(["none", "vector", "rows"]), "scale": rng.choice([1.0, 0.5, 0.125]),
             "dtype": dtype, "packed": way == "train" and rng.random() < 0.4}
        while c["rows"] * c["cols"] > 53248 * 4096:
            c["rows"] //= 2
        return c
    c = {"op": op, "dir": way, "rows": _log_int(rng, 1, 13063),
         "cols": rng.choice([768, 1024, 2048, 4096, 4096]),
         "width": rng.choice([1000, 2304, 4096, 6144, 14336]),
         "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh"]), "dtype": dtype,
         "frozen": way == "forward" or rng.random() < 0.5,
         "packed": way == "train" and rng.random() < 0.4}
    while work(c)["flops"] > 4.6e12:
        c["rows"] //= 2
    return c


# ---- what a case holds ----------------------------------------------------------------------


def work(case):
    n, k = case["rows"], case["cols"]
    if case["op"] == "checkpoint":  # rows read, rows written; an operation to scale, one to round
        return {"bytes": 2 * 2 * n * k, "flops": 4 * n * k}
    train = case["dir"] == "train"
    if case["op"] == "norm":
        # x, b, r, y, and dr, dy, dx, db
        gates = {"none": 0, "vector": k, "rows": n * k}[case["gate"]]
        vectors = k * (1 + case["post"]) * (2 if case["kind"] == "layer" else 1)
        bytes_ = 2 * 4 * n * k + 2 * gates + 2 * vectors
        flops = n * k * (10 + 6 * case["post"])
        if train:
            bytes_, flops = 2 * bytes_, 3 * flops
        return {"bytes": bytes_, "flops": flops}
    f = case["width"]
    weights = 2 * 2 * k * f
    bytes_, flops = 2 * n * (k + f) + weights, 4 * n * k * f
    if train:  # dh in, dx out, and the weights' gradients
        bytes_, flops = bytes_ + 2 * n * (k + f), 2 * flops
        if not case["frozen"]:
            bytes_, flops = bytes_ + weights, flops + 4 * n * k * f
    return {"bytes": bytes_, "flops": flops}


# ---- inputs ---------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std + mean).to(dtype)


def _stream(g, n, k, dtype):
    """A residual stream's rows: a few channels far larger than the others."""
    channels = torch.rand(k, generator=g, device=DEV)
    size = torch.where(channels < 0.01, 20.0, 1.0) * (0.5 + torch.rand(k, generator=g, device=DEV))
    return (torch.randn((n, k), generator=g, device=DEV) * size + 0.1).to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    dt = _TYPES[case["dtype"]]
    n, k = case["rows"], case["cols"]
    st = {"case": case}
    if case["op"] == "checkpoint":
        st["x"] = _stream(g, n, k, dt)
        return st
    train = case["dir"] == "train"
    if case["op"] == "gated":
        f = case["width"]
        st["x"] = _normal(g, n, k, dtype=dt)
        st["wg"] = _normal(g, f, k, dtype=dt, std=k ** -0.5)
        st["wu"] = _normal(g, f, k, dtype=dt, std=k ** -0.5)
        if train:
            st["dh"] = _normal(g, n, f, dtype=dt, std=0.1)
        return st
    st["x"] = _stream(g, n, k, dt)
    st["b"] = _normal(g, n, k, dtype=dt, mean=0.05)
    st["w"] = _normal(g, k, dtype=dt, std=0.2, mean=1.0)
    st["c"] = _normal(g, k, dtype=dt, std=0.1) if case["kind"] == "layer" else None
    st["pw"] = _normal(g, k, dtype=dt, std=0.2, mean=1.0) if case["post"] else None
    st["pc"] = (_normal(g, k, dtype=dt, std=0.1) if case["post"] and case["kind"] == "layer"
                else None)
    shape = {"none": None, "vector": (k,), "rows": (n, k)}[case["gate"]]
    st["gate"] = (torch.rand(shape, generator=g, device=DEV).to(dt) if shape else None)
    if train:
        st["dr"] = _normal(g, n, k, dtype=dt, std=0.1)
        st["dy"] = _normal(g, n, k, dtype=dt, std=0.1)
    return st


# ---- the plain forms ------------------------------------------------------------------------


def _plain_packed(x):
    """The values that x's codes stand for, in 32 bits: for every 32 values of a row 2^e with
    e = floor(log2 max|x|) - 6 (not below the type's smallest step, or 2^-126), and whole numbers
    of at most 127 times it."""
    n, k = x.shape
    wide = -(-k // 32) * 32
    v = torch.zeros((n, wide), device=DEV)
    v[:, :k] = x.float()
    v = v.view(n, wide // 32, 32)
    top = v.abs().amax(-1, keepdim=True)
    # floor(log2) of a normal 32-bit number is its exponent; smaller ones are below every limit
    e = (top.view(torch.int32) >> 23) - 127 - 6
    e = e.clamp(min=-24 if x.dtype == torch.float16 else -126)
    one = ((e + 127) << 23).view(torch.float32)
    inverse = ((127 - e) << 23).view(torch.float32)
    code = torch.round(v * inverse).clamp(-127, 127)
    return (code * one).view(n, wide)[:, :k]


def _plain_checkpoint(st):
    return [_plain_packed(st["x"]).to(st["x"].dtype)]


def _plain_act(name, g):
    """act(g) and its derivative."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        cdf = 0.5 * torch.erfc(g * -math.sqrt(0.5))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    s = 1 / (1 + torch.exp(-2 * c * (g + 0.044715 * g ** 3)))  # (1 + tanh) / 2
    return g * s, s + g * s * (1 - s) * 2 * c * (1 + 3 * 0.044715 * g * g)


def _plain_gated(st):
    case = st["case"]
    dt = st["x"].dtype
    x, wg, wu = st["x"].float(), st["wg"].float(), st["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, slope = _plain_act(case["act"], g)
    out = [(a * u).to(dt)]
    if case["dir"] == "forward":
        return out
    if case["packed"]:
        x = _plain_packed(st["x"])
        g, u = x @ wg.t(), x @ wu.t()
        a, slope = _plain_act(case["act"], g)
    dh = st["dh"].float()
    dg, du = dh * u * slope, dh * a
    out.append((dg @ wg + du @ wu).to(dt))
    if not case["frozen"]:
        out += [(dg.t() @ x).to(dt), (du.t() @ x).to(dt)]
    return out


def _plain_norm_of(v, w, c, kind):
    """The norm, its rows before weight and bias, and the rows' inverse deviation."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    rs = torch.rsqrt((v * v).mean(-1, keepdim=True) + _EPS[kind])
    hat = v * rs
    return hat * w + (0 if c is None else c), hat, rs


def _plain_norm_back(d, hat, rs, w, kind):
    """Gradient with respect to the norm's input, from d with respect to its output."""
    e = d * w
    back = e - hat * (e * hat).mean(-1, keepdim=True)
    if kind == "layer":
        back = back - e.mean(-1, keepdim=True)
    return back * rs


def _column_sum(t):
    """Sums over the rows in runs of 256: one long run in 32 bits loses what the gradients keep."""
    n, k = t.shape
    whole = n // 256 * 256
    s = t[:whole].view(-1, 256, k).sum(1).double().sum(0)
    return s + t[whole:].double().sum(0)


def _plain_residual_norm(st):
    case = st["case"]
    kind, scale, dt = case["kind"], case["scale"], st["x"].dtype
    w, c, pw, pc, gate = [None if st[t] is None else st[t].float()
                          for t in ("w", "c", "pw", "pc", "gate")]
    one = torch.ones((), device=DEV)

    def forward(x, b):
        p, hat, rs = (_plain_norm_of(b, pw, pc, kind) if case["post"] else (b, b, None))
        r = x + scale * (one if gate is None else gate) * p
        y, hat_r, rs_r = _plain_norm_of(r, w, c, kind)
        return p, hat, rs, r, y, hat_r, rs_r

    p, hat, rs, r, y, hat_r, rs_r = forward(st["x"].float(), st["b"].float())
    out = [r.to(dt), y.to(dt)]
    if case["dir"] == "forward":
        return out
    if case["packed"]:
        p, hat, rs, r, y, hat_r, rs_r = forward(_plain_packed(st["x"]), _plain_packed(st["b"]))
    dy = st["dy"].float()
    dx = st["dr"].float() + _plain_norm_back(dy, hat_r, rs_r, w, kind)
    dp = scale * dx * (one if gate is None else gate)
    db = _plain_norm_back(dp, hat, rs, pw, kind) if case["post"] else dp
    out += [dx.to(dt), db.to(dt), _column_sum(dy * hat_r).to(dt)]
    if c is not None:
        out.append(_column_sum(dy).to(dt))
    if pw is not None:
        out.append(_column_sum(dp * hat).to(dt))
    if pc is not None:
        out.append(_column_sum(dp).to(dt))
    if gate is not None:
        dgate = scale * dx * p
        out.append((dgate if case["gate"] == "rows" else _column_sum(dgate)).to(dt))
    return out


# ---- a pass ---------------------------------------------------------------------------------


def _own(st):
    import paper_2505_04846_amd as hpr
    case = st["case"]
    if case["op"] == "checkpoint":
        return [hpr.checkpoint_unpack(hpr.checkpoint_pack(st["x"]))]
    train = case["dir"] == "train"
    if case["op"] == "gated":
        how = (st["wg"], st["wu"], case["act"])
        h = hpr.gated_linear_fwd(st["x"], *how)["h"]
        if not train:
            return [h]
        x = hpr.checkpoint_pack(st["x"]) if case["packed"] else st["x"]
        b = hpr.gated_linear_bwd(st["dh"], x, *how, need_dw=not case["frozen"])
        return [h, b["dx"]] + ([] if case["frozen"] else [b["dw_gate"], b["dw_up"]])
    how = dict(weight=st["w"], bias=st["c"], post_weight=st["pw"], post_bias=st["pc"],
               gate=st["gate"], scale=case["scale"], kind=case["kind"], eps=_EPS[case["kind"]])
    f = hpr.residual_norm_fwd(st["x"], st["b"], **how)
    out = [f["r"], f["y"]]
    if not train:
        return out
    x, b = st["x"], st["b"]
    if case["packed"]:
        x, b = hpr.checkpoint_pack(x), hpr.checkpoint_pack(b)
    g = hpr.residual_norm_bwd(st["dr"], st["dy"], x, b, **how)
    names = ["dx", "db", "dweight"] + ["dbias"] * (st["c"] is not None)
    names += ["dpost_weight"] * (st["pw"] is not None) + ["dpost_bias"] * (st["pc"] is not None)
    return out + [g[t] for t in names + ["dgate"] * (st["gate"] is not None)]


def run(state):
    if own:
        return _own(state)
    return {"gated": _plain_gated, "norm": _plain_residual_norm,
            "checkpoint": _plain_checkpoint}[state["case"]["op"]](state)


# ---- in 64 bits -----------------------------------------------------------------------------


def _exact_packed(x):
    """By mantissa and exponent: max|x| = m 2^q with m in [1/2, 1), so the step is 2^(q - 7)."""
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    least = -24 if x.dtype == torch.float16 else -126
    for j in range(0, x.shape[1], 32):
        part = x[:, j:j + 32].double()
        top = part.abs().max(dim=1).values
        q = torch.frexp(top).exponent - 7
        q = torch.where(top > 0, q, torch.full_like(q, least)).clamp(min=least)
        step = ((q.long() + 1023) << 52).view(torch.float64)[:, None]  # 2^q, without rounding
        out[:, j:j + 32] = torch.clamp(torch.round(part / step), -127, 127) * step
    return out


def _exact_act(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * torch.special.ndtr(g)
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def _exact_gated(st):
    """The definition on blocks of rows, its gradients by automatic differentiation."""
    case = st["case"]
    train, n = case["dir"] == "train", st["x"].shape[0]
    weights = [st[t].double().requires_grad_(train and not case["frozen"]) for t in ("wg", "wu")]
    h, dx = [], []
    dw = [torch.zeros_like(w) for w in weights]
    block = 2048
    for i in range(0, n, block):
        x = st["x"][i:i + block].double()
        with torch.no_grad():
            h.append(_exact_act(case["act"], x @ weights[0].t()) * (x @ weights[1].t()))
        if not train:
            continue
        x = (_exact_packed(st["x"][i:i + block]) if case["packed"] else x).requires_grad_()
        y = _exact_act(case["act"], x @ weights[0].t()) * (x @ weights[1].t())
        of = [x] if case["frozen"] else [x, *weights]
        got = torch.autograd.grad(y, of, st["dh"][i:i + block].double())
        dx.append(got[0])
        for d, more in zip(dw, got[1:]):
            d += more
    return [torch.cat(h)] + ([torch.cat(dx)] if train else []) + (
        dw if train and not case["frozen"] else [])


def _exact_norm(st):
    """The definition by means and variances on blocks of rows, differentiated automatically."""
    case = st["case"]
    n, k = st["x"].shape
    train, eps = case["dir"] == "train", _EPS[case["kind"]]

    def normed(v, w, c):
        if case["kind"] == "rms":
            return v / torch.sqrt(v.square().mean(1, keepdim=True) + eps) * w
        var, mean = torch.var_mean(v, dim=1, correction=0, keepdim=True)
        return (v - mean) / torch.sqrt(var + eps) * w + c

    def define(x, b, w, c, pw, pc, gate):
        part = normed(b, pw, pc) if case["post"] else b
        if gate is not None:
            part = part * gate
        r = x + case["scale"] * part
        return r, normed(r, w, c)

    vectors = {t: st[t].double() for t in ("w", "c", "pw", "pc") if st[t] is not None}
    if case["gate"] == "vector":
        vectors["gate"] = st["gate"].double()
    sums = {t: torch.zeros_like(v) for t, v in vectors.items()}
    rows = {t: [] for t in ("r", "y", "x", "b", "gate")}
    block = max(1, (1 << 24) // k)
    for i in range(0, n, block):
        at = slice(i, i + block)
        a = {t: None for t in ("w", "c", "pw", "pc", "gate")} | vectors
        if case["gate"] == "rows":
            a["gate"] = st["gate"][at].double()
        r, y = define(st["x"][at].double(), st["b"][at].double(), **a)
        rows["r"].append(r)
        rows["y"].append(y)
        if not train:
            continue
        x, b = [_exact_packed(st[t][at]) if case["packed"] else st[t][at].double() for t in "xb"]
        a = {t: None if v is None else v.detach().requires_grad_() for t, v in a.items()}
        leaves = {"x": x.requires_grad_(), "b": b.requires_grad_()}
        leaves |= {t: v for t, v in a.items() if v is not None}
        got = torch.autograd.grad(define(x, b, **a), list(leaves.values()),
                                  (st["dr"][at].double(), st["dy"][at].double()))
        for t, v in zip(leaves, got):
            if t in sums:
                sums[t] += v
            else:
                rows[t].append(v)
    out = [torch.cat(rows["r"]), torch.cat(rows["y"])]
    if train:
        out += [torch.cat(rows["x"]), torch.cat(rows["b"])]
        out += [sums[t] for t in ("w", "c", "pw", "pc") if t in sums]
        if st["gate"] is not None:
            out.append(sums["gate"] if "gate" in sums else torch.cat(rows["gate"]))
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "checkpoint":
        return [_exact_packed(st["x"])]
    return (_exact_gated if case["op"] == "gated" else _exact_norm)(st)
