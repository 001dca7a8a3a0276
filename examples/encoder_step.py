"""One fine-tuning step of a small causal encoder under the ColTrast loss, and a question encoded token
by token over a cache.

    python -m examples.encoder_step      (from the repository root)

The encoder is one attention layer with grouped heads over packed sequences: questions and documents
lie one after another without padding, in the CSR layout that the losses and the search read.  Its
projections are frozen and fine-tuned through low-rank adapters:

    adapter_linear (queries, keys, values) -> rotary -> packed_attention -> adapter_linear (output)
    -> unit rows -> coltrast_total_loss

`answer_tokens` runs the same layer one token at a time, its keys and values in a cache with room.
"""

import torch

import paper_2505_04846_amd as hpr


class Encoder:
    """hidden -> heads of dim -> out, with frozen weights and adapters of rank `rank`."""

    def __init__(self, hidden=256, heads=8, kv_heads=2, dim=64, out=128, rank=8, n_adapters=1,
                 positions=2048, device="cuda:0", seed=0):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        wide = (heads + 2 * kv_heads) * dim

        def weight(*shape, std):
            return (torch.randn(shape, generator=g) * std).to(torch.bfloat16).to(device)

        self.w_qkv = weight(wide, hidden, std=hidden ** -0.5)
        self.w_out = weight(out, heads * dim, std=(heads * dim) ** -0.5)
        # as usual for such adapters, A is random and B starts at zero
        self.adapters = [weight(n_adapters, rank, hidden, std=hidden ** -0.5),
                         torch.zeros(n_adapters, wide, rank, dtype=torch.bfloat16, device=device),
                         weight(n_adapters, rank, heads * dim, std=(heads * dim) ** -0.5),
                         torch.zeros(n_adapters, out, rank, dtype=torch.bfloat16, device=device)]
        for p in self.adapters:
            p.requires_grad_()
        self.scale = torch.full((n_adapters,), 2.0, device=device)
        half = dim // 2
        freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
        angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq
        self.cos, self.sin = angle.cos().float().to(device), angle.sin().float().to(device)

    def project(self, x, pos, off, adapter):
        """Rotated queries and keys, and values, of packed rows x [n, hidden]."""
        qkv = hpr.adapter_linear(x, self.w_qkv, *self.adapters[:2], self.scale, off, adapter)
        qkv = qkv.view(x.shape[0], -1, self.dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        q, k = hpr.rotary(q, k, pos, self.cos, self.sin)
        return q, k, v

    def output(self, a, off, adapter):
        """Unit token embeddings of the attention's output."""
        y = hpr.adapter_linear(a.reshape(a.shape[0], -1), self.w_out, *self.adapters[2:], self.scale,
                               off, adapter)
        return torch.nn.functional.normalize(y.float(), dim=-1).to(y.dtype)

    def __call__(self, x, off, req_off, adapter):
        """Token embeddings of packed sequences; the rows req_off[s]..req_off[s+1] use adapter[s]."""
        n = x.shape[0]
        seq = torch.searchsorted(off[1:].contiguous(), torch.arange(n, device=x.device), right=True)
        pos = (torch.arange(n, device=x.device) - off[seq]).to(torch.int32)
        q, k, v = self.project(x, pos, req_off, adapter)
        return self.output(hpr.packed_attention(q, k, v, off), req_off, adapter)


def train_step(enc, x, n_questions, question_len, doc_lens, pos_idx, logit_scale=1.5625, tau=0.05,
               lr=0.0):
    """Loss and adapter gradients of one batch: x [n, hidden] holds the questions' tokens, then the
    documents'.  With lr, the adapters take one step along them."""
    dev = x.device
    lens = [question_len] * n_questions + list(doc_lens)
    off = torch.tensor([0] + lens, dtype=torch.int64).cumsum(0).to(dev)
    req = torch.tensor([0, x.shape[0]], dtype=torch.int64, device=dev)  # one adapter for all rows
    emb = enc(x, off, req, torch.zeros(1, dtype=torch.int32, device=dev))
    rows = n_questions * question_len
    Q = emb[:rows].view(n_questions, question_len, -1)
    D, d_off = emb[rows:], off[n_questions:] - rows
    loss = hpr.coltrast_total_loss(Q, D.contiguous(), d_off.contiguous(), pos_idx, logit_scale, tau)
    grads = torch.autograd.grad(loss, enc.adapters)
    if lr:
        with torch.no_grad():
            for p, g in zip(enc.adapters, grads):
                p -= lr * g
    return loss.detach(), grads


@torch.no_grad()
def answer_tokens(enc, x, adapter, room):
    """The layer's embeddings of n_seq sequences x [n_seq, steps, hidden], one token of each at a time
    against caches of `room` rows; adapter int32 [n_seq]."""
    n_seq, steps, _ = x.shape
    dev = x.device
    kc = torch.empty(n_seq * room, enc.kv_heads, enc.dim, dtype=x.dtype, device=dev)
    vc = torch.empty_like(kc)
    each = torch.arange(n_seq + 1, device=dev)
    first = each[:-1] * room
    out = []
    for t in range(steps):
        q, k, v = enc.project(x[:, t].contiguous(),
                              torch.full((n_seq,), t, dtype=torch.int32, device=dev), each, adapter)
        kc[first + t], vc[first + t] = k, v
        a = hpr.packed_attention(q, kc, vc, each, k_off=each * room,
                                 k_len=torch.full((n_seq,), t + 1, dtype=torch.int64, device=dev))
        out.append(enc.output(a, each, adapter))
    return torch.stack(out, 1)


def main():
    g = torch.Generator().manual_seed(1)
    enc = Encoder()
    n_q, lq, docs = 8, 32, [40, 200, 64, 97, 33, 150, 128, 71, 55, 180, 60, 90]
    x = torch.randn(n_q * lq + sum(docs), 256, generator=g).to(torch.bfloat16).to("cuda:0")
    pos = torch.arange(n_q, dtype=torch.int32, device="cuda:0")
    for step in range(5):
        loss, grads = train_step(enc, x, n_q, lq, docs, pos, lr=0.03)
        print(f"step {step}: loss {loss.item():.4f}, |dB| {grads[1].float().norm().item():.4f}")
    one = answer_tokens(enc, x[:2 * lq].view(2, lq, -1), torch.zeros(2, dtype=torch.int32,
                                                                     device="cuda:0"), room=64)
    print("token by token:", tuple(one.shape))


if __name__ == "__main__":
    main()
