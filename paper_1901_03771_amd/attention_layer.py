"""A causal attention layer on the lazy arrays: projections as recorded products, rotary positions, attention and its
gradient on packed documents, weights updated in place, and generation of single tokens against a cache.

    python -m paper_1901_03771_amd.attention_layer

trains the layer for a few steps to repeat each document's tokens two places later and then generates with it; it
prints the loss per step and how far generated rows are from those of a whole forward pass.  float32 throughout: the
projections are the lazy arrays' own products."""
from __future__ import annotations

import torch

from . import lazy as gr


class AttentionLayer:
    """y = attention(rotary(x Wq), rotary(x Wk), x Wv) Wo; x (B, N, width), `heads` heads of `values` values on `shared` heads of k and v."""

    def __init__(self, ctx: gr.Context, width: int, heads: int, shared: int, values: int, cap: float = 0.0, seed: int = 0):
        self.ctx, self.width, self.heads, self.shared, self.values, self.cap = ctx, width, heads, shared, values, cap
        g = torch.Generator().manual_seed(seed)
        device = f"cuda:{ctx.device}"
        self.weights = {name: (torch.randn(rows, cols, generator=g) * rows ** -0.5).to(device) for name, rows, cols in
                        (("q", width, heads * values), ("k", width, shared * values), ("v", width, shared * values), ("o", heads * values, width))}
        self._w = {name: ctx.array(t) for name, t in self.weights.items()}
        self.frequencies = gr.rotary_frequencies(values)

    def _projected(self, x, name: str, shape):
        return gr.reshape(gr.dot(x, self._w[name]), shape)

    def forward(self, x, positions, documents):
        """Returns y (B * N, width), unevaluated, and what the gradient needs."""
        B, N, _ = x.shape
        lx = self.ctx.array(x.view(B * N, self.width))
        q = gr.rotary(self._projected(lx, "q", (B, N, self.heads, self.values)), self.frequencies, positions)
        k = gr.rotary(self._projected(lx, "k", (B, N, self.shared, self.values)), self.frequencies, positions)
        v = self._projected(lx, "v", (B, N, self.shared, self.values)).materialize()
        scores = self.ctx.scores(cap=self.cap, causal=True, documents=documents)
        out, lse = gr.attention(q, k, v, scores)
        y = gr.dot(gr.reshape(out, (B * N, self.heads * self.values)), self._w["o"])
        return y, (lx, positions, scores, q, k, v, out, lse)

    def gradients(self, dy, kept):
        """The weights' gradients, unevaluated, for the gradient `dy` (B * N, width) of y."""
        lx, positions, scores, q, k, v, out, lse = kept
        B, N = q.shape[:2]
        flat = gr.reshape(out, (B * N, self.heads * self.values)).materialize()
        dout = gr.reshape(gr.dot(dy, self._w["o"].T), (B, N, self.heads, self.values))
        dq, dk, dv = gr.attention_grad(dout, q, k, v, scores, out, lse)
        for d in (dq, dk):
            gr.rotary(d, self.frequencies, positions, inverse=True, out=d)   # back through the turn, in place
        rows = B * N
        return {"o": gr.dot(flat.T, dy),
                "q": gr.dot(lx.T, gr.reshape(dq, (rows, self.heads * self.values)).materialize()),
                "k": gr.dot(lx.T, gr.reshape(dk, (rows, self.shared * self.values)).materialize()),
                "v": gr.dot(lx.T, gr.reshape(dv, (rows, self.shared * self.values)).materialize())}

    def train_step(self, x, target, positions, documents, rate: float) -> float:
        """One step of gradient descent on the mean square of y - target; returns it."""
        rows = x.shape[0] * x.shape[1]
        y, kept = self.forward(x, positions, documents)
        off = (y - self.ctx.array(target.view(rows, self.width))).materialize()
        loss = (off * off).sum()
        grads = self.gradients((off * (2.0 / (rows * self.width))).materialize(), kept)
        for g in grads.values():
            g.materialize()
        for name, g in grads.items():
            self._w[name][:, :] = self._w[name] - g * rate
        return float(loss.numpy()) / (rows * self.width)

    def step(self, x, cache_k, cache_v, lengths):
        """The next token x (B, width) of each sequence: its k and v go into row lengths[b] of the caches (B, M, shared, values), lengths (i32)
        grows by one, and y (B, width) comes back as a tensor."""
        B = x.shape[0]
        lx = self.ctx.array(x)
        positions = self.ctx.array(lengths.view(B, 1))
        q = gr.rotary(self._projected(lx, "q", (B, 1, self.heads, self.values)), self.frequencies, positions)
        k = gr.rotary(self._projected(lx, "k", (B, 1, self.shared, self.values)), self.frequencies, positions)
        v = self._projected(lx, "v", (B, 1, self.shared, self.values))
        each, at = torch.arange(B, device=x.device), lengths.long()
        cache_k[each, at] = k.torch(copy=False)[:, 0]
        cache_v[each, at] = v.torch(copy=False)[:, 0]
        lengths += 1
        out = gr.attention_step(self.ctx.array(q.torch(copy=False)[:, 0]), self.ctx.array(cache_k), self.ctx.array(cache_v),
                                self.ctx.scores(cap=self.cap, lengths=self.ctx.array(lengths)))
        return gr.dot(gr.reshape(out, (B, self.heads * self.values)), self._w["o"]).torch()


def packed_documents(batch: int, rows: int, device, seed: int = 0):
    """Document numbers (B, N) of ragged pieces and each token's place in its own."""
    g = torch.Generator().manual_seed(seed)
    cuts = torch.zeros(batch, rows, dtype=torch.int32)
    cuts.scatter_(1, torch.randint(1, rows, (batch, 3), generator=g), 1)
    ids = torch.cumsum(cuts, 1, dtype=torch.int32)
    start = torch.where(cuts.bool() | (torch.arange(rows) == 0), torch.arange(rows), 0).cummax(1)[0]
    return ids.to(device), (torch.arange(rows) - start).to(torch.int32).to(device)


def main():
    ctx = gr.Context()
    layer = AttentionLayer(ctx, width=64, heads=4, shared=2, values=32, cap=30.0)
    device = f"cuda:{ctx.device}"
    ids, places = packed_documents(2, 256, device)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2, 256, 64, generator=g).to(device)
    target = torch.where(places[..., None] >= 2, x.roll(2, 1), torch.zeros_like(x))
    documents, positions = ctx.array(ids), ctx.array(places)
    for i in range(8):
        print(f"step {i}: mean square {layer.train_step(x, target, positions, documents, rate=20.0):.4f}", flush=True)
    one = x[:, :32].contiguous()
    whole, _ = layer.forward(one, 0, None)
    whole = whole.torch().view(2, 32, 64)
    cache = [torch.full((2, 40, 2, 32), float("nan"), device=device) for _ in range(2)]   # rows that hold nothing yet have no say
    lengths = torch.zeros(2, dtype=torch.int32, device=device)
    rows = torch.stack([layer.step(one[:, i].contiguous(), *cache, lengths) for i in range(32)], 1)
    print(f"generated rows differ from the forward pass by {float((rows - whole).abs().max()):.2e} at most")
    ctx.close()


if __name__ == "__main__":
    main()
