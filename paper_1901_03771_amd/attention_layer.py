"""A causal attention layer on the lazy arrays: projections as recorded products, rotary positions, attention and its
gradient on packed documents, weights updated in place, and generation of single tokens against a cache.

    python -m paper_1901_03771_amd.attention_layer

trains the layer for a few steps to repeat each document's tokens two places later and then generates with it; it
prints the loss per step and how far generated rows are from those of a whole forward pass.  float32 throughout: the
projections are the lazy arrays' own products.

    python -m paper_1901_03771_amd.attention_layer --norm --eight

the same with a norm in front of the projections, whose gain is trained too, and with the projections of training and of
generation as products of 8-bit tensors (attention and the weights that are updated stay in float32)."""
from __future__ import annotations

import sys

import torch

from . import lazy as gr


class AttentionLayer:
    """y = attention(rotary(x Wq), rotary(x Wk), x Wv) Wo; x (B, N, width), `heads` heads of `values` values on `shared` heads of k and v.
    norm: x / sqrt(mean(x ** 2)) * gain in its place.  eight: products of 8-bit tensors with scales, forward and backward.
    Every call takes the tensors in `weights` as they are then, whoever has written into them."""

    def __init__(self, ctx: gr.Context, width: int, heads: int, shared: int, values: int, cap: float = 0.0, seed: int = 0, norm: bool = False, eight: bool = False):
        self.ctx, self.width, self.heads, self.shared, self.values, self.cap = ctx, width, heads, shared, values, cap
        self.norm, self.eight = norm, eight
        g = torch.Generator().manual_seed(seed)
        device = f"cuda:{ctx.device}"
        self.weights = {name: (torch.randn(rows, cols, generator=g) * rows ** -0.5).to(device) for name, rows, cols in
                        (("q", width, heads * values), ("k", width, shared * values), ("v", width, shared * values), ("o", heads * values, width))}
        if norm:
            self.weights["gain"] = torch.ones(width, device=device)
        self._w = {name: ctx.array(t) for name, t in self.weights.items()}
        self.frequencies = gr.rotary_frequencies(values)

    def _weight8(self, name: str, transposed: bool):
        """The weight in 8 bits, in blocks: (columns, rows) for products with it, or as it lies for those with its transpose."""
        return gr.quantize(self._w[name], blocks=True, transposed=transposed)

    def laid_out(self):
        """The weights in 8 bits as `forward` and `step` take them, for a program that makes many calls of weights that stay; None without eight.  They are those of now:
        the layer keeps none, and after a change of the weights the program lays them out again."""
        return {name: self._weight8(name, True) for name in "qkvo"} if self.eight else None

    def _product(self, x, name: str, laid=None):
        """x W; with eight, x may come as (values, scales) already."""
        if laid is not None and not self.eight:
            raise ValueError("weights in 8 bits for a layer in float32")
        if not self.eight:
            return gr.dot(x, self._w[name])
        q, s = x if isinstance(x, tuple) else gr.quantize(x)
        return gr.dot_scaled(q, s, *(laid[name] if laid else self._weight8(name, True)), dtype=gr.GR_F32)

    def _product_back(self, dy, name: str):
        """dy W'."""
        if not self.eight:
            return gr.dot(dy, self._w[name].T)
        return gr.dot_scaled(*gr.quantize(dy), *self._weight8(name, False), dtype=gr.GR_F32)

    def _weight_gradient(self, x, dy):
        """x' dy: with eight, sums over tokens of both sides' columns in 8 bits."""
        if not self.eight:
            return gr.dot(x.T, dy)
        return gr.dot_scaled(*gr.quantize(x, transposed=True), *gr.quantize(dy, transposed=True), dtype=gr.GR_F32)

    def _normed(self, lx):
        """What the projections take of the rows lx; with eight, (values, scales), which all of them share."""
        if not self.norm:
            return gr.quantize(lx) if self.eight else lx
        h, _, scales = gr.rms_norm(lx, self._w["gain"], eight=self.eight)
        return (h, scales) if self.eight else h

    def _projected(self, x, name: str, shape, laid):
        return gr.reshape(self._product(x, name, laid), shape)

    def forward(self, x, positions, documents, laid=None):
        """Returns y (B * N, width), unevaluated, and what the gradient needs.  laid: the weights as `laid_out` gave them, in place of those of now."""
        B, N, _ = x.shape
        lx = self.ctx.array(x.view(B * N, self.width))
        h = self._normed(lx)
        q = gr.rotary(self._projected(h, "q", (B, N, self.heads, self.values), laid), self.frequencies, positions)
        k = gr.rotary(self._projected(h, "k", (B, N, self.shared, self.values), laid), self.frequencies, positions)
        v = self._projected(h, "v", (B, N, self.shared, self.values), laid).materialize()
        scores = self.ctx.scores(cap=self.cap, causal=True, documents=documents)
        out, lse = gr.attention(q, k, v, scores)
        y = self._product(gr.reshape(out, (B * N, self.heads * self.values)), "o", laid)
        return y, (lx, h, positions, scores, q, k, v, out, lse)

    def gradients(self, dy, kept):
        """The weights' gradients, unevaluated, for the gradient `dy` (B * N, width) of y."""
        lx, h, positions, scores, q, k, v, out, lse = kept
        B, N = q.shape[:2]
        flat = gr.reshape(out, (B * N, self.heads * self.values)).materialize()
        dout = gr.reshape(self._product_back(dy, "o"), (B, N, self.heads, self.values))
        dq, dk, dv = gr.attention_grad(dout, q, k, v, scores, out, lse)
        for d in (dq, dk):
            gr.rotary(d, self.frequencies, positions, inverse=True, out=d)   # back through the turn, in place
        rows = B * N
        d = {name: gr.reshape(g, (rows, heads * self.values)).materialize() for name, g, heads in (("q", dq, self.heads), ("k", dk, self.shared), ("v", dv, self.shared))}
        if self.eight:   # (by rows is not how a sum over tokens takes them)
            h = gr.rms_norm(lx, self._w["gain"])[0] if self.norm else lx
        grads = {"o": self._weight_gradient(flat, dy), **{name: self._weight_gradient(h, g) for name, g in d.items()}}
        if self.norm:
            dh = (self._product_back(d["q"], "q") + self._product_back(d["k"], "k")) + self._product_back(d["v"], "v")
            grads["gain"] = gr.rms_norm_grad(dh, lx, self._w["gain"])[1]
        return grads

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
            w = self._w[name]
            w[tuple([slice(None)] * w.ndim)] = w - g * rate
        return float(loss.numpy()) / (rows * self.width)

    def step(self, x, cache_k, cache_v, lengths, laid=None):
        """The next token x (B, width) of each sequence: its k and v go into row lengths[b] of the caches (B, M, shared, values), lengths (i32)
        grows by one, and y (B, width) comes back as a tensor.  laid: as for `forward`."""
        B = x.shape[0]
        h = self._normed(self.ctx.array(x))
        positions = self.ctx.array(lengths.view(B, 1))
        q = gr.rotary(self._projected(h, "q", (B, 1, self.heads, self.values), laid), self.frequencies, positions)
        k = gr.rotary(self._projected(h, "k", (B, 1, self.shared, self.values), laid), self.frequencies, positions)
        v = self._projected(h, "v", (B, 1, self.shared, self.values), laid)
        each, at = torch.arange(B, device=x.device), lengths.long()
        cache_k[each, at] = k.torch(copy=False)[:, 0]
        cache_v[each, at] = v.torch(copy=False)[:, 0]
        lengths += 1
        out = gr.attention_step(self.ctx.array(q.torch(copy=False)[:, 0]), self.ctx.array(cache_k), self.ctx.array(cache_v),
                                self.ctx.scores(cap=self.cap, lengths=self.ctx.array(lengths)))
        return self._product(gr.reshape(out, (B, self.heads * self.values)), "o", laid).torch()


def packed_documents(batch: int, rows: int, device, seed: int = 0):
    """Document numbers (B, N) of ragged pieces and each token's place in its own."""
    g = torch.Generator().manual_seed(seed)
    cuts = torch.zeros(batch, rows, dtype=torch.int32)
    cuts.scatter_(1, torch.randint(1, rows, (batch, 3), generator=g), 1)
    ids = torch.cumsum(cuts, 1, dtype=torch.int32)
    start = torch.where(cuts.bool() | (torch.arange(rows) == 0), torch.arange(rows), 0).cummax(1)[0]
    return ids.to(device), (torch.arange(rows) - start).to(torch.int32).to(device)


def main(arguments=()):
    ctx = gr.Context()
    layer = AttentionLayer(ctx, width=64, heads=4, shared=2, values=32, cap=30.0, norm="--norm" in arguments, eight="--eight" in arguments)
    device = f"cuda:{ctx.device}"
    ids, places = packed_documents(2, 256, device)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2, 256, 64, generator=g).to(device)
    target = torch.where(places[..., None] >= 2, x.roll(2, 1), torch.zeros_like(x))
    documents, positions = ctx.array(ids), ctx.array(places)
    for i in range(8):
        print(f"step {i}: mean square {layer.train_step(x, target, positions, documents, rate=20.0):.4f}", flush=True)
    one = x[:, :32].contiguous()
    laid = layer.laid_out()   # generation leaves the weights as they are
    whole, _ = layer.forward(one, 0, None, laid)
    whole = whole.torch().view(2, 32, 64)
    cache = [torch.full((2, 40, 2, 32), float("nan"), device=device) for _ in range(2)]   # rows that hold nothing yet have no say
    lengths = torch.zeros(2, dtype=torch.int32, device=device)
    rows = torch.stack([layer.step(one[:, i].contiguous(), *cache, lengths, laid) for i in range(32)], 1)
    print(f"generated rows differ from the forward pass by {float((rows - whole).abs().max()):.2e} at most")
    ctx.close()


if __name__ == "__main__":
    main(sys.argv[1:])
