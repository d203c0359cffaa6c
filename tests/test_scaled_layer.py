"""The layer in 8 bits, call by call and as a whole: every norm, 8-bit tensor and product that a training step and generated tokens consist of against binary64
of what it was given, and their results against the layer in binary64 with the roundings to 8 bits that the calls made."""
import math

import pytest
import torch

import scaled_reference as plain
from paper_1901_03771_amd import lazy as gr
from test_scaled import ROW, check_eight

F64 = torch.float64


def host(a):
    return a.torch().cpu()


class Calls:
    """Stands before the layer's calls, checks each against binary64 of its operands and keeps what it has rounded."""

    def __init__(self, monkeypatch):
        self.rounded, self.products = [], []
        for name in ("quantize", "rms_norm", "rms_norm_grad", "dot_scaled"):
            monkeypatch.setattr(gr, name, getattr(self, "_" + name)(getattr(gr, name)))

    def _keep(self, x, q, s, blocks):
        """x: the values in binary64 that q and s stand for."""
        self.rounded.append(dict(x=x, by=q.double() * plain.spread(s, q.shape) - x, blocks=blocks, used=False))

    def _quantize(self, real):
        def call(x, blocks=False, transposed=False):
            q, s = real(x, blocks=blocks, transposed=transposed)
            v = host(x).double()
            v = v.T.contiguous() if transposed else v
            check_eight(host(q).float(), host(s), v, blocks)
            self._keep(v, host(q), host(s), blocks)
            return q, s
        return call

    def _rms_norm(self, real):
        def call(x, weight, eight=False):
            out, total, s = real(x, weight, eight=eight)
            want, _ = plain.norm(host(x), None, host(weight), 1e-6, 0.0)
            if eight:
                check_eight(host(out).float(), host(s), want, off=ROW + 2.0 ** -22)
                self._keep(want, host(out), host(s), False)
            else:
                assert ((host(out).double() - want).abs() <= (ROW + 2.0 ** -24) * want.abs()).all()
            return out, total, s
        return call

    def _rms_norm_grad(self, real):
        def call(dout, total, weight):
            dx, dw = real(dout, total, weight)
            want, wgain, size, terms = plain.norm_grad(host(dout), host(total), host(weight), None, 1e-6, 0.0)
            assert ((host(dx).double() - want).abs() <= 4 * ROW * size + 2.0 ** -24 * want.abs()).all()
            assert ((host(dw).double() - wgain).abs() <= (ROW + (len(want) + 4) * 2.0 ** -24) * terms).all()
            return dx, dw
        return call

    def _dot_scaled(self, real):
        def call(a, sa, b, sb, dtype):
            out = real(a, sa, b, sb, dtype=dtype)
            assert dtype == gr.GR_F32
            want, size = plain.product(host(a), host(sa), host(b), host(sb))
            # of a block: 127 additions that may cut what they drop; the factors, and the sum of the blocks
            assert ((host(out).double() - want).abs() <= (127 * 2.0 ** -23 + (sa.shape[1] + 4) * 2.0 ** -24) * size).all()
            self.products.append(host(out).double())
            return out
        return call

    def take(self, x, blocks=False):
        """x as the layer's call rounded it: the call whose operand was x, but for float32 errors, added the same to it.  (A rounding of x itself would fall to the other side of a middle
        here and there.)"""
        near = [r for r in self.rounded if r["blocks"] == blocks and r["x"].shape == x.shape and (r["x"] - x).norm() <= 0.01 * x.norm()]
        assert near, "no call has rounded this"
        for r in near:
            r["used"] = True
        return x + near[0]["by"]

    def product(self):
        """x W and its gradients in binary64 with these roundings, each of which counts as the identity in a derivative."""
        calls = self

        class Product(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, w):
                ctx.save_for_backward(x, w)
                return calls.take(x) @ calls.take(w.T.contiguous(), True).T

            @staticmethod
            def backward(ctx, dy):
                x, w = ctx.saved_tensors   # (the layer forms no gradient of its input)
                return calls.take(dy) @ calls.take(w, True).T if ctx.needs_input_grad[0] else None, calls.take(x.T.contiguous()) @ calls.take(dy.T.contiguous()).T
        return Product.apply


def turned(t, first, frequencies):
    a = (first + torch.arange(t.shape[1], dtype=F64))[:, None, None] * torch.tensor(list(frequencies), dtype=F64)
    lo, hi = t[..., :12], t[..., 12:]
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)


def attended(q, k, v, first):
    """Rows first .. of a causal attention with capped scores: q (B, N, 4, 24), k and v (B, M, 2, 24) -> (B N, 96)."""
    k, v = k.repeat_interleave(2, 2), v.repeat_interleave(2, 2)
    s = 8.0 * torch.tanh(torch.einsum("bihd,bjhd->bhij", q, k) * 24 ** -0.5 / 8.0)
    hidden = torch.arange(k.shape[1]) > first + torch.arange(q.shape[1])[:, None]
    p = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
    return torch.einsum("bhij,bjhd->bihd", p, v).reshape(-1, 96)


def normed(h, gain):
    return h if gain is None else h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * gain


# float32 alone is left between the two: sums of up to 140 rows or 144 values in a handful of products one after another, each off by at most (rows + values) 2^-24 of its terms' sizes
# (a product's block by 127 2^-23), which are below 16 times the result's norm here.
BAR = 6 * (140 + 144) * 2.0 ** -24 * 16


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
def test_a_training_step_in_eight_bits(norm, monkeypatch):
    from paper_1901_03771_amd import attention_layer as al
    c = gr.Context()
    layer = al.AttentionLayer(c, width=144, heads=4, shared=2, values=24, cap=8.0, seed=4, norm=norm, eight=True)
    g = torch.Generator().manual_seed(6)
    x, target = torch.randn(2, 70, 144, generator=g), torch.randn(2, 70, 144, generator=g)
    if norm:
        layer.weights["gain"].copy_(1 + 0.2 * torch.randn(144, generator=g))
    before = {n: t.cpu().double() for n, t in layer.weights.items()}
    calls = Calls(monkeypatch)
    got = layer.train_step(x.cuda(), target.cuda(), 0, None, rate=1.0)
    w = {n: t.clone().requires_grad_() for n, t in before.items()}
    times = calls.product()
    h = normed(x.double().view(140, 144), w.get("gain"))
    q, k, v = (times(h, w[n]).view(2, 70, heads, 24) for n, heads in (("q", 4), ("k", 2), ("v", 2)))
    q, k = turned(q, 0, layer.frequencies), turned(k, 0, layer.frequencies)
    y = times(attended(q, k, v, 0), w["o"])
    loss = ((y - target.double().view(140, 144)) ** 2).mean()
    loss.backward()
    assert (calls.products[3] - y).norm() <= BAR * y.norm()                 # (the products of q, k, v, then y)
    assert abs(got - loss.item()) <= BAR * loss.item()
    for n, t in layer.weights.items():
        step = before[n] - t.cpu().double()
        assert (step - w[n].grad).norm() <= BAR * w[n].grad.norm() + 2.0 ** -24 * before[n].norm(), n
    # forward four products; backward one for every weight, that of out, and under a norm those of its result by q, k and v
    assert len(calls.products) == (12 if norm else 9) and all(r["used"] for r in calls.rounded)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
def test_generated_tokens_in_eight_bits(norm, monkeypatch):
    from paper_1901_03771_amd import attention_layer as al
    c = gr.Context()
    layer = al.AttentionLayer(c, width=144, heads=4, shared=2, values=24, cap=8.0, seed=5, norm=norm, eight=True)
    g = torch.Generator().manual_seed(7)
    x = torch.randn(2, 20, 144, generator=g)
    if norm:
        layer.weights["gain"].copy_(1 + 0.2 * torch.randn(144, generator=g))
    w = {n: t.cpu().double() for n, t in layer.weights.items()}
    cache = [torch.full((2, 30, 2, 24), math.nan, device="cuda") for _ in range(2)]
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    ks, vs = [], []
    calls = Calls(monkeypatch)
    times = calls.product()
    for i in range(20):
        calls.rounded.clear()
        calls.products.clear()
        y = layer.step(x[:, i].contiguous().cuda(), *cache, lengths).cpu().double()
        h = normed(x[:, i].double(), w.get("gain"))
        q, k, v = (times(h, w[n]).view(2, 1, heads, 24) for n, heads in (("q", 4), ("k", 2), ("v", 2)))
        ks.append(turned(k, i, layer.frequencies))
        vs.append(v)
        want = times(attended(turned(q, i, layer.frequencies), torch.cat(ks, 1), torch.cat(vs, 1), i), w["o"])
        assert (y - want).norm() <= BAR * want.norm(), i
        assert torch.equal(y, calls.products[3]) and len(calls.products) == 4 and all(r["used"] for r in calls.rounded)
    c.close()
