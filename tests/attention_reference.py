"""Plain attention, its gradient, and rotary positions in binary64, head by head, and how far a kernel's results may be from them."""
import math

import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step of a type, relative to the value


def attention(q, k, v, dout=None, scale=None, cap=0.0, slopes=None, causal=False, position=0, prefix=None, documents=None, lengths=None,
              step=False):
    """q (B, N, H, D), k, v (B, M, HK, D): dict of out, lse and, with dout, dq, dk, dv, all binary64; `*_abs`: the same sums with every term
    made positive, what rounding errors are relative to; `score`: largest sum of |q k| scale plus bias, per batch and head."""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    B, N, H, D = q.shape
    M, HK = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    got = {w: torch.zeros(s, dtype=torch.float64) for w, s in
           (("out", (B, N, H, D)), ("out_abs", (B, N, H, D)), ("lse", (B, H, N)), ("score", (B, H)), ("dq", (B, N, H, D)), ("dq_abs", (B, N, H, D)),
            ("dk", (B, M, HK, D)), ("dk_abs", (B, M, HK, D)), ("dv", (B, M, HK, D)), ("dv_abs", (B, M, HK, D)))}
    qd, kd = (documents if isinstance(documents, tuple) else (documents, documents)) if documents is not None else (None, None)
    j = torch.arange(M)
    for b in range(B):
        n = M if lengths is None else min(max(int(lengths[b]), 0), M)
        place = torch.full((N,), n - 1) if step else torch.arange(N) + position
        see = torch.ones(N, M, dtype=torch.bool)
        if causal:
            see = j[None] <= place[:, None]
            if prefix is not None:
                see = see | (j[None] < int(prefix[b]))
        see = see & (j[None] < n)
        if kd is not None:
            see = see & (qd[b].cpu()[:, None] == kd[b].cpu()[None]) & (kd[b].cpu()[None] >= 0)
        for h in range(H):
            g = h // (H // HK)
            kk, vv = k[b, :, g].clone(), v[b, :, g].clone()
            kk[n:], vv[n:] = 0.0, 0.0
            raw = q[b, :, h] @ kk.T * scale
            s = cap * torch.tanh(raw / cap) if cap else raw
            size = q[b, :, h].abs() @ kk.abs().T * scale
            if slopes is not None:
                bias = float(slopes[h]) * (place[:, None] - j[None]).abs().double()
                s = s - bias
                size = size + bias
            got["score"][b, h] = torch.where(see, size, torch.zeros_like(size)).max() if M and N else 0.0
            s = s.masked_fill(~see, -math.inf)
            lse = torch.logsumexp(s, 1) if M else torch.full((N,), -math.inf)
            p = torch.where(see, torch.exp(s - lse[:, None]), torch.zeros_like(s))
            got["lse"][b, h] = lse
            o = p @ vv
            got["out"][b, :, h], got["out_abs"][b, :, h] = o, p @ vv.abs()
            if dout is None:
                continue
            do = dout[b, :, h].detach().cpu().double()
            dp, delta = do @ vv.T, (do * o).sum(1, keepdim=True)
            bend = 1 - torch.tanh(raw / cap) ** 2 if cap else torch.ones_like(raw)
            ds = p * (dp - delta) * bend * scale
            # what the terms of ds are made of: rounding of dp and delta is relative to their own terms
            ds_abs = p * (do.abs() @ vv.abs().T + (do * o).abs().sum(1, keepdim=True)) * scale
            got["dq"][b, :, h], got["dq_abs"][b, :, h] = ds @ kk, ds_abs @ kk.abs()
            got["dk"][b, :, g] += ds.T @ q[b, :, h]
            got["dk_abs"][b, :, g] += ds_abs.T @ q[b, :, h].abs()
            got["dv"][b, :, g] += p.T @ do
            got["dv_abs"][b, :, g] += p.T @ do.abs()
    return got


def check(got, ref, dtype, D, M, N, group, what, cap=0.0):
    """Every element of `got[w]` against `ref[w]`.

    A score is off by (D + 10) 2^-24 of the sum of its terms' sizes (products exact or rounded once, summed in some order; scaling, cap and
    bias a few roundings more), and by 2^-21 of a cap where bfloat16 takes the short form of tanh: a probability and its normalisation by
    twice that, relatively.  A sum over n terms is off by n 2^-24 of the sum of the terms' sizes.  bfloat16 rounds a probability, or a
    score's gradient, once more (2^-8), the gradient's own sum delta from the rounded output as well, and the result in the end."""
    u, half = 2.0 ** -24, HALF[dtype]
    score = float(ref["score"].max()) if ref["score"].numel() else 0.0
    off = (D + 10) * u * score + (2.0 ** -21 * cap if dtype != torch.float32 else 4 * u * cap)
    extra = half if dtype != torch.float32 else 0.0
    n = {"out": M, "dq": M, "dv": N * group, "dk": N * group}
    for w, x in got.items():
        y = ref[w]
        x = x.detach().cpu().double()
        assert x.shape == y.shape, (what, w, x.shape, y.shape)
        if w == "lse":
            none = y == -math.inf
            assert torch.equal(none, x == -math.inf), f"{what}: lse of rows that see nothing"
            bad = (x - y).abs()[~none] > (off + (M + 16) * u + 4 * u * y.abs())[~none]
            assert not bad.any(), f"{what}: lse off by up to {(x - y).abs()[~none].max():.3g}"
            continue
        rel = 2 * off + (n[w] + 2 * D + 32) * u + extra * (2.0 if w in ("dq", "dk") else 1.0)
        bar = rel * ref[w + "_abs"] + half * y.abs() + 1e-37
        worst = ((x - y).abs() / bar).max() if x.numel() else 0.0
        assert torch.isfinite(x).all(), f"{what}: {w} is not finite"
        assert worst <= 1.0, f"{what}: {w} is {float(worst):.3g} times its bar"
        # and all together: independent roundings add up as their squares do, a rounding being off by half a step / sqrt(3) at most in the mean.
        # Each term of a sum is rounded by itself, so its share is that of its size, not of the sum's
        if x.numel() and y.norm() > 0:
            mean = half * 0.5774 * y.norm() + (extra * 0.5774 * (2.0 if w in ("dq", "dk") else 1.0) + 2 * off + 4 * (n[w] ** 0.5 + D ** 0.5 + 16) * u) * ref[w + "_abs"].norm()
            assert (x - y).norm() <= mean, f"{what}: {w} off by {float((x - y).norm() / y.norm()):.3g} in norm"


def rotary(x, frequencies, positions, interleaved=False, inverse=False, factor=1.0):
    """x (B, N, H, D) turned, in binary64, by rotation matrices written out pair by pair."""
    x = x.detach().cpu().double().numpy()
    y = x.copy()
    half = len(frequencies)
    for i, f in enumerate(frequencies):
        a = np.asarray(positions, dtype=np.float64) * float(f)
        c, s = factor * np.cos(a)[..., None], factor * np.sin(a)[..., None] * (-1.0 if inverse else 1.0)
        l, h = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
        y[..., l], y[..., h] = x[..., l] * c - x[..., h] * s, x[..., h] * c + x[..., l] * s
    return torch.from_numpy(y)
