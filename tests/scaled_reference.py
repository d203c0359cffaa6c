"""Plain binary64 forms of the norms, the 8-bit tensors and their products (include/grumpy_hip_scaled.h), on the CPU."""
import torch

F64 = torch.float64


def half_step(v):
    """Half the distance between the two e4m3 numbers around |v| <= 448: 3 bits of fraction, exponents from -6 on."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    return torch.exp2(e - 4)


def scales_of(x, blocks=False):
    """max|x| / 448 over 128 neighbours of each row, or over 128 x 128 values."""
    m, k = x.shape
    high = 128 if blocks else 1
    s = torch.empty((m + high - 1) // high, (k + 127) // 128, dtype=F64)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            part = x[i * high:(i + 1) * high, 128 * j:128 * j + 128]
            s[i, j] = part.abs().max() / 448 if torch.isfinite(part).all() else float("nan")
    return s.clamp(min=2.0 ** -126)


def spread(scales, shape):
    """The scale of every value."""
    high = 128 if scales.shape[0] != shape[0] else 1
    return scales.double().repeat_interleave(high, 0)[:shape[0]].repeat_interleave(128, 1)[:, :shape[1]]


def norm(x, residual, weight, eps, offset):
    """(out, total): of rows (R, D); total rounded to the type of x."""
    total = x if residual is None else (x.double() + residual.double()).to(x.dtype)
    t = total.double()
    w = 1.0 if weight is None else weight.double() + offset
    return t / torch.sqrt((t * t).mean(1, keepdim=True) + eps) * w, total


def norm_grad(dout, total, weight, dtotal, eps, offset):
    """(dx, dweight, and the sizes of the sums that each is formed of)."""
    t, y = total.double(), dout.double()
    w = torch.ones(t.shape[1], dtype=F64) if weight is None else weight.double() + offset
    r = 1.0 / torch.sqrt((t * t).mean(1, keepdim=True) + eps)
    g = y * w
    dx = r * g - t * r ** 3 * (g * t).mean(1, keepdim=True)
    size = (r * g).abs() + t.abs() * r ** 3 * (g * t).abs().mean(1, keepdim=True)
    if dtotal is not None:
        dx, size = dx + dtotal.double(), size + dtotal.double().abs()
    terms = y * t * r
    return dx, terms.sum(0), size, terms.abs().sum(0)


def product(a, sa, b, sb):
    """(a b.T, the same of sizes) of the values that 8-bit ones stand for."""
    x, y = a.double() * spread(sa, a.shape), b.double() * spread(sb, b.shape)
    return x @ y.T, x.abs() @ y.abs().T
