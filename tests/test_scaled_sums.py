"""What a float32 result of 8-bit tensors promises: the sum of each 128 products is float32 proper, in every form of the product.  The 8-bit matrix cores, which
results in bfloat16 take, drop what lies 13 binary places below the largest of eight neighbouring products: here they would drop bits of every result."""
import pytest
import torch

import scaled_reference as plain
from paper_1901_03771_amd import lazy as gr
from test_scaled import Guarded, strided

F32, E4M3 = torch.float32, torch.float8_e4m3fn

# (m, n, k, values between rows): few rows with whole words and without, with splits and without; tiles of 64 and of 128 rows straight into LDS and through
# registers, with splits and without
FORMS = [(3, 300, 4096, 0), (16, 300, 16384, 0), (9, 100, 129, 0), (32, 300, 4095, 0), (32, 130, 16381, 0), (20, 300, 4088, 0), (4, 300, 2048, 3), (64, 256, 2048, 0), (64, 256, 16384, 0),
         (1000, 2000, 4096, 0), (2000, 3000, 400, 0), (2000, 3000, 1040, 0), (200, 300, 1003, 0), (100, 200, 16381, 0), (512, 1500, 4096, 5), (2000, 3000, 401, 0), (3000, 4000, 261, 0),
         (2000, 3000, 1040, 5)]


def far_apart(seed, m, n, k):
    """Operands of ones, zeros and 2^8, products of ones and of 2^16 side by side: at most 200 of the large ones, one of each eight neighbours in some blocks of 128, so that
    the sizes of all terms are less than 2^24 together, and every sum in float32 is exact in any order."""
    g = torch.Generator().manual_seed(seed)
    sign = lambda *shape: torch.randint(0, 2, shape, generator=g).float() * 2 - 1  # noqa: E731
    a, b = sign(m, k) * (torch.rand(m, k, generator=g) < 0.8), sign(n, k) * (torch.rand(n, k, generator=g) < 0.8)
    eights = torch.randperm((k + 7) // 8, generator=g)[:200] if k < 1600 else (torch.randperm(k // 128, generator=g)[:12, None] * 16 + torch.arange(16)).flatten()
    at = eights * 8 + torch.randint(0, 8, eights.shape, generator=g)
    at = at[at < k]
    a[:, at], b[:, at] = 256 * sign(m, len(at)), 256 * sign(n, len(at))
    assert len(at) * 2 ** 16 + k < 2 ** 24
    return a.to(E4M3), b.to(E4M3)


def dropping(a, b):
    """The sums as the 8-bit matrix cores form them: of eight neighbouring products, what lies below 2^-13 of the largest one's leading place is dropped."""
    m, k = a.shape
    x, y = (torch.nn.functional.pad(t.double(), (0, -k % 8)) for t in (a, b))
    out = torch.zeros(m, b.shape[0], dtype=torch.float64)
    for j in range(0, x.shape[1], 8):
        p = x[:, None, j:j + 8] * y[None, :, j:j + 8]
        step = torch.exp2(torch.floor(torch.log2(p.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -18))) - 13)
        out += (torch.trunc(p / step) * step).sum(-1)
    return out


@pytest.mark.parametrize("m,n,k,pad", FORMS)
def test_the_operands_tell_the_two_kinds_of_sums_apart(m, n, k, pad):
    """On the CPU: sums that drop as the 8-bit matrix cores do are not those of the formula, for nearly all results of a corner of each size."""
    a, b = (t[:16] for t in far_apart(m + n + k, m, n, k))
    exact = a.double() @ b.double().T
    assert (dropping(a, b) != exact).double().mean() > 0.8
    assert torch.equal(exact.float().double(), exact)


@pytest.mark.gpu
@pytest.mark.parametrize("blocks", [True, False], ids=["blocks", "rows"])
@pytest.mark.parametrize("m,n,k,pad", FORMS)
def test_float32_results_are_sums_in_float32(blocks, m, n, k, pad):
    """Bit for bit; the scales are powers of two, of a row or of 128 rows the same throughout, so that a result's terms keep their distances."""
    c = gr.Context()
    a, b = far_apart(m + n + k, m, n, k)
    g = torch.Generator().manual_seed(k)
    high, kb = 128 if blocks else 1, (k + 127) // 128
    sa, sb = (torch.exp2(torch.randint(-3, 4, (rows, 1), generator=g).float()).expand(rows, kb).contiguous() for rows in (m, (n + high - 1) // high))
    want = (a.float() @ b.float().T).double() * plain.spread(sa, (m, 1)) * plain.spread(sb, (n, 1)).T   # (exact in float32, as above)
    out = Guarded((m, n), F32)
    la, lb = (c.array(strided(t, pad) if pad else t.cuda()) for t in (a, b))
    gr.dot_scaled(la, c.array(sa.cuda()), lb, c.array(sb.cuda()), out=c.array(out.t))
    got = out.t.cpu().double()
    assert torch.equal(got, want), int((got != want).sum())
    assert out.untouched()
    c.close()
