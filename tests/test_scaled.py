"""Norms, their gradient, 8-bit tensors with scales and their products (include/grumpy_hip_scaled.h) against plain binary64 forms
(scaled_reference.py), and what the calls refuse."""
import math

import pytest
import torch

import scaled_reference as plain
from paper_1901_03771_amd import lazy as gr
from test_attention import Specs, dry, refused  # noqa: F401

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
NAMES = {F32: "f32", BF16: "bf16"}
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}   # of a rounding to the type, relative
# A row's sum of squares: at most 32 terms a thread one after another, six steps across a wave and 15 across waves, 2^-24 each, which the root halves; then a
# quotient, a root, a reciprocal, offset + weight and two products.
ROW = (0.5 * (32 + 6 + 15) + 6) * 2.0 ** -24


# ---------------------------------------------------------------- without a GPU --
def test_parts_of_packed_rows_are_told_from_overlapping_ones(dry):  # noqa: F811
    s = Specs(dry)
    base, w = s.at, s((200,))
    s.at += 1 << 20
    part = lambda off, rows=6, step=700, cols=200: dry.from_device(base + 4 * off, gr.GR_F32, (rows, cols), (step, 1))  # noqa: E731
    gr.rms_norm(part(0), w, part(200), out=part(400), total=part(200))
    gr.rms_norm(part(0), w, out=part(500))
    for off in (1, 199, 501, 700):                                          # into the columns, around the end of a row, a row further
        refused("GR_ERR_ALIAS", gr.rms_norm, part(0), w, out=part(off))
    refused("GR_ERR_ALIAS", gr.rms_norm, part(0), w, out=part(300, step=800))
    wide = lambda off: dry.from_device(base + 4 * off, gr.GR_F32, (2, 6, 200), (4200, 700, 1))  # noqa: E731
    gr.rms_norm(wide(0), w, out=wide(300))
    refused("GR_ERR_ALIAS", gr.rms_norm, wide(0), w, out=wide(600))
    refused("GR_ERR_ALIAS", gr.rms_norm, wide(0), w, out=wide(4200))


@pytest.mark.parametrize("dtype", [gr.GR_F32, gr.GR_BF16])
def test_calls_run_dry_and_count_their_launches(dry, dtype):  # noqa: F811
    s = Specs(dry)
    n = lambda: dry.stats()["kernel_launches"]  # noqa: E731
    x, res, out, total = (s((2, 40, 260), dtype) for _ in range(4))
    w, q, sc = s((260,)), s((2, 40, 260), gr.GR_E4M3), s((2, 40, 3))
    before = n()
    assert gr.rms_norm(x, w, res, out=out, total=total) == (out, total, None)
    assert gr.rms_norm(x, w, out=q, scales=sc) == (q, x, sc)
    assert n() == before + 2
    dw = s((260,))
    assert gr.rms_norm_grad(out, x, w, dtotal=res, dx=total, dweight=dw) == (total, dw)
    assert n() == before + 4
    y, yq, ys = s((300, 260), dtype), s((300, 260), gr.GR_E4M3), s((300, 3))
    gr.quantize(y, out=yq, scales=ys)
    gr.quantize(y, blocks=True, transposed=True, out=s((260, 300), gr.GR_E4M3), scales=s((3, 3)))
    assert n() == before + 6
    b, rows, blocks = s((70, 260), gr.GR_E4M3), s((70, 3)), s((1, 3))
    gr.dot_scaled(yq, ys, b, rows, out=s((300, 70), dtype))
    gr.dot_scaled(yq, ys, b, blocks, out=s((300, 70), dtype))
    assert n() >= before + 8


def test_norm_refusals(dry):  # noqa: F811
    s = Specs(dry)
    x, res, out, total, w = s((6, 200)), s((6, 200)), s((6, 200)), s((6, 200)), s((200,))
    call = lambda x=x, w=w, res=res, **kw: gr.rms_norm(x, w, res, **{**dict(out=out, total=total), **kw})  # noqa: E731
    call()
    refused("GR_ERR_SHAPE", call, res=s((6, 201)))
    refused("GR_ERR_SHAPE", call, w=s((6,)))
    refused("GR_ERR_SHAPE", call, out=s((6, 100)))
    refused("GR_ERR_SHAPE", call, x=s(()), res=None, out=s(()), total=None)
    refused("GR_ERR_SHAPE", call, x=s((1, 1, 1, 1, 6)))
    refused("GR_ERR_DTYPE", call, x=s((6, 200), gr.GR_I32))
    refused("GR_ERR_DTYPE", call, res=s((6, 200), gr.GR_BF16))
    refused("GR_ERR_DTYPE", call, w=s((200,), gr.GR_BF16))               # a narrower weight than x
    refused("GR_ERR_DTYPE", call, total=s((6, 200), gr.GR_BF16))
    refused("GR_ERR_DTYPE", call, out=s((6, 200), gr.GR_BF16))
    refused("GR_ERR_UNSUPPORTED", call, x=s((6, 200), strides=(400, 2)))
    refused("GR_ERR_UNSUPPORTED", call, out=s((6, 200), strides=(100, 1)))
    refused("GR_ERR_UNSUPPORTED", call, out=s((6, 200), strides=(0, 1)))
    refused("GR_ERR_UNSUPPORTED", call, out=s((6, 200)) + 1.0)
    refused("GR_ERR_UNSUPPORTED", call, x=s((6, 32769)), w=None, res=None, total=None, out=s((6, 32769)))
    refused("GR_ERR_ARG", call, res=None)                                # a total without a residual
    refused("GR_ERR_ARG", call, w=None, offset=1.0)
    for eps in (0.0, -1.0, math.nan, math.inf, 1e-13, 2.0):
        refused("GR_ERR_ARG", call, eps=eps)
    for offset in (math.nan, math.inf, 1e39):
        refused("GR_ERR_ARG", call, offset=offset)
    q, sc = s((6, 200), gr.GR_E4M3), s((6, 2))
    call(out=q, scales=sc)
    refused("GR_ERR_SHAPE", call, out=q, scales=s((6, 1)))
    refused("GR_ERR_DTYPE", call, out=q, scales=s((6, 2), gr.GR_BF16))
    refused("GR_ERR_ARG", call, scales=sc)                               # scales of a result that has none
    # results that overlap operands or each other; the same view may be written over
    call(out=x, total=res)
    call(out=res, total=x)
    refused("GR_ERR_ALIAS", call, out=total)
    base = s.at
    s.at += 1 << 16
    a, b = (dry.from_device(base + off, gr.GR_F32, (6, 200)) for off in (0, 800))
    refused("GR_ERR_ALIAS", call, x=a, out=b)
    refused("GR_ERR_ALIAS", call, out=dry.from_device(w.data_ptr()[0], gr.GR_F32, (6, 200)))
    g = lambda **kw: gr.rms_norm_grad(**{**dict(dout=s((6, 200)), total=x, weight=w, dtotal=res, dx=out, dweight=s((200,))), **kw})  # noqa: E731
    g()
    g(dx=x)
    g(dtotal=None, dweight=False)
    assert g(weight=None, dweight=None) == (out, None)
    refused("GR_ERR_SHAPE", g, dout=s((6, 201)))
    refused("GR_ERR_SHAPE", g, dweight=s((201,)))
    refused("GR_ERR_SHAPE", g, dtotal=s((200,)))
    refused("GR_ERR_DTYPE", g, dweight=s((200,), gr.GR_BF16))
    refused("GR_ERR_DTYPE", g, dx=s((6, 200), gr.GR_BF16))
    refused("GR_ERR_DTYPE", g, dout=s((6, 200), gr.GR_E4M3))
    refused("GR_ERR_ARG", g, eps=0.0)
    refused("GR_ERR_ARG", g, weight=None, offset=1.0)
    refused("GR_ERR_ALIAS", g, dx=a, dweight=dry.from_device(base + 400, gr.GR_F32, (200,)))


def test_quantize_and_product_refusals(dry):  # noqa: F811
    s = Specs(dry)
    x, q, sc = s((300, 200)), s((300, 200), gr.GR_E4M3), s((300, 2))
    call = lambda x=x, **kw: gr.quantize(x, **{**dict(out=q, scales=sc), **kw})  # noqa: E731
    call()
    refused("GR_ERR_SHAPE", call, x=s((3, 100, 200)))
    refused("GR_ERR_SHAPE", call, out=s((200, 300), gr.GR_E4M3))
    refused("GR_ERR_SHAPE", call, blocks=True)
    refused("GR_ERR_SHAPE", call, transposed=True)
    refused("GR_ERR_DTYPE", call, x=s((300, 200), gr.GR_I32))
    refused("GR_ERR_DTYPE", call, x=q)
    refused("GR_ERR_DTYPE", call, out=s((300, 200)))
    refused("GR_ERR_DTYPE", call, scales=s((300, 2), gr.GR_I32))
    refused("GR_ERR_UNSUPPORTED", call, x=s((300, 200), strides=(1, 300)))
    refused("GR_ERR_UNSUPPORTED", call, out=s((300, 200), gr.GR_E4M3, strides=(1, 300)))
    refused("GR_ERR_UNSUPPORTED", call, scales=s((300, 2), strides=(0, 1)))
    refused("GR_ERR_ALIAS", call, scales=dry.from_device(x.data_ptr()[0], gr.GR_F32, (300, 2)))
    refused("GR_ERR_ALIAS", call, out=dry.from_device(x.data_ptr()[0], gr.GR_E4M3, (300, 200)))
    L = gr.lib()
    assert L.gr_quantize(dry._p, x.h, 2, 0, q.h, sc.h) == 6 and L.gr_quantize(dry._p, x.h, 0, -1, q.h, sc.h) == 6
    assert L.gr_quantize(dry._p, 1 << 40, 0, 0, q.h, sc.h) == 1 and L.gr_quantize(None, x.h, 0, 0, q.h, sc.h) == 6
    b, sb, out = s((70, 200), gr.GR_E4M3), s((70, 2)), s((300, 70))
    dot = lambda a=q, sa=sc, b=b, sb=sb, out=out: gr.dot_scaled(a, sa, b, sb, out=out)  # noqa: E731
    dot()
    dot(sb=s((1, 2)))
    refused("GR_ERR_SHAPE", dot, b=s((70, 201), gr.GR_E4M3))
    refused("GR_ERR_SHAPE", dot, sb=s((2, 2)))
    refused("GR_ERR_SHAPE", dot, sb=s((70,)))
    refused("GR_ERR_SHAPE", dot, sa=s((3, 2)))                            # a has scales of rows
    refused("GR_ERR_SHAPE", dot, sa=s((300, 1)))
    refused("GR_ERR_SHAPE", dot, out=s((70, 300)))
    refused("GR_ERR_DTYPE", dot, a=x)
    refused("GR_ERR_DTYPE", dot, b=s((70, 200), gr.GR_BF16))
    refused("GR_ERR_DTYPE", dot, out=s((300, 70), gr.GR_I32))
    refused("GR_ERR_DTYPE", dot, sb=s((70, 2), gr.GR_I32))
    refused("GR_ERR_UNSUPPORTED", dot, a=s((300, 200), gr.GR_E4M3, strides=(1, 300)))
    refused("GR_ERR_UNSUPPORTED", dot, out=s((300, 70), strides=(1, 300)))
    refused("GR_ERR_UNSUPPORTED", dot, out=s((300, 70), strides=(60, 1)))
    refused("GR_ERR_ALIAS", dot, out=dry.from_device(sc.data_ptr()[0], gr.GR_F32, (300, 70)))
    assert L.gr_dot_scaled(dry._p, q.h, sc.h, b.h, sb.h, 1 << 40) == 1 and L.gr_dot_scaled(dry._p, q.h, sc.h, b.h, 0, out.h) == 1
    assert L.gr_rms_norm(dry._p, 0, 0, 0, 1e-6, 0.0, 0, 0, 0) == 1 and L.gr_rms_norm_grad(None, 0, 0, 0, 0, 1e-6, 0.0, 0, 0) == 6


def test_calls_beyond_a_launch_are_refused(dry):  # noqa: F811
    """Nothing is launched where a launch does not hold the call."""
    big = lambda shape, t=gr.GR_E4M3, strides=None, at=[1 << 41]: (at.__setitem__(0, at[0] + (1 << 43)), dry.from_device(at[0], t, shape, strides))[1]  # noqa: E731,B006
    n = dry.stats()["kernel_launches"]
    m = 1 << 20
    refused("GR_ERR_UNSUPPORTED", gr.dot_scaled, big((m, 1)), big((m, 1), gr.GR_F32), big((m, 1)), big((m, 1), gr.GR_F32), out=big((m, m), gr.GR_F32))
    refused("GR_ERR_UNSUPPORTED", gr.dot_scaled, big((m << 11, 1)), big((m << 11, 1), gr.GR_F32), big((1, 1)), big((1, 1), gr.GR_F32), out=big((m << 11, 1), gr.GR_F32))
    refused("GR_ERR_UNSUPPORTED", gr.dot_scaled, big((1, 1)), big((1, 1), gr.GR_F32), big((1 << 28, 1)), big((1 << 28, 1), gr.GR_F32), out=big((1, 1 << 28), gr.GR_F32))
    refused("GR_ERR_UNSUPPORTED", gr.quantize, big((1 << 30, 1), gr.GR_F32), out=big((1 << 30, 1)), scales=big((1 << 30, 1), gr.GR_F32))
    refused("GR_ERR_UNSUPPORTED", gr.rms_norm, big((1 << 31, 1), gr.GR_F32), out=big((1 << 31, 1), gr.GR_F32))
    assert dry.stats()["kernel_launches"] == n


def test_empty_tensors(dry):  # noqa: F811
    s = Specs(dry)
    n = lambda: dry.stats()["kernel_launches"]  # noqa: E731
    before = n()
    gr.rms_norm(s((0, 64)), s((64,)), out=s((0, 64)))
    gr.rms_norm(s((3, 0)), out=s((3, 0)))
    gr.quantize(s((0, 64)), out=s((0, 64), gr.GR_E4M3), scales=s((0, 1)))
    gr.quantize(s((5, 0)), out=s((5, 0), gr.GR_E4M3), scales=s((5, 0)))
    gr.dot_scaled(s((0, 64), gr.GR_E4M3), s((0, 1)), s((9, 64), gr.GR_E4M3), s((1, 1)), out=s((0, 9)))
    assert n() == before
    gr.rms_norm_grad(s((0, 64)), s((0, 64)), s((64,)), dx=s((0, 64)), dweight=s((64,)))              # dweight is zero, and written
    gr.dot_scaled(s((4, 0), gr.GR_E4M3), s((4, 0)), s((9, 0), gr.GR_E4M3), s((1, 0)), out=s((4, 9)))   # so is a product over nothing
    assert n() == before + 2


def test_e4m3_arrays_go_nowhere_else(dry):  # noqa: F811
    s = Specs(dry)
    a, b = s((4, 8), gr.GR_E4M3), s((4, 8))
    for f in (lambda: a + 1.0, lambda: a + a, lambda: a + b, lambda: -a, lambda: gr.exp(a), lambda: a.sum(), lambda: a.cumsum(0), lambda: a.reshape(32),
              lambda: gr.dot(a, a), lambda: a[1:] * 2.0, lambda: a[1:].plan(), lambda: gr.rotary(a, [1.0])):
        refused("GR_ERR_DTYPE", f)

    def assign():
        a[1:] = s((3, 8), gr.GR_E4M3)
    refused("GR_ERR_DTYPE", assign)
    assert a[1:, 2:].shape == (3, 6) and a.T.shape == (8, 4) and a[1:].dtype_code == gr.GR_E4M3
    assert a[1:, 2:].data_ptr()[0] == a.data_ptr()[0] + 8 + 2


def test_what_python_is_given_wrong_is_said_so(dry):  # noqa: F811
    s = Specs(dry)
    x, w, q, sc = s((6, 200)), s((200,)), s((6, 200), gr.GR_E4M3), s((6, 2))
    for bad in (1.0, None, torch.ones(6, 200)):
        for call in (lambda: gr.rms_norm(bad), lambda: gr.rms_norm_grad(bad, x), lambda: gr.rms_norm_grad(x, bad), lambda: gr.quantize(bad),
                     lambda: gr.dot_scaled(bad, sc, q, sc), lambda: gr.dot_scaled(q, sc, q, bad)):
            with pytest.raises(TypeError):
                call()
    with pytest.raises(TypeError):
        gr.rms_norm(x, 1.0)
    other = gr.Context(device=-1)
    with pytest.raises(ValueError):
        gr.rms_norm(x, Specs(other)((200,)), out=s((6, 200)))
    with pytest.raises(ValueError):
        gr.dot_scaled(q, sc, q, Specs(other)((6, 2)), out=s((6, 6)))
    other.close()
    i = s((6, 200), gr.GR_I32)
    for call in (lambda: gr.rms_norm(i), lambda: gr.rms_norm_grad(i, i), lambda: gr.dot_scaled(q, sc, q, sc, dtype=gr.GR_I32)):
        refused("GR_ERR_DTYPE", call)
    for call in (lambda: gr.rms_norm(s(())), lambda: gr.quantize(w), lambda: gr.dot_scaled(q, sc, s((200,), gr.GR_E4M3), sc)):
        refused("GR_ERR_SHAPE", call)
    for call in (lambda: gr.rms_norm(x, w), lambda: gr.rms_norm(x, w, eight=True), lambda: gr.rms_norm_grad(x, x, w), lambda: gr.quantize(x), lambda: gr.dot_scaled(q, sc, q, sc)):
        refused("GR_ERR_NODEVICE", call)                                  # no memory for new results


def test_both_routes_of_the_binding(dry, monkeypatch):  # noqa: F811
    """The C type's route and the longer one make the same launches and refuse the same calls."""
    s = Specs(dry)
    x, res, out, total, w = (s((6, 200)) for _ in range(5))
    w, q, sc, dw = s((200,)), s((6, 200), gr.GR_E4M3), s((6, 2)), s((200,))
    b, sb, y = s((70, 200), gr.GR_E4M3), s((70, 2)), s((6, 70))
    calls = [(lambda: gr.rms_norm(x, w, res, out=out, total=total), None), (lambda: gr.rms_norm(x, w, res, out=out, total=False), None), (lambda: gr.rms_norm(x, out=q, scales=sc), None),
             (lambda: gr.rms_norm(x, w, out=out, eps=1), None), (lambda: gr.rms_norm(x, w, out=out, eps=0.0), "GR_ERR_ARG"), (lambda: gr.rms_norm(x, w, out=q), "GR_ERR_NODEVICE"),
             (lambda: gr.rms_norm(x, w, res, out=out), "GR_ERR_NODEVICE"), (lambda: gr.rms_norm_grad(x, res, w, dx=out, dweight=dw), None),
             (lambda: gr.rms_norm_grad(x, res, w, dx=out, dweight=False), None), (lambda: gr.rms_norm_grad(x, res, w, dx=out, dweight=sc), "GR_ERR_SHAPE"),
             (lambda: gr.quantize(x, out=q, scales=sc), None), (lambda: gr.quantize(x, blocks=1, out=q, scales=s((1, 2))), None), (lambda: gr.quantize(x, blocks=True, out=q, scales=sc), "GR_ERR_SHAPE"),
             (lambda: gr.dot_scaled(q, sc, b, sb, out=y), None), (lambda: gr.dot_scaled(q, sc, b, sc, out=y), "GR_ERR_SHAPE")]
    seen = []
    for fast in (gr._fastbind, None):
        monkeypatch.setattr(gr, "_fastbind", fast)
        got = []
        for call, code in calls:
            n = dry.stats()["kernel_launches"]
            if code:
                refused(code, call)
            else:
                call()
            got.append(dry.stats()["kernel_launches"] - n)
        seen.append(got)
    assert seen[0] == seen[1] and all((n > 0) == (code is None) for n, (_, code) in zip(seen[0], calls))
    monkeypatch.undo()
    other = gr.Context(device=-1)
    o = Specs(other)((6, 200))
    with pytest.raises(ValueError):
        gr.rms_norm(x, out=o)
    other.close()
    with pytest.raises((RuntimeError, gr.GrError)):
        gr.rms_norm(o, out=o)                                             # a context that is closed


def test_reference_gradient_against_differences():
    g = torch.Generator().manual_seed(5)
    x, dout, dtotal = (torch.randn(4, 7, generator=g, dtype=torch.float64) for _ in range(3))
    w = torch.randn(7, generator=g, dtype=torch.float64)
    f = lambda x, w: float((plain.norm(x, None, w, 1e-3, 1.0)[0] * dout).sum() + (x * dtotal).sum())  # noqa: E731
    dx, dw = plain.norm_grad(dout, x, w, dtotal, 1e-3, 1.0)[:2]
    for at in [(0, 0), (1, 6), (3, 3)]:
        e = torch.zeros_like(x)
        e[at] = 1e-6
        assert abs((f(x + e, w) - f(x - e, w)) / 2e-6 - dx[at]) < 1e-8
    for at in range(7):
        e = torch.zeros_like(w)
        e[at] = 1e-6
        assert abs((f(x, w + e) - f(x, w - e)) / 2e-6 - dw[at]) < 1e-8


# ------------------------------------------------------------------- on the GPU --
@pytest.fixture(scope="module")
def ctx():
    c = gr.Context()
    yield c
    c.close()


def normal(seed, *shape, dtype=F32, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * by).to(dtype)


class Guarded:
    """A result within a larger buffer, whose other bytes have to stay as they are.  pad: values between rows; off: before the first."""

    def __init__(self, shape, dtype, pad=3, off=5):
        size = torch.tensor([], dtype=dtype).element_size()
        n = max(1, math.prod(shape[:-1]))
        step = shape[-1] + pad
        self.bytes = torch.full(((off + n * step + 64) * size,), 0x5a, dtype=torch.uint8, device="cuda")
        self.flat = self.bytes.view(dtype)
        strides = [1]
        for i in range(len(shape) - 1, 0, -1):
            strides.insert(0, step if i == len(shape) - 1 else strides[0] * shape[i])
        self.t = torch.as_strided(self.flat, shape, strides, off)
        self.inside = torch.zeros(self.flat.numel(), dtype=torch.bool, device="cuda")
        torch.as_strided(self.inside, shape, strides, off).fill_(True)

    def untouched(self):
        size = self.bytes.numel() // self.flat.numel()
        return bool((self.bytes.view(-1, size)[~self.inside] == 0x5a).all())


def strided(t, pad):
    """The same values with `pad` more between rows and one in front, on the GPU."""
    big = torch.full((*t.shape[:-1], t.shape[-1] + pad), 3.0).to(t.dtype)
    flat = torch.cat([torch.full((1,), 3.0).to(t.dtype), big.flatten()]).cuda()
    view = flat[1:].view(big.shape)[..., :t.shape[-1]]
    view.copy_(t.cuda())
    return view


def check_eight(q, scales, exact, blocks=False, off=2.0 ** -22):
    """q in e4m3 over f32 scales against values in binary64, all (M, K) on the CPU: scales right to `off` more than a rounding, values to half a step and `off`."""
    want = plain.scales_of(exact, blocks)
    bad = (scales.double() - want).abs() > want * (2.0 ** -24 + off)
    assert not bad.any(), (int(bad.sum()), scales[bad][:4], want[bad][:4])
    v = exact / plain.spread(scales, exact.shape)
    room = plain.half_step(v.clamp(-448, 448)) + off * v.abs() + (v.abs() - 448).clamp(min=0)
    far = (q.double() - v).abs() > room
    assert not far.any(), (int(far.sum()), q[far][:4], v[far][:4])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("blocks,transposed", [(False, False), (True, False), (False, True), (True, True)], ids=["rows", "blocks", "columns", "blocks_transposed"])
@pytest.mark.parametrize("m,k,pad", [(1, 1, 0), (1, 128, 0), (128, 1, 2), (128, 128, 0), (3, 129, 1), (129, 127, 0), (257, 300, 4), (130, 1031, 5), (64, 4096, 8), (640, 256, 0)])
def test_quantize(ctx, dtype, blocks, transposed, m, k, pad):
    x = normal(m + k, m, k, dtype=dtype) * torch.exp(normal(k, m, 1)).to(dtype)
    x[m // 2, k // 2] = 0.0
    rows, cols = (k, m) if transposed else (m, k)
    out = Guarded((rows, cols), E4M3, pad=pad)
    sc = Guarded(((rows + 127) // 128 if blocks else rows, (cols + 127) // 128), F32, pad=1)
    gr.quantize(ctx.array(strided(x, pad) if pad else x.cuda()), blocks=blocks, transposed=transposed, out=ctx.array(out.t), scales=ctx.array(sc.t))
    exact = (x.T if transposed else x).double()
    check_eight(out.t.float().cpu(), sc.t.cpu(), exact, blocks)
    # the scale is the quotient of f32, and to the last place
    top = plain.scales_of(exact, blocks) * 448
    assert torch.equal(sc.t.cpu(), torch.clamp(top.float() / 448.0, min=2.0 ** -126))
    assert out.untouched() and sc.untouched()
    q, s = gr.quantize(ctx.array(x.cuda()), blocks=blocks, transposed=transposed)      # new results
    assert torch.equal(q.torch().float(), out.t.float()) and torch.equal(s.torch(), sc.t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("blocks,transposed", [(False, False), (True, False), (False, True), (True, True)], ids=["rows", "blocks", "columns", "blocks_transposed"])
def test_quantize_of_extreme_values(ctx, dtype, blocks, transposed):
    """Zeros, numbers below the least scale, the largest floats, infinities and NaN: what is not a number stays in its block."""
    x = normal(9, 700, 256, dtype=dtype)
    most = torch.finfo(dtype).max
    x[0:128, :128] = 0.0
    x[128:256, :128] = 1e-39
    x[256:384, :128] *= 1e38
    x[256, 3], x[300, 100], x[301, 101] = most, -most, most / 3
    x[384, 5] = math.inf
    x[520, 7] = math.nan
    x[641, 9] = -math.inf
    q, s = gr.quantize(ctx.array(x.cuda()), blocks=blocks, transposed=transposed)
    q, s = q.torch().float().cpu(), s.torch().cpu()
    exact = (x.T if transposed else x).double()
    want = plain.scales_of(exact, blocks)
    assert torch.equal(want.isnan(), s.isnan())
    each = plain.spread(s, exact.shape)
    assert torch.equal(q.isnan(), each.isnan())
    fine = ~each.isnan()
    v = exact[fine] / each[fine]
    assert ((q[fine] - v).abs() <= plain.half_step(v.clamp(-448, 448)) + 2.0 ** -22 * v.abs() + (v.abs() - 448).clamp(min=0)).all()
    assert ((s - want).abs() <= want * 2.0 ** -23)[~want.isnan()].all() and float(s[~s.isnan()].min()) == 2.0 ** -126


@pytest.mark.gpu
def test_quantize_rounds_ties_to_even_and_keeps_small_numbers(ctx):
    """All numbers of the type and all middles between them, under a scale of one."""
    codes = torch.arange(127, dtype=torch.uint8).view(E4M3).double()          # 0 .. 448
    mid = (codes[1:] + codes[:-1]) / 2
    even = torch.where(torch.arange(126) % 2 == 0, codes[:-1], codes[1:])     # a code is even where its last bit is
    for v, want in ((codes, codes), (mid, even)):
        row = torch.zeros(2, 128)
        row[0, :len(v)], row[1, :len(v)] = v.float(), -v.float()
        row[:, 127] = 448.0
        q, s = gr.quantize(ctx.array(row.cuda()))
        assert bool((s.torch() == 1.0).all())
        got = q.torch().double().cpu()[:, :len(v)]
        assert torch.equal(got[0], want) and torch.equal(got[1], -want)


NORMS = [(1, 1), (1, 64), (5, 80), (3, 127), (7, 128), (2, 129), (9, 256), (33, 300), (4, 513), (3, 1031), (5, 2048), (2, 2052), (3, 4096), (2, 5003), (2, 8192), (2, 8200), (2, 16384),
         (2, 16390), (1, 32768), (700, 96), (2500, 64), (2100, 520)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("eight", [False, True], ids=["same", "eight"])
@pytest.mark.parametrize("rows,D", NORMS)
def test_norm(ctx, dtype, eight, rows, D):
    n = rows + D
    x, res = normal(n, rows, D, dtype=dtype), normal(n + 1, rows, D, dtype=dtype, by=3.0)
    w = normal(n + 2, D, by=0.3)
    for residual, weight, offset in ((None, w, 1.0), (res, w.to(dtype), 0.0), (res, None, 0.0)):
        y, total = plain.norm(x, residual, weight, 1e-5, offset)
        out, sums = Guarded((rows, D), E4M3 if eight else dtype), Guarded((rows, D), dtype, pad=0, off=0)
        sc = Guarded((rows, (D + 127) // 128), F32)
        got = gr.rms_norm(ctx.array(x.cuda()), None if weight is None else ctx.array(weight.cuda()), None if residual is None else ctx.array(strided(residual, 7)), eps=1e-5,
                          offset=offset, out=ctx.array(out.t), total=None if residual is None else ctx.array(sums.t), scales=ctx.array(sc.t) if eight else None)
        if residual is not None:
            assert torch.equal(sums.t.cpu(), total) and sums.untouched()
        else:
            assert got[1].data_ptr()[0] != sums.t.data_ptr()
        if eight:
            check_eight(out.t.float().cpu(), sc.t.cpu(), y, off=ROW + 2.0 ** -22)
            assert sc.untouched()
        else:
            far = (out.t.cpu().double() - y).abs() > (ROW + HALF[dtype]) * y.abs()
            assert not far.any(), (int(far.sum()), float(((out.t.cpu().double() - y).abs() / y.abs()).max()))
        assert out.untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("rows,D", NORMS)
def test_norm_gradient(ctx, dtype, rows, D):
    n = rows * 7 + D
    total, dout, more = (normal(n + i, rows, D, dtype=dtype) for i in range(3))
    w = normal(n + 3, D, by=0.3)
    for dtotal, weight, offset in ((None, w, 1.0), (more, w.to(dtype), 0.0), (more, None, 0.0)):
        dx, dw, size, terms = plain.norm_grad(dout, total, weight, dtotal, 1e-5, offset)
        to, dweight = Guarded((rows, D), dtype), Guarded((D,), F32)
        gr.rms_norm_grad(ctx.array(strided(dout, 3)), ctx.array(total.cuda()), None if weight is None else ctx.array(weight.cuda()), None if dtotal is None else ctx.array(dtotal.cuda()),
                         eps=1e-5, offset=offset, dx=ctx.array(to.t), dweight=ctx.array(dweight.t))
        # dx: both sums as long as a norm's, three factors of r; the rounding of the result
        far = (to.t.cpu().double() - dx).abs() > 4 * ROW * size + HALF[dtype] * dx.abs()
        assert not far.any(), int(far.sum())
        # dweight: a row's r, two products, and a sum of the rows in any order
        far = (dweight.t.cpu().double() - dw).abs() > (ROW + (rows + 4) * 2.0 ** -24) * terms
        assert not far.any(), int(far.sum())
        assert to.untouched() and dweight.untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_norm_of_views_and_in_place(ctx, dtype):
    """Heads within packed rows, axes in another order, rows walked backwards; results over operands."""
    packed = normal(1, 6, 5, 12, 80, dtype=dtype).cuda()
    w = normal(2, 80).cuda()
    for view in (packed[:, :, 3:7], packed.permute(1, 0, 2, 3), packed.permute(2, 1, 0, 3)[::1, 1:4], packed[:, 2], packed[3, 2]):
        flat = view.reshape(-1, 80).cpu()
        y, _ = plain.norm(flat, None, w.cpu(), 1e-6, 0.0)
        out = torch.zeros_like(view.contiguous())
        gr.rms_norm(ctx.array(view), ctx.array(w), out=ctx.array(out))
        assert ((out.reshape(-1, 80).cpu().double() - y).abs() <= (ROW + HALF[dtype]) * y.abs()).all()
        q, x, s = gr.rms_norm(ctx.array(view), ctx.array(w), eight=True)
        assert q.shape == tuple(view.shape) and s.shape == tuple(view.shape[:-1]) + (1,)
        check_eight(q.torch().float().reshape(-1, 80).cpu(), s.torch().reshape(-1, 1).cpu(), y, off=ROW + 2.0 ** -22)
        dx, dw, size, terms = plain.norm_grad(flat, flat, w.cpu(), None, 1e-6, 0.0)
        gx, gw = gr.rms_norm_grad(ctx.array(view), ctx.array(view), ctx.array(w))
        assert ((gx.torch().reshape(-1, 80).cpu().double() - dx).abs() <= 4 * ROW * size + HALF[dtype] * dx.abs()).all()
        assert ((gw.torch().cpu().double() - dw).abs() <= (ROW + (len(flat) + 4) * 2.0 ** -24) * terms).all()
    x, res = packed[0].contiguous(), packed[1].contiguous()
    want, total = plain.norm(x.reshape(-1, 80).cpu(), res.reshape(-1, 80).cpu(), w.cpu(), 1e-6, 0.0)
    ax, ar = ctx.array(x), ctx.array(res)
    gr.rms_norm(ax, ctx.array(w), ar, out=ax, total=ar)
    assert torch.equal(res.reshape(-1, 80).cpu(), total)
    assert ((x.reshape(-1, 80).cpu().double() - want).abs() <= (ROW + HALF[dtype]) * want.abs()).all()
    d = packed[2].contiguous()
    dx, _, size, _ = plain.norm_grad(d.reshape(-1, 80).cpu(), total, w.cpu(), total, 1e-6, 0.0)
    ad = ctx.array(d)
    gr.rms_norm_grad(ad, ar, ctx.array(w), dtotal=ar, dx=ad)
    assert ((d.reshape(-1, 80).cpu().double() - dx).abs() <= 4 * ROW * size + HALF[dtype] * dx.abs()).all()
    back = packed.flip(0).contiguous()   # rows walked backwards
    lazy = ctx.from_device(back[-1].data_ptr(), gr.GR_F32 if dtype == F32 else gr.GR_BF16, back.shape, (-back.stride(0), *back.stride()[1:]), back)
    y, _ = plain.norm(packed.reshape(-1, 80).cpu(), None, w.cpu(), 1e-6, 0.0)
    got = gr.rms_norm(lazy, ctx.array(w))[0].torch()
    assert ((got.reshape(-1, 80).cpu().double() - y).abs() <= (ROW + HALF[dtype]) * y.abs()).all()


@pytest.mark.gpu
def test_norm_of_rows_that_are_no_numbers(ctx):
    """NaN and infinities stay in their rows; a row of zeros gives zeros."""
    x = normal(3, 40, 300, dtype=BF16)
    x[3, 7], x[11, 299], x[20] = math.nan, math.inf, 0.0
    w = torch.ones(300)
    out, _, _ = gr.rms_norm(ctx.array(x.cuda()), ctx.array(w.cuda()))
    q, _, s = gr.rms_norm(ctx.array(x.cuda()), ctx.array(w.cuda()), eight=True)
    dx, _ = gr.rms_norm_grad(ctx.array(torch.ones_like(x).cuda()), ctx.array(x.cuda()), ctx.array(w.cuda()))
    out, q, s, dx = (t.torch().float().cpu() for t in (out, q, s, dx))
    good = torch.tensor([i not in (3, 11) for i in range(40)])
    assert out[3].isnan().all() and s[3].isnan().all() and q[3].isnan().all() and dx[3].isnan().all()
    assert out[11, 299].isnan() and bool((out[11, :299] == 0).all())                     # 1 / inf of what is finite
    assert s[11, 2].isnan() and bool((q[11, :256] == 0).all()) and q[11, 256:].isnan().all()
    assert bool(out[good].isfinite().all() and s[good].isfinite().all() and dx[good].isfinite().all())
    assert bool((out[20] == 0).all() and (q[20] == 0).all() and (s[20] == 2.0 ** -126).all())


def whole(seed, rows, k, high):
    """Small whole numbers in e4m3 and scales that are powers of two, so that every sum is exact."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(-2, 3, (rows, k), generator=g).float()
    s = torch.exp2(torch.randint(-2, 2, ((rows + high - 1) // high, (k + 127) // 128), generator=g).float())
    return q.to(E4M3), s


PRODUCTS = [(1, 1, 1), (1, 128, 128), (1, 300, 1000), (2, 64, 4096), (3, 129, 257), (16, 256, 512), (17, 130, 640), (33, 513, 300), (64, 1024, 1024), (65, 200, 2048), (100, 100, 100),
            (128, 128, 128), (129, 127, 384), (192, 384, 5120), (255, 257, 1003), (300, 1100, 260), (513, 300, 144), (1000, 777, 400), (256, 2048, 256), (1, 1, 8192), (4, 16, 16384),
            (3, 40, 40000), (32, 33, 12288), (40, 64, 40000)]


@pytest.mark.gpu
@pytest.mark.parametrize("out", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("blocks", [True, False], ids=["blocks", "rows"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product_of_whole_numbers(ctx, out, blocks, m, n, k):
    """Every product and sum is exact: results are equal to the last bit, wherever the places, tiles and splits are.  Sums stay below 4 x 4 x 40000, in sixteenths below 2^24."""
    a, sa = whole(m + k, m, k, 1)
    b, sb = whole(n + k, n, k, 128 if blocks else 1)
    want = plain.product(a, sa, b, sb)[0].to(out)
    to = Guarded((m, n), out)
    gr.dot_scaled(*(ctx.array(t.cuda()) for t in (a, sa, b, sb)), out=ctx.array(to.t))
    assert torch.equal(to.t.cpu(), want), int((to.t.cpu() != want).sum())
    assert to.untouched()
    # rows at any address, scales side by side
    to2 = Guarded((m, n), out, pad=0, off=0)
    gr.dot_scaled(ctx.array(strided(a, 5)), ctx.array(sa.cuda().T.contiguous().T), ctx.array(strided(b, 11)), ctx.array(sb.cuda().T.contiguous().T), out=ctx.array(to2.t))
    assert torch.equal(to2.t.cpu(), want) and to2.untouched()
    # rows of whole vectors within wider ones
    wide = [torch.zeros(t.shape[0], (t.shape[1] + 31) // 16 * 16, dtype=torch.uint8, device="cuda").fill_(0x7f).view(E4M3) for t in (a, b)]
    for w, t in zip(wide, (a, b)):
        w[:, :k] = t.cuda()
    got = gr.dot_scaled(ctx.array(wide[0][:, :k]), ctx.array(sa.cuda()), ctx.array(wide[1][:, :k]), ctx.array(sb.cuda()), dtype=gr.GR_F32 if out == F32 else gr.GR_BF16)
    assert torch.equal(got.torch().cpu(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("out", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("blocks", [True, False], ids=["blocks", "rows"])
@pytest.mark.parametrize("k", [1, 7, 15, 16, 17, 128, 130, 144, 256, 257, 272, 383, 384, 400, 511, 512, 640, 701, 784, 896, 1168])
def test_product_of_few_blocks(ctx, out, blocks, k):
    """Tiles that are sent for ahead of their use, where there are fewer blocks than are under way, as many, and some more; NaN behind rows and operands."""
    m, n = 70, 133
    a, sa = whole(k, m, k, 1)
    b, sb = whole(k + 1, n, k, 128 if blocks else 1)
    want = plain.product(a, sa, b, sb)[0].to(out)
    wide = [torch.full((t.shape[0] + 64, k + 48), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for t in (a, b)]
    scales = [torch.full((t.shape[0] + 64, t.shape[1] + 4), float("nan"), device="cuda") for t in (sa, sb)]
    for w, t in zip(wide + scales, (a, b, sa, sb)):
        w[:t.shape[0], :t.shape[1]] = t.cuda()
    to = Guarded((m, n), out)
    gr.dot_scaled(*(ctx.array(w[:t.shape[0], :t.shape[1]]) for w, t in zip((wide[0], scales[0], wide[1], scales[1]), (a, sa, b, sb))), out=ctx.array(to.t))
    assert torch.equal(to.t.cpu(), want) and to.untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("blocks", [True, False], ids=["blocks", "rows"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(ctx, blocks, m, n, k):
    a, b = normal(m, m, k) * torch.exp(normal(m + 1, m, 1)), normal(n, n, k)
    qa, sa = gr.quantize(ctx.array(a.cuda()))
    qb, sb = gr.quantize(ctx.array(b.cuda()), blocks=blocks)
    want, size = plain.product(*(t.torch().cpu() for t in (qa, sa, qb, sb)))
    # of a block: 127 additions in float32, which may cut what they drop (2^-23); the scales' product, its product with the sum (twice where rows have scales of
    # their own), and the sum of the blocks, over splits too.  The 8-bit cores of a bf16 result drop less than 2^-13 of the largest of eight products from each of the other seven.
    room = 127 * 2.0 ** -23 + ((k + 127) // 128 + 4) * 2.0 ** -24
    for dtype, more in ((F32, 0.0), (BF16, 7 * 2.0 ** -13)):
        got = gr.dot_scaled(qa, sa, qb, sb, dtype=gr.GR_F32 if dtype == F32 else gr.GR_BF16).torch().cpu().double()
        far = (got - want).abs() > (room + more) * size + HALF[dtype] * want.abs()
        assert not far.any(), int(far.sum())


@pytest.mark.gpu
def test_product_with_what_is_no_number(ctx):
    """A block of a row that is NaN makes its row of the result NaN, and no other; what lies behind the ends of rows has no say."""
    m, n, k = 40, 50, 300
    a, sa = whole(1, m, k, 1)
    b, sb = whole(2, n, k, 1)
    want = plain.product(a, sa, b, sb)[0]
    sa[7, 1], sb[9, 2] = math.nan, math.nan
    a[7, 128:256] = math.nan
    b[9, 256:] = math.nan
    got = gr.dot_scaled(*(ctx.array(t.cuda()) for t in (a, sa, b, sb)), dtype=gr.GR_F32).torch().cpu().double()
    bad = torch.zeros(m, n, dtype=torch.bool)
    bad[7], bad[:, 9] = True, True
    assert got[bad].isnan().all() and torch.equal(got[~bad], want[~bad])
    zero = gr.dot_scaled(*(ctx.array(t.cuda()) for t in (a[:, :0], sa[:, :0], b[:, :0], sb[:, :0])), dtype=gr.GR_F32).torch()
    assert bool((zero == 0).all()) and zero.shape == (m, n)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(4100, 3100, 272), (8200, 1700, 144), (2050, 6200, 640), (3001, 4500, 261), (12289, 1300, 128), (4090, 4070, 1040), (4090, 4070, 272),
                                   (2040, 4000, 1552), (384, 2048, 16384), (1500, 3000, 2061)])
@pytest.mark.parametrize("blocks", [True, False], ids=["blocks", "rows"])
def test_large_products_of_whole_numbers(ctx, blocks, m, n, k):
    """Tiles of every size, with rows of whole vectors and without, splits, last tiles and last blocks of K that are not full."""
    a, sa = whole(m + k, m, k, 1)
    b, sb = whole(n + k, n, k, 128 if blocks else 1)
    x, y = a.float() * plain.spread(sa, a.shape).float(), b.float() * plain.spread(sb, b.shape).float()
    want = (x @ y.T)                                # (exact in float32 too: below 2^24 sixteenths)
    for out in (BF16, F32):
        to = Guarded((m, n), out)
        gr.dot_scaled(*(ctx.array(t.cuda()) for t in (a, sa, b, sb)), out=ctx.array(to.t))
        got = to.t.cpu()
        assert torch.equal(got, want.to(out)), int((got != want.to(out)).sum())
        assert to.untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,D", [(BF16, 4200, 4100), (F32, 2100, 4100), (F32, 140000, 70), (BF16, 70000, 300), (BF16, 2100, 8192), (F32, 600, 16000), (BF16, 1100, 16400)])
def test_large_norms(ctx, dtype, rows, D):
    """Tensors that go past the caches, and more rows than workgroups."""
    n = rows + D
    x, res, more = (normal(n + i, rows, D, dtype=dtype) for i in range(3))
    w = normal(n + 5, D, by=0.3)
    y, total = plain.norm(x, res, w, 1e-6, 1.0)
    gx, gres, gw = (ctx.array(t.cuda()) for t in (x, res, w))
    out, sums, _ = gr.rms_norm(gx, gw, gres, offset=1.0)
    assert torch.equal(sums.torch().cpu(), total)
    assert ((out.torch().cpu().double() - y).abs() <= (ROW + HALF[dtype]) * y.abs()).all()
    q, _, s = gr.rms_norm(gx, gw, gres, offset=1.0, eight=True, total=False)
    s = s.torch().cpu()
    v = y / plain.spread(s, y.shape)
    assert ((q.torch().float().cpu() - v).abs() <= plain.half_step(v.clamp(-448, 448)) + (ROW + 2.0 ** -22) * v.abs() + (v.abs() - 448).clamp(min=0)).all()
    dx, dw, size, terms = plain.norm_grad(more, total, w, x, 1e-6, 1.0)
    gdx, gdw = gr.rms_norm_grad(ctx.array(more.cuda()), sums, gw, dtotal=gx, offset=1.0)
    assert ((gdx.torch().cpu().double() - dx).abs() <= 4 * ROW * size + HALF[dtype] * dx.abs()).all()
    # (rows of a workgroup one after another, then of the workgroups: fewer than all rows)
    assert ((gdw.torch().cpu().double() - dw).abs() <= (ROW + (rows + 4) * 2.0 ** -24) * terms).all()


@pytest.mark.gpu
@pytest.mark.parametrize("blocks,transposed", [(False, False), (True, False), (False, True), (True, True)], ids=["rows", "blocks", "columns", "blocks_transposed"])
@pytest.mark.parametrize("dtype,m,k", [(BF16, 8300, 4100), (F32, 4099, 4100)])
def test_large_quantize(ctx, dtype, m, k, blocks, transposed):
    x = normal(m, m, k, dtype=dtype)
    q, s = gr.quantize(ctx.array(x.cuda()), blocks=blocks, transposed=transposed)
    exact = (x.T if transposed else x).contiguous()
    high = 128 if blocks else 1
    wide = torch.nn.functional.pad(exact.float(), (0, -exact.shape[1] % 128, 0, -exact.shape[0] % high)).abs()
    top = wide.view(wide.shape[0] // high, high, wide.shape[1] // 128, 128).amax((1, 3))
    assert torch.equal(s.torch().cpu(), top / 448.0)
    v = exact.double() / plain.spread(s.torch().cpu(), exact.shape)
    assert ((q.torch().float().cpu() - v).abs() <= plain.half_step(v.clamp(-448, 448)) + 2.0 ** -22 * v.abs() + (v.abs() - 448).clamp(min=0)).all()


@pytest.mark.gpu
def test_rows_far_apart(ctx):
    """Offsets beyond 2^31 and 2^32 bytes and elements, in operands and results."""
    step = (1 << 30) + 48
    flat = torch.empty(5 * step, dtype=torch.bfloat16, device="cuda")        # 10 GiB
    x = torch.as_strided(flat, (5, 520), (step, 1))
    vals = normal(4, 5, 520, dtype=BF16)
    x.copy_(vals.cuda())
    w = normal(5, 520)
    y, _ = plain.norm(vals, None, w, 1e-6, 0.0)
    out = torch.as_strided(flat, (5, 520), (step, 1), 4096)
    gr.rms_norm(ctx.array(x), ctx.array(w.cuda()), out=ctx.array(out))
    assert ((out.cpu().double() - y).abs() <= (ROW + HALF[BF16]) * y.abs()).all()
    dx, dw, size, terms = plain.norm_grad(vals, vals, w, None, 1e-6, 0.0)
    _, gw = gr.rms_norm_grad(ctx.array(x), ctx.array(x), ctx.array(w.cuda()), dx=ctx.array(out))
    assert ((out.cpu().double() - dx).abs() <= 4 * ROW * size + HALF[BF16] * dx.abs()).all()
    assert ((gw.torch().cpu().double() - dw).abs() <= (ROW + 9 * 2.0 ** -24) * terms).all()
    bytes_ = torch.empty(10 * step, dtype=torch.uint8, device="cuda").view(E4M3)
    q = torch.as_strided(bytes_, (5, 520), (2 * step, 1), 16384)
    for blocks in (False, True):
        q2, s2 = gr.quantize(ctx.array(x), blocks=blocks, out=ctx.array(q))
        want, ws = gr.quantize(ctx.array(vals.cuda()), blocks=blocks)
        assert torch.equal(q2.torch().float(), want.torch().float()) and torch.equal(s2.torch(), ws.torch())
    # a product of rows 2 GiB apart: few rows, and 40 of them 256 MiB apart, aligned and not
    b, sb = whole(1, 300, 520, 128)
    for rows, apart, off in ((5, 2 * step, 16384), (40, 1 << 28, 0), (40, (1 << 28) + 3, 1), (3, 2 * step + 5, 7)):
        a, sa = whole(rows, rows, 520, 1)
        far = torch.as_strided(bytes_, (rows, 520), (apart, 1), off)
        far.copy_(a.cuda())
        got = gr.dot_scaled(ctx.array(far), ctx.array(sa.cuda()), ctx.array(b.cuda()), ctx.array(sb.cuda()), dtype=gr.GR_F32).torch().cpu()
        assert torch.equal(got.double(), plain.product(a, sa, b, sb)[0])
        wide = torch.as_strided(flat.view(torch.float32), (rows, 300), (apart // 4 // 4 * 4, 1), 1 << 20)
        gr.dot_scaled(ctx.array(a.cuda()), ctx.array(sa.cuda()), ctx.array(b.cuda()), ctx.array(sb.cuda()), out=ctx.array(wide))
        assert torch.equal(wide.cpu(), got)
        back = gr.dot_scaled(ctx.array(b.cuda()), ctx.array(spread_rows(sb, 300).cuda()), ctx.array(far), ctx.array(sa.cuda()), dtype=gr.GR_F32).torch().cpu()
        assert torch.equal(back, got.T)


def spread_rows(blocks, rows):
    return blocks.repeat_interleave(128, 0)[:rows].contiguous()


@pytest.mark.gpu
def test_lazy_operands_and_pending_readers(ctx):
    """Operands that are expressions or views of expressions are evaluated first; what was recorded on a result's memory keeps what it was recorded with."""
    x, w = normal(1, 40, 256), normal(2, 256)
    gx, gw = ctx.array(x.cuda()), ctx.array(w.cuda())
    y, _ = plain.norm((x * 2 + 1)[:, 128:], None, (w * w)[:128], 1e-6, 0.0)
    out = gr.rms_norm((gx * 2 + 1)[:, 128:], (gw * gw)[:128])[0].torch().cpu()
    assert ((out.double() - y).abs() <= (ROW + HALF[F32]) * y.abs()).all()
    t = torch.ones(40, 256, device="cuda")
    at = ctx.array(t)
    reader = at + 1.0
    gr.rms_norm(gx, gw, out=at)
    assert bool((reader.torch() == 2.0).all()) and not bool((t == 1.0).all())
    q, s = gr.quantize(gx * 3.0)
    want = gr.quantize(ctx.array((x * 3.0).cuda()))
    assert torch.equal(q.torch().float(), want[0].torch().float()) and torch.equal(s.torch(), want[1].torch())
    # (a product's scales may be lazy too: here twice as large)
    a, sa = gr.quantize(gx)
    b, sb = gr.quantize(ctx.array(normal(3, 30, 256).cuda()), blocks=True)
    once, twice = gr.dot_scaled(a, sa, b, sb, dtype=gr.GR_F32), gr.dot_scaled(a, sa * 2.0, b, sb, dtype=gr.GR_F32)
    assert torch.equal(twice.torch(), once.torch() * 2)
    total = (gr.dot_scaled(a, sa, b, sb, dtype=gr.GR_F32) * 2.0).sum()                       # and results go on as lazy arrays
    assert abs(float(total.numpy()) - 2 * float(once.torch().double().sum())) <= 1e-5 * float(once.torch().double().abs().sum())


@pytest.mark.gpu
def test_captured_calls_replay(ctx):
    """Calls with temporary memory and without in a graph, replayed with other contents and eager calls between; a capture that would have to allocate is refused."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = gr.Context(stream=stream.cuda_stream)
        A = c.array
        rows, D, N = 96, 2048, 512
        x, res, dy = (torch.empty(rows, D, device="cuda", dtype=BF16) for _ in range(3))
        w = normal(1, D).cuda()
        b, sb = (t.torch() for t in gr.quantize(A(normal(2, N, D).cuda()), blocks=True))
        total, dx = torch.empty_like(x), torch.empty_like(x)
        q, s, dw = torch.empty(rows, D, device="cuda", dtype=E4M3), torch.empty(rows, D // 128, device="cuda"), torch.empty(D, device="cuda")
        y, qt, st = torch.empty(rows, N, device="cuda", dtype=BF16), torch.empty(D, rows, device="cuda", dtype=E4M3), torch.empty(D, 1, device="cuda")
        # (a product of many blocks and few tiles is split, and its parts are temporary memory)
        (p, sp), (v, sv) = ([t.torch() for t in gr.quantize(A(normal(3 + i, n, 16384).cuda()), blocks=i == 1)] for i, n in enumerate((rows, N)))
        z = torch.empty(rows, N, device="cuda")

        def fill(seed):
            for i, t in enumerate((x, res, dy)):
                t.copy_(normal(seed + i, rows, D, dtype=BF16))

        def step():
            gr.rms_norm(A(x), A(w), A(res), out=A(q), total=A(total), scales=A(s))
            gr.dot_scaled(A(q), A(s), A(b), A(sb), out=A(y))
            gr.dot_scaled(A(p), A(sp), A(v), A(sv), out=A(z))
            gr.rms_norm_grad(A(dy), A(total), A(w), dx=A(dx), dweight=A(dw))
            gr.quantize(A(dx), transposed=True, out=A(qt), scales=A(st))

        def results():
            return [t.float().clone() for t in (total, q, s, y, z, dx, dw, qt, st)]

        fill(10)
        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for seed in (20, 30, 40):
            fill(seed)
            step()
            want = results()
            for t in (total, q, s, y, z, dx, dw, qt, st):
                t.view(torch.uint8).zero_()
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(results(), want)), seed
            # an eager call that needs more temporary memory leaves the graph's where it is
            gr.rms_norm_grad(A(torch.zeros(seed * 40, 4096, device="cuda")), A(torch.ones(seed * 40, 4096, device="cuda")), A(torch.ones(4096, device="cuda")))
        del graph
        fresh = gr.Context(stream=stream.cuda_stream)
        F = fresh.array
        graph = torch.cuda.CUDAGraph()
        codes = []
        with torch.cuda.graph(graph, stream=stream):
            torch.zeros(1, device="cuda").add_(1)
            for call in (lambda: gr.rms_norm_grad(F(dy), F(total), F(w), dx=F(dx), dweight=F(dw)), lambda: gr.dot_scaled(F(p), F(sp), F(v), F(sv), out=F(z))):
                try:
                    call()
                    codes.append("none")
                except gr.GrError as e:
                    codes.append(e.code)
        assert codes == ["GR_ERR_OOM", "GR_ERR_OOM"]
        stream.synchronize()
        fresh.close()
        c.close()


@pytest.mark.gpu
def test_calls_on_a_stream_that_is_not_torchs(ctx):
    """The context's stream carries the work, and new results are taken for it."""
    stream = torch.cuda.Stream()
    c = gr.Context(stream=stream.cuda_stream)
    x, w = normal(7, 300, 1024, dtype=BF16), normal(8, 1024)
    gx, gw = x.cuda(), w.cuda()
    torch.cuda.synchronize()
    y, _ = plain.norm(x, None, w, 1e-6, 0.0)
    for _ in range(5):
        q, _, s = gr.rms_norm(c.array(gx), c.array(gw), eight=True)
        p = gr.dot_scaled(q, s, q, s, dtype=gr.GR_F32)
        c.sync()
        check_eight(q.torch().float().cpu(), s.torch().cpu(), y, off=ROW + 2.0 ** -22)
        want, size = plain.product(q.torch().cpu(), s.torch().cpu(), q.torch().cpu(), s.torch().cpu())
        assert ((p.torch().cpu().double() - want).abs() <= (127 * 2.0 ** -23 + 12 * 2.0 ** -24) * size).all()
    c.close()


@pytest.mark.gpu
def test_results_are_the_same_every_time(ctx):
    x, w, dy = normal(1, 3000, 1024, dtype=BF16).cuda(), normal(2, 1024).cuda(), normal(3, 3000, 1024, dtype=BF16).cuda()
    b, sb = gr.quantize(ctx.array(normal(4, 700, 1024).cuda()))
    first = None
    for _ in range(4):
        q, _, s = gr.rms_norm(ctx.array(x), ctx.array(w), eight=True)
        dx, dw = gr.rms_norm_grad(ctx.array(dy), ctx.array(x), ctx.array(w))
        got = [t.torch().float() for t in (q, s, dx, dw, gr.dot_scaled(q, s, b, sb), gr.dot_scaled(q, s, b, sb, dtype=gr.GR_F32), gr.dot_scaled(q[:40], s[:40], b, sb))]
        first = first or got
        assert all(torch.equal(u, v) for u, v in zip(first, got))


class EightProduct(torch.autograd.Function):
    """x W and its gradients in binary64, of the values that the 8-bit tensors of a layer stand for."""

    @staticmethod
    def rounded(x, blocks=False):
        s = plain.scales_of(x, blocks).float()
        each = plain.spread(s, x.shape)
        return (x.float() / each.float()).clamp(-448, 448).to(E4M3).double() * each

    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return EightProduct.rounded(x) @ EightProduct.rounded(w.T, True).T

    @staticmethod
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        return EightProduct.rounded(dy) @ EightProduct.rounded(w, True).T, EightProduct.rounded(x.T) @ EightProduct.rounded(dy.T).T


@pytest.mark.gpu
@pytest.mark.parametrize("norm,eight", [(True, False), (True, True), (False, True)], ids=["norm", "norm_eight", "eight"])
def test_layer_with_norm_and_eight_bits(norm, eight):
    """The layer's training step and its generation against the same in binary64 with automatic differentiation, 8-bit roundings included."""
    from paper_1901_03771_amd import attention_layer as al
    c = gr.Context()
    layer = al.AttentionLayer(c, width=144, heads=4, shared=2, values=24, cap=8.0, seed=4, norm=norm, eight=eight)
    g = torch.Generator().manual_seed(6)
    x, target = torch.randn(2, 70, 144, generator=g).cuda(), torch.randn(2, 70, 144, generator=g).cuda()
    if norm:
        layer.weights["gain"].copy_(1 + 0.2 * torch.randn(144, generator=g))
    w = {n: t.cpu().double().requires_grad_() for n, t in layer.weights.items()}
    times = EightProduct.apply if eight else torch.matmul

    def turned(t):
        a = torch.arange(70).double()[:, None, None] * torch.tensor(list(layer.frequencies), dtype=torch.float64)
        lo, hi = t[..., :12], t[..., 12:]
        return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)

    h = x.cpu().double().view(140, 144)
    if norm:
        h = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * w["gain"]
    q, k, v = turned(times(h, w["q"]).view(2, 70, 4, 24)), turned(times(h, w["k"]).view(2, 70, 2, 24)), times(h, w["v"]).view(2, 70, 2, 24)
    k, v = k.repeat_interleave(2, 2), v.repeat_interleave(2, 2)
    s = 8.0 * torch.tanh(torch.einsum("bihd,bjhd->bhij", q, k) * 24 ** -0.5 / 8.0)
    p = torch.softmax(s.masked_fill(torch.ones(70, 70, dtype=torch.bool).triu(1), -math.inf), -1)
    y = times(torch.einsum("bhij,bjhd->bihd", p, v).reshape(140, 96), w["o"])
    loss = ((y - target.cpu().double().view(140, 144)) ** 2).mean()
    loss.backward()
    before = {n: t.cpu().double() for n, t in layer.weights.items()}
    got = layer.train_step(x, target, 0, None, rate=1.0)
    # float32: a handful of products and sums of up to 144 values one after another, as for the layer without norm, and the norm's own error.
    bar = 6 * (140 + 144) * 2.0 ** -24 * 16
    if eight:
        # Two computations that agree to `bar` before a rounding to 8 bits fall to different sides of a middle where a value is that near to one: of the steps between numbers, 2^-4 of a value
        # at least, a share of 2 bar / 2^-4; there they differ by 2^-3 of the value, in norm by 2^-3 sqrt(share) of all.  Four roundings in a row, their gradients as many.
        bar = 8 * 2.0 ** -3 * math.sqrt(2 * bar / 2.0 ** -4)
    assert abs(got - loss.item()) <= bar * loss.item()
    for n, t in layer.weights.items():
        step = before[n] - t.cpu().double()
        assert (step - w[n].grad).norm() <= bar * w[n].grad.norm() + 2.0 ** -24 * before[n].norm(), n
    one = x[:, :20].contiguous()
    whole = layer.forward(one, 0, None)[0].torch().view(2, 20, 144)
    cache = [torch.full((2, 30, 2, 24), math.nan, device="cuda") for _ in range(2)]
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    for i in range(20):
        y1 = layer.step(one[:, i].contiguous(), *cache, lengths)
        assert (y1 - whole[:, i]).norm() <= bar * whole[:, i].norm(), i
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("arguments", [["--norm"], ["--norm", "--eight"]])
def test_layer_command_runs(arguments, capsys):
    from paper_1901_03771_amd import attention_layer as al
    al.main(arguments)
    assert "step 7: mean square" in capsys.readouterr().out


@pytest.mark.gpu
def test_a_step_of_a_layer_in_eight_bits(ctx):
    """The calls as they follow one another in training: norm, product, both gradients of the product, the norm's gradient; each against binary64 of what the one before it gave."""
    rows, D, N = 300, 520, 260
    x, res, dy = normal(1, rows, D, dtype=BF16), normal(2, rows, D, dtype=BF16, by=2.0), normal(3, rows, N, dtype=BF16)
    w, gain = normal(4, N, D, by=D ** -0.5), 1 + normal(5, D, by=0.2)
    A = lambda t: ctx.array(t.cuda())  # noqa: E731
    h8, stream, hs = gr.rms_norm(A(x), A(gain), A(res), eight=True)
    y64, total = plain.norm(x, res, gain, 1e-6, 0.0)
    assert torch.equal(stream.torch().cpu(), total)
    check_eight(h8.torch().float().cpu(), hs.torch().cpu(), y64, off=ROW + 2.0 ** -22)
    w8, ws = gr.quantize(A(w), blocks=True)
    out = gr.dot_scaled(h8, hs, w8, ws)
    want, size = plain.product(h8.torch().cpu(), hs.torch().cpu(), w8.torch().cpu(), ws.torch().cpu())
    room = 127 * 2.0 ** -23 + 16 * 2.0 ** -24
    assert ((out.torch().cpu().double() - want).abs() <= (room + 7 * 2.0 ** -13) * size + HALF[BF16] * want.abs()).all()
    # dx = dy W: the same blocks, transposed
    wt, wts = gr.quantize(A(w), blocks=True, transposed=True)
    assert torch.equal(wt.torch().float(), w8.torch().float().T) and torch.equal(wts.torch(), ws.torch().T)
    d8, ds = gr.quantize(A(dy))
    dh = gr.dot_scaled(d8, ds, wt, wts)
    want, size = plain.product(d8.torch().cpu(), ds.torch().cpu(), wt.torch().cpu(), wts.torch().cpu())
    assert ((dh.torch().cpu().double() - want).abs() <= (room + 7 * 2.0 ** -13) * size + HALF[BF16] * want.abs()).all()
    # dW = dy' h: sums over tokens
    h = gr.rms_norm(stream, A(gain))[0]
    dt, dts = gr.quantize(A(dy), transposed=True)
    ht, hts = gr.quantize(h, transposed=True)
    dw = gr.dot_scaled(dt, dts, ht, hts, dtype=gr.GR_F32)
    want, size = plain.product(dt.torch().cpu(), dts.torch().cpu(), ht.torch().cpu(), hts.torch().cpu())
    assert ((dw.torch().cpu().double() - want).abs() <= room * size).all()
    dx, dgain = gr.rms_norm_grad(dh, stream, A(gain), dtotal=A(dy[:, :1].expand(rows, D).contiguous()))
    want, wgain, size, terms = plain.norm_grad(dh.torch().cpu(), total, gain, dy[:, :1].expand(rows, D), 1e-6, 0.0)
    assert ((dx.torch().cpu().double() - want).abs() <= 4 * ROW * size + HALF[BF16] * want.abs()).all()
    assert ((dgain.torch().cpu().double() - wgain).abs() <= (ROW + (rows + 4) * 2.0 ** -24) * terms).all()
