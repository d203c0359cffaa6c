"""Norms, 8-bit tensors and their products as programs use them: a layer whose weights change, calls that fail after their launch, errors that other calls have
left."""
import ctypes

import pytest
import torch

from paper_1901_03771_amd import lazy as gr
from test_attention import Specs, dry, refused  # noqa: F401


# ---------------------------------------------------------------- without a GPU --
class FailsAfterwards:
    """The binding's C type, whose calls with kernels of their own run and then report a failure."""

    def __init__(self, real):
        self.real = real

    def __getattr__(self, name):
        f = getattr(self.real, name)
        if name not in ("rms_norm", "rms_norm_grad", "quantize", "dot_scaled"):
            return f

        def call(*a):
            st = f(*a)
            return 8 if st == 0 else st   # GR_ERR_HIP
        return call


def test_a_failure_after_a_launch_is_reported_and_the_call_not_repeated(dry, monkeypatch):  # noqa: F811
    """A norm in place that ran twice would have added its residual to its own result."""
    s = Specs(dry)
    x, res, out, w, dw, q, sc = s((6, 200)), s((6, 200)), s((6, 200)), s((200,)), s((200,)), s((6, 200), gr.GR_E4M3), s((6, 2))
    b, sb, y = s((70, 200), gr.GR_E4M3), s((70, 2)), s((6, 70))
    monkeypatch.setattr(gr, "_fastbind", FailsAfterwards(gr._fastbind))
    for call, launches in ((lambda: gr.rms_norm(x, w, res, out=x, total=res), 1), (lambda: gr.rms_norm(x, w, res, out=q, total=res, scales=sc), 1),
                           (lambda: gr.rms_norm(x, out=q, scales=sc, eight=True), 1), (lambda: gr.rms_norm(x, w, res, out=out, total=False), 1),
                           (lambda: gr.rms_norm_grad(x, res, w, dx=out, dweight=dw), 2), (lambda: gr.quantize(x, out=q, scales=sc), 1),
                           (lambda: gr.dot_scaled(q, sc, b, sb, out=y), 1)):
        n = dry.stats()["kernel_launches"]
        refused("GR_ERR_HIP", call)
        assert dry.stats()["kernel_launches"] == n + launches


def test_an_8_bit_result_without_scales_goes_the_longer_way_at_once(dry, monkeypatch):  # noqa: F811
    """No call of the library is refused on the way to the new scales."""
    s = Specs(dry)
    x, q = s((6, 200)), s((6, 200), gr.GR_E4M3)
    answers = []

    class Watched(FailsAfterwards):
        def __getattr__(self, name):
            f = getattr(self.real, name)
            return (lambda *a: answers.append(f(*a)) or answers[-1]) if name == "rms_norm" else f
    monkeypatch.setattr(gr, "_fastbind", Watched(gr._fastbind))
    refused("GR_ERR_NODEVICE", gr.rms_norm, x, out=q)                     # (a dry context has no memory for new scales)
    assert answers == [None]


# ------------------------------------------------------------------- on the GPU --
def wide_layer(c, norm, eight=True):
    from paper_1901_03771_amd import attention_layer as al
    return al.AttentionLayer(c, width=144, heads=4, shared=2, values=24, cap=8.0, seed=4, norm=norm, eight=eight)


def results_of(layer, **laid):
    """What the layer answers for the same rows: of a forward pass, its gradients and two tokens of generation."""
    g = torch.Generator().manual_seed(7)
    x, dy = torch.randn(2, 70, 144, generator=g).cuda(), torch.randn(140, 144, generator=g).cuda()
    y, kept = layer.forward(x, 0, None, **laid)
    got = {"y": y.torch(), **{n: t.torch() for n, t in layer.gradients(layer.ctx.array(dy), kept).items()}}
    cache = [torch.zeros(2, 4, 2, 24, device="cuda") for _ in range(2)]
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    for i in range(2):
        got[f"token {i}"] = layer.step(x[:, i].contiguous(), *cache, lengths, **laid)
    return got


def same(a, b):
    return {n for n in a if torch.equal(a[n], b[n])}


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [False, True], ids=["plain", "norm"])
def test_layer_in_eight_bits_takes_its_weights_as_they_are(norm):
    """Weights that a caller's own optimizer, a checkpoint or an assignment through the lazy arrays has changed, between calls that have used them."""
    c = gr.Context()
    layer, other = wide_layer(c, norm), wide_layer(c, norm)
    first = results_of(layer)
    g = torch.Generator().manual_seed(8)
    new = {n: t.cpu() + 0.1 * torch.randn(t.shape, generator=g) for n, t in layer.weights.items()}
    changes = [lambda t, v: t.copy_(v), lambda t, v: t.data.copy_(v), lambda t, v: c.array(t).__setitem__((slice(None),) * t.dim(), c.array(v) * 1.0)]
    for i, (name, t) in enumerate(layer.weights.items()):
        v = new[name].cuda()
        changes[i % 3](t, v)
        assert torch.equal(t, v)
        other.weights[name].copy_(v)
    torch.cuda.synchronize()
    now, want = results_of(layer), results_of(other)      # (the other layer's first calls)
    assert same(now, want) == set(want) and not same(now, first)
    c.close()


@pytest.mark.gpu
def test_layer_with_weights_that_a_program_has_laid_out():
    """They give what the weights gave that they were made of, until the program makes them anew; the gradients are always of the weights themselves."""
    c = gr.Context()
    layer = wide_layer(c, True)
    first, laid = results_of(layer), layer.laid_out()
    assert same(results_of(layer, laid=laid), first) == set(first)
    for t in layer.weights.values():
        t.mul_(1.25)
    now, old = results_of(layer), results_of(layer, laid=laid)
    assert not same(now, first) and not same(now, old)
    assert same(results_of(layer, laid=layer.laid_out()), now) == set(first)
    assert wide_layer(c, True, eight=False).laid_out() is None
    with pytest.raises(ValueError):
        results_of(wide_layer(c, True, eight=False), laid=laid)
    c.close()


@pytest.mark.gpu
def test_an_error_that_an_earlier_call_left_is_not_taken_for_the_launchs():
    """HIP keeps a thread's last error until somebody asks for it: a launch that goes through is not failed by it."""
    hip = gr.lib()                                                           # (its dependencies' names are found through it)
    hip.hipSetDevice.argtypes, hip.hipSetDevice.restype = [ctypes.c_int], ctypes.c_int
    c = gr.Context()
    A = c.array
    leave = lambda: hip.hipSetDevice(1 << 20)  # noqa: E731  (refused by the runtime)
    x, w, one = torch.randn(40, 256, device="cuda"), torch.randn(256, device="cuda"), torch.ones(40, 256, device="cuda")
    heads = torch.randn(1, 40, 2, 64, device="cuda")
    torch.cuda.synchronize()
    b, sb = gr.quantize(A(w[None].expand(30, 256).contiguous()))

    def calls():
        total, normed, copy = x.clone(), one.clone(), torch.empty(40, 256, device="cuda")
        torch.cuda.synchronize()

        def run(f):
            assert leave() != 0
            return f()
        run(lambda: gr.rms_norm(A(normed), A(w), A(total), out=A(normed), total=A(total)))     # once: the residual is added to the stream in place
        q, s = run(lambda: gr.quantize(A(x)))
        y = run(lambda: gr.dot_scaled(q, s, b, sb))
        dx, dw = run(lambda: gr.rms_norm_grad(A(one), A(x), A(w)))
        out, _ = run(lambda: gr.attention(A(heads), A(heads), A(heads), c.scores()))
        turned = run(lambda: gr.rotary(A(heads), gr.rotary_frequencies(64), 3))
        run(lambda: c.stream_copy(copy, x))
        got = [total, normed, *(t.torch().float() for t in (q, s, y, dx, dw, out, turned)), copy]
        c.sync()
        return got

    got = calls()
    leave = lambda: 1  # noqa: E731
    assert all(torch.equal(a, b) for a, b in zip(got, calls()))
    assert torch.equal(got[0], x + 1) and torch.equal(got[-1], x)
    c.close()


@pytest.mark.gpu
def test_an_error_that_an_earlier_call_left_is_not_taken_for_the_interpreters():
    hip = gr.lib()
    hip.hipSetDevice.argtypes, hip.hipSetDevice.restype = [ctypes.c_int], ctypes.c_int
    c = gr.Context()
    c.set_option("interp", 2)
    x = torch.rand(300, 200, device="cuda")
    a = c.array(x)
    for f, want in ((lambda: gr.exp(a * 0.5) + 0.25, torch.exp(x * 0.5) + 0.25), (lambda: (a * 3.0).sum(axis=1), (x * 3.0).sum(1)), (lambda: a.cumsum(0), x.cumsum(0))):
        assert hip.hipSetDevice(1 << 20) != 0
        assert torch.allclose(f().torch(), want, rtol=1e-4)   # (of up to 300 positive values: 300 2^-24 each)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(1 << 18, 1 << 18), (449, (1 << 27) - 127)])
def test_a_product_over_nothing_of_as_many_tiles_as_a_launch_holds(m, n):
    """2^22 tiles of 128 x 128: with twice as many of 64 x 128 the launch would pass 2^32 threads.  All results are zero, and written."""
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("128 GiB of results")
    c = gr.Context()
    none = lambda *shape, dtype=torch.uint8: torch.empty(*shape, device="cuda", dtype=dtype)  # noqa: E731
    out = torch.empty(m * n, dtype=torch.bfloat16, device="cuda").fill_(3.0).view(m, n)
    gr.dot_scaled(*(c.array(t) for t in
                     (none(m, 0).view(torch.float8_e4m3fn), none(m, 0, dtype=torch.float32), none(n, 0).view(torch.float8_e4m3fn), none((n + 127) // 128, 0, dtype=torch.float32))), out=c.array(out))
    assert not any(bool(part.any()) for part in out.view(torch.int16).flatten().split(1 << 33))
    del out
    torch.cuda.empty_cache()
    c.close()
