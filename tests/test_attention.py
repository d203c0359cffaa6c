"""Attention, its gradient, single-token steps and rotary positions (include/grumpy_hip_attention.h) against plain binary64 forms
(attention_reference.py), and what the calls refuse."""
import ctypes
import math

import pytest
import torch

import attention_reference as plain
from paper_1901_03771_amd import lazy as gr

F32, BF16 = torch.float32, torch.bfloat16
NAMES = {F32: "f32", BF16: "bf16"}


# ---------------------------------------------------------------- without a GPU --
@pytest.fixture()
def dry():
    c = gr.Context(device=-1)
    c.set_option("dry_run", 2)
    yield c
    c.close()


def refused(code, call, /, *a, **kw):
    with pytest.raises(gr.GrError) as e:
        call(*a, **kw)
    assert e.value.code == code, e.value


class Specs:
    """Leaves at addresses of their own that are never read."""

    def __init__(self, ctx):
        self.ctx, self.at = ctx, 1 << 20

    def __call__(self, shape, dtype=gr.GR_F32, strides=None, off=0):
        n = 1
        for s in shape:
            n *= max(s, 1)
        a = self.ctx.from_device(self.at + off, dtype, tuple(shape), strides)
        self.at += (64 * n + 8191) // 4096 * 4096
        return a


@pytest.mark.parametrize("dtype", [gr.GR_F32, gr.GR_BF16])
def test_calls_run_dry_and_count_their_launches(dry, dtype):
    s = Specs(dry)
    q, k, v, o, do, dq = (s((2, 40, 6, 64), dtype) for _ in range(6))
    k2, v2, dk, dv = (s((2, 50, 2, 64), dtype) for _ in range(4))
    lse = s((2, 6, 40))
    sc = dry.scores(cap=30.0, slopes=s((6,)), causal=True, position=10, prefix=s((2,), gr.GR_I32), lengths=s((2,), gr.GR_I32),
                    documents=(s((2, 40), gr.GR_I32), s((2, 50), gr.GR_I32)))
    before = dry.stats()["kernel_launches"]
    gr.attention(q, k2, v2, sc, out=o, lse=lse)
    gr.attention_grad(do, q, k2, v2, sc, o, lse, dq=dq, dk=dk, dv=dv)
    assert dry.stats()["kernel_launches"] >= before + 5
    gr.attention_step(s((2, 6, 64), dtype), k2, v2, dry.scores(lengths=s((2,), gr.GR_I32)), out=s((2, 6, 64), dtype))
    gr.rotary(q, gr.rotary_frequencies(64), 5, out=q)
    gr.rotary(q, gr.rotary_frequencies(32), s((2, 40), gr.GR_I32), interleaved=True, inverse=True, out=o)


def test_refusals(dry):
    s = Specs(dry)
    q, k, v, o = s((2, 8, 4, 64)), s((2, 9, 2, 64)), s((2, 9, 2, 64)), s((2, 8, 4, 64))
    lse, i2 = s((2, 4, 8)), s((2,), gr.GR_I32)
    ok = dry.scores()
    call = lambda sc=ok, q=q, k=k, v=v, o=o, lse=lse, rest=None: gr.attention(q, k, v, sc, out=o, lse=lse, rest=rest)  # noqa: E731
    call()
    refused("GR_ERR_SHAPE", call, q=s((2, 8, 3, 64)))                       # 3 heads on 2
    refused("GR_ERR_SHAPE", call, q=s((8, 4, 64)))
    refused("GR_ERR_SHAPE", call, v=s((2, 10, 2, 64)))
    refused("GR_ERR_SHAPE", call, k=s((2, 9, 2, 32)))
    refused("GR_ERR_SHAPE", call, o=s((2, 8, 4, 32)))
    refused("GR_ERR_SHAPE", call, lse=s((2, 8, 4)))
    refused("GR_ERR_UNSUPPORTED", call, q=s((2, 8, 4, 257)), k=s((2, 9, 2, 257)), v=s((2, 9, 2, 257)), o=s((2, 8, 4, 257)))
    refused("GR_ERR_UNSUPPORTED", call, q=s((2, 8, 4, 0)), k=s((2, 9, 2, 0)), v=s((2, 9, 2, 0)), o=s((2, 8, 4, 0)))
    refused("GR_ERR_DTYPE", call, q=s((2, 8, 4, 64), gr.GR_I32))
    refused("GR_ERR_DTYPE", call, k=s((2, 9, 2, 64), gr.GR_BF16))
    refused("GR_ERR_DTYPE", call, rest=s((2, 8, 4, 64)))                    # f32 results are not rounded further
    refused("GR_ERR_UNSUPPORTED", call, q=s((2, 8, 4, 64), strides=(4096, 256, 64, 2)))
    refused("GR_ERR_UNSUPPORTED", call, o=s((2, 8, 4, 64), strides=(4096, 0, 64, 1)))
    refused("GR_ERR_UNSUPPORTED", call, o=s((2, 8, 4, 64), strides=(4096, 32, 64, 1)))
    refused("GR_ERR_UNSUPPORTED", call, lse=s((2, 4, 8), strides=(64, 8, 1)))
    refused("GR_ERR_UNSUPPORTED", call, o=s((2, 8, 4, 64)) + 1.0)           # nothing to write to
    refused("GR_ERR_ALIAS", call, o=q)
    refused("GR_ERR_ARG", call, dry.scores(scale=0.0))
    refused("GR_ERR_ARG", call, dry.scores(scale=math.nan))
    refused("GR_ERR_ARG", call, dry.scores(scale=-1.0))
    refused("GR_ERR_ARG", call, dry.scores(cap=-1.0))
    refused("GR_ERR_ARG", call, dry.scores(cap=math.inf))
    refused("GR_ERR_ARG", call, dry.scores(prefix=i2))
    refused("GR_ERR_ARG", call, dry.scores(position=1 << 40))
    refused("GR_ERR_SHAPE", call, dry.scores(slopes=s((2,))))
    refused("GR_ERR_DTYPE", call, dry.scores(slopes=s((4,), gr.GR_I32)))
    refused("GR_ERR_DTYPE", call, dry.scores(lengths=s((2,))))
    refused("GR_ERR_SHAPE", call, dry.scores(lengths=s((3,), gr.GR_I32)))
    refused("GR_ERR_ARG", call, dry.scores(documents=(s((2, 8), gr.GR_I32), None)))
    refused("GR_ERR_SHAPE", call, dry.scores(documents=s((2, 8), gr.GR_I32)))
    d = [s((2, 8, 4, 64)), s((2, 9, 2, 64)), s((2, 9, 2, 64))]
    grad = lambda **kw: gr.attention_grad(s((2, 8, 4, 64)), q, k, v, ok, o, lse, **{**dict(dq=d[0], dk=d[1], dv=d[2]), **kw})  # noqa: E731
    grad()
    refused("GR_ERR_ALIAS", grad, dv=d[1])
    refused("GR_ERR_ALIAS", grad, dk=k)
    refused("GR_ERR_SHAPE", grad, dq=d[1])
    st = lambda sc, q=s((2, 4, 64)), o=s((2, 4, 64)): gr.attention_step(q, k, v, sc, out=o)  # noqa: E731
    st(dry.scores(lengths=i2))
    refused("GR_ERR_ARG", st, ok)                                           # no lengths
    refused("GR_ERR_ARG", st, dry.scores(lengths=i2, causal=True))
    refused("GR_ERR_SHAPE", st, dry.scores(lengths=i2), q=q)
    rot = lambda x=q, f=gr.rotary_frequencies(64), p=0, o=o, **kw: gr.rotary(x, f, p, out=o, **kw)  # noqa: E731
    rot()
    refused("GR_ERR_SHAPE", rot, f=gr.rotary_frequencies(66))
    refused("GR_ERR_ARG", rot, f=[math.inf])
    refused("GR_ERR_ARG", rot, f=gr.rotary_frequencies(514))
    refused("GR_ERR_ARG", rot, factor=math.nan)
    refused("GR_ERR_SHAPE", rot, p=s((2, 9), gr.GR_I32))
    refused("GR_ERR_DTYPE", rot, p=s((2, 8)))
    refused("GR_ERR_DTYPE", rot, x=s((2, 8, 4, 64), gr.GR_I32))
    # NULL scores, dead handles
    L, u = gr.lib(), ctypes.c_uint64
    assert L.gr_attention(dry._p, None, q.h, k.h, v.h, o.h, 0, 0) == 6
    assert L.gr_attention_step(dry._p, None, 1 << 40, k.h, v.h, o.h) == 1
    assert L.gr_attention(None, None, u(1), u(1), u(1), u(1), u(0), u(0)) == 6


def test_calls_beyond_a_launch_are_refused(dry):
    """2^24 heads and documents of 2^32 entries: no launch holds them; nothing is launched."""
    a = lambda B, N, H, t=gr.GR_F32: dry.from_device(1 << 40, t, (B, N, H, 64))  # noqa: E731
    at = [1 << 41]

    def result(*shape):
        at[0] += 1 << 44
        return dry.from_device(at[0], gr.GR_F32, shape)

    n = dry.stats()["kernel_launches"]
    B = 1 << 24
    refused("GR_ERR_UNSUPPORTED", gr.attention, a(B, 1, 1), a(B, 1, 1), a(B, 1, 1), dry.scores(), out=result(B, 1, 1, 64), lse=result(B, 1, 1))
    refused("GR_ERR_UNSUPPORTED", gr.attention_step, dry.from_device(1 << 40, gr.GR_F32, (B, 1, 64)), a(B, 1, 1), a(B, 1, 1), dry.scores(lengths=dry.from_device(1 << 40, gr.GR_I32, (B,))),
            out=result(B, 1, 64))
    B = 1 << 21
    refused("GR_ERR_UNSUPPORTED", gr.attention_grad, *[a(B, 1, 1)] * 4, dry.scores(), a(B, 1, 1), dry.from_device(1 << 40, gr.GR_F32, (B, 1, 1)),
            **{w: result(B, 1, 1, 64) for w in ("dq", "dk", "dv")})
    ids = lambda n: dry.from_device(1 << 40, gr.GR_I32, (1 << 20, n), (0, 1))  # noqa: E731
    wide = lambda n: dry.from_device(1 << 40, gr.GR_F32, (1 << 20, n, 1, 64), (0, 64, 64, 1))  # noqa: E731
    refused("GR_ERR_UNSUPPORTED", gr.attention, wide(1), wide(8192), wide(8192), dry.scores(documents=(ids(1), ids(8192))), out=result(1 << 20, 1, 1, 64), lse=result(1 << 20, 1, 1))
    assert dry.stats()["kernel_launches"] == n


@pytest.mark.parametrize("of", ["slice", "transpose", "scan"])
def test_lazy_views_of_lse_are_looked_at_once_evaluated(dry, of):
    """A view of an expression keeps its steps when the expression is evaluated: one that is not dense is refused, like one of a stored array."""
    s = Specs(dry)
    q, k, v, o, do = (s((1, 8, 2, 64)) for _ in range(5))
    dense = lambda: gr.dot(s((2, 8)), s((8, 8)))  # noqa: E731
    lse = {"slice": lambda: gr.reshape(gr.dot(s((2, 8)), s((8, 16))), (1, 2, 16))[:, :, :8],
           "transpose": lambda: gr.reshape(gr.dot(s((8, 2)), s((2, 2))), (8, 2, 1)).T,
           "scan": lambda: s((1, 2, 16)).cumsum(2)[:, :, :8]}[of]()
    assert lse.shape == (1, 2, 8)
    results = lambda: {w: s((1, 8, 2, 64)) for w in ("dq", "dk", "dv")}  # noqa: E731
    refused("GR_ERR_UNSUPPORTED", gr.attention_grad, do, q, k, v, dry.scores(), o, lse, **results())
    refused("GR_ERR_UNSUPPORTED", gr.attention_grad, do, q, k, v, dry.scores(), o, lse, **results())   # (stored by now)
    gr.attention_grad(do, q, k, v, dry.scores(), o, gr.reshape(dense(), (1, 2, 8)), **results())
    # values of a row that are not neighbours are refused likewise
    wide = gr.reshape(gr.dot(s((8, 8)), s((8, 256))), (1, 8, 2, 128))[:, :, :, ::2]
    refused("GR_ERR_UNSUPPORTED", gr.attention, wide, k, v, dry.scores(), out=s((1, 8, 2, 64)), lse=False)


def test_without_a_device_arguments_are_checked_first():
    c = gr.Context(device=-1)
    s = Specs(c)
    q, k = s((1, 8, 4, 64)), s((1, 8, 4, 64))
    refused("GR_ERR_NODEVICE", gr.attention, q, k, s((1, 8, 4, 64)), c.scores(), out=s((1, 8, 4, 64)), lse=False)
    refused("GR_ERR_SHAPE", gr.attention, q, k, s((1, 9, 4, 64)), c.scores(), out=s((1, 8, 4, 64)), lse=False)
    refused("GR_ERR_NODEVICE", gr.rotary, q, gr.rotary_frequencies(64), 0, out=k)
    c.close()


def test_bf16_arrays_go_nowhere_else(dry):
    s = Specs(dry)
    a, b = s((4, 8), gr.GR_BF16), s((4, 8))
    for f in (lambda: a + 1.0, lambda: a + a, lambda: a + b, lambda: -a, lambda: gr.exp(a), lambda: a.sum(), lambda: a.cumsum(0), lambda: a.reshape(32),
              lambda: gr.dot(a, a), lambda: a[1:] * 2.0):
        refused("GR_ERR_DTYPE", f)

    def assign():
        a[1:] = s((3, 8), gr.GR_BF16)
    refused("GR_ERR_DTYPE", assign)
    refused("GR_ERR_DTYPE", lambda: a[1:].plan())
    assert a[1:, 2:].shape == (3, 6) and a.T.shape == (8, 4) and a[1:].dtype_code == gr.GR_BF16
    assert a[1:, 2:].data_ptr()[0] == a.data_ptr()[0] + 2 * (8 + 2)


def test_packed_results_are_told_from_overlapping_ones(dry):
    s = Specs(dry)
    q, k, v, o, do, lse = s((2, 8, 4, 64)), s((2, 8, 4, 64)), s((2, 8, 4, 64)), s((2, 8, 4, 64)), s((2, 8, 4, 64)), s((2, 4, 8))
    base, row = s.at, 3 * 4 * 64
    s.at += 1 << 20
    part = lambda off, heads=4: dry.from_device(base + 4 * off, gr.GR_F32, (2, 8, heads, 64), (8 * row, row, 64, 1))  # noqa: E731
    gr.attention_grad(do, q, k, v, dry.scores(), o, lse, dq=part(0), dk=part(256), dv=part(512))
    refused("GR_ERR_ALIAS", gr.attention_grad, do, q, k, v, dry.scores(), o, lse, dq=part(0), dk=part(255), dv=part(512))
    refused("GR_ERR_ALIAS", gr.attention_grad, do, q, k, v, dry.scores(), o, lse, dq=part(0), dk=part(256), dv=part(768))   # the next row
    refused("GR_ERR_ALIAS", gr.attention_grad, do, part(0), k, v, dry.scores(), o, lse, dq=part(0), dk=part(256), dv=part(512))


def test_frequencies():
    f = gr.rotary_frequencies(8, base=100.0)
    assert [round(x, 12) for x in f] == [round(100.0 ** (-i / 4), 12) for i in range(4)]
    assert all(a == b / 4 for a, b in zip(gr.rotary_frequencies(8, 100.0, stretch=4.0), f))
    g = gr.rotary_frequencies(64, stretch=8.0, context=4096)
    plain_f = gr.rotary_frequencies(64)
    assert g[0] == plain_f[0] and g[31] == plain_f[31] / 8 and all(a <= b <= 8 * a * (1 + 1e-12) for a, b in zip(g, plain_f))
    with pytest.raises(ValueError):
        gr.rotary_frequencies(7)


@pytest.mark.parametrize("of", [list, tuple, lambda f: (ctypes.c_float * len(f))(*f), lambda f: torch.tensor(f), lambda f: torch.tensor(f).numpy()])
def test_frequencies_of_every_kind_are_read_as_numbers(dry, of):
    """Also arrays of single precision, which are half as long: what is not finite in them is found, what is finite is taken."""
    x = Specs(dry)((1, 4, 2, 64))
    gr.rotary(x, of([0.5] * 32), 5, out=x)
    refused("GR_ERR_ARG", gr.rotary, x, of([math.inf] * 32), 5, out=x)


def test_numbers_are_not_cut_to_fit(dry):
    x = Specs(dry)((1, 4, 2, 64))
    f = gr.rotary_frequencies(64)
    for p in (1 << 64, 1 << 70, -(1 << 64), 1 << 41):
        refused("GR_ERR_ARG", gr.rotary, x, f, p, out=x)
    for p in (1 << 64, -(1 << 70)):
        refused("GR_ERR_ARG", dry.scores, position=p)
    for p in (2.5, "3"):
        with pytest.raises(TypeError):
            gr.rotary(x, f, p, out=x)
        with pytest.raises(TypeError):
            dry.scores(position=p)
    for factor in (1e39, -1e300, math.inf, math.nan):
        refused("GR_ERR_ARG", gr.rotary, x, f, 5, factor=factor, out=x)


def test_scales_and_caps_that_no_float_holds_are_refused(dry):
    """A factor that is zero or infinite as a float would make NaN of masked scores and of zeros."""
    s = Specs(dry)
    q, o, lse, d = s((1, 4, 2, 64)), s((1, 4, 2, 64)), s((1, 2, 4)), [s((1, 4, 2, 64)) for _ in range(3)]
    one, to, n = s((1, 2, 64)), s((1, 2, 64)), s((1,), gr.GR_I32)
    for kw in (dict(scale=1e-46), dict(scale=1e-320), dict(scale=1e-29), dict(scale=1e30), dict(scale=1e29, cap=1e-29), dict(scale=1e-27, cap=1e29), dict(cap=1e-31),
               dict(cap=1e30), dict(cap=math.nan), dict(scale=math.inf)):
        refused("GR_ERR_ARG", gr.attention, q, q, q, dry.scores(causal=True, **kw), out=o, lse=lse)
        refused("GR_ERR_ARG", gr.attention_grad, q, q, q, q, dry.scores(causal=True, **kw), q, lse, dq=d[0], dk=d[1], dv=d[2])
        refused("GR_ERR_ARG", gr.attention_step, one, q, q, dry.scores(lengths=n, **kw), out=to)
    for kw in (dict(scale=1e-27), dict(scale=1e29), dict(scale=1e29, cap=1e-8), dict(cap=1e-29), dict(scale=1e-7, cap=9e29)):
        gr.attention(q, q, q, dry.scores(causal=True, **kw), out=o, lse=lse)


def test_queries_far_from_all_keys_under_a_bias_are_refused(dry):
    """Behind 2^24 positions f32 holds no single distance, and no lse of which the gradient could form a probability again."""
    s = Specs(dry)
    q, k, o, lse, slopes = s((1, 5, 2, 64)), s((1, 9, 2, 64)), s((1, 5, 2, 64)), s((1, 2, 5)), s((2,))
    far = 1 << 24
    for position, ok in ((9 + far, True), (10 + far, False), (-far - 5, True), (-far - 6, False), (-(1 << 31), False), (1 << 31, False)):
        for sc, may in ((dry.scores(slopes=slopes, position=position), ok), (dry.scores(position=position), True)):
            calls = [lambda: gr.attention(q, k, k, sc, out=o, lse=lse),
                     lambda: gr.attention_grad(q, q, k, k, sc, q, lse, dq=o, dk=s((1, 9, 2, 64)), dv=s((1, 9, 2, 64)))]
            for call in calls:
                if may:
                    call()
                else:
                    refused("GR_ERR_ARG", call)


def test_what_python_is_given_wrong_is_said_so(dry):
    """Element types, ranks and objects that do not fit, with and without results given; a context without a device has no memory for new ones."""
    s = Specs(dry)
    ok, f, i, none, lse = dry.scores(), s((1, 4, 2, 64)), s((1, 4, 2, 64), gr.GR_I32), s(()), s((1, 2, 4))
    one = s((1, 2, 64))
    refused("GR_ERR_DTYPE", gr.attention, i, i, i, ok)
    refused("GR_ERR_DTYPE", gr.attention_step, s((1, 2, 64), gr.GR_I32), i, i, ok)
    refused("GR_ERR_DTYPE", gr.attention_grad, i, i, i, i, ok, i, lse)
    refused("GR_ERR_DTYPE", gr.rotary, i, gr.rotary_frequencies(64))
    refused("GR_ERR_SHAPE", gr.attention, none, f, f, ok)
    refused("GR_ERR_SHAPE", gr.attention, none, f, f, ok, out=s((1, 4, 2, 64)), lse=False)
    refused("GR_ERR_SHAPE", gr.attention_step, none, f, f, ok, out=one)
    refused("GR_ERR_SHAPE", gr.attention_grad, f, none, f, f, ok, f, lse, dq=s((1, 4, 2, 64)), dk=s((1, 4, 2, 64)), dv=s((1, 4, 2, 64)))
    refused("GR_ERR_NODEVICE", gr.attention, f, f, f, ok)
    refused("GR_ERR_NODEVICE", gr.rotary, f, gr.rotary_frequencies(64))
    for q in (1.0, None, torch.ones(1, 4, 2, 64)):
        for call in (lambda: gr.attention(q, f, f, ok), lambda: gr.attention(f, q, f, ok, out=one, lse=False), lambda: gr.attention_step(q, f, f, ok),
                     lambda: gr.attention_grad(f, q, f, f, ok, f, lse), lambda: gr.rotary(q, gr.rotary_frequencies(64))):
            with pytest.raises(TypeError):
                call()
    for bad in (0.5, torch.zeros(2), [1.0, 2.0]):
        for name in ("slopes", "prefix", "lengths", "documents"):
            with pytest.raises((TypeError, ValueError)):
                dry.scores(**{name: bad, "causal": True})
    for sc in (None, 1.0, gr._Scores()):
        with pytest.raises(TypeError):
            gr.attention(f, f, f, sc, out=s((1, 4, 2, 64)), lse=False)


def test_scores_of_another_context(dry):
    """Handles are numbers of a context: the same number names another array in the next."""
    other = gr.Context(device=-1)
    s = Specs(dry)
    q, o, lse = s((1, 4, 2, 64)), s((1, 4, 2, 64)), s((1, 2, 4))
    slopes = Specs(other)((2,))
    for sc in (other.scores(slopes=slopes), other.scores()):
        with pytest.raises(ValueError):
            gr.attention(q, q, q, sc, out=o, lse=lse)
        with pytest.raises(ValueError):
            gr.attention_grad(q, q, q, q, sc, q, lse, dq=o, dk=s((1, 4, 2, 64)), dv=s((1, 4, 2, 64)))
        with pytest.raises(ValueError):
            gr.attention_step(s((1, 2, 64)), q, q, sc, out=s((1, 2, 64)))
    other.close()


def test_reference_gradient_against_differences():
    """The formulas that the kernels are compared with, against central differences of the plain output."""
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(1, 5, h, 6, generator=g, dtype=torch.float64) for h in (4, 2, 2))
    w = torch.randn(1, 5, 4, 6, generator=g, dtype=torch.float64)
    kw = dict(cap=2.0, slopes=[0.5, 0.25, 0.1, 0.0], causal=True, prefix=torch.tensor([2]), documents=torch.tensor([[0, 0, 0, 1, 1]]))
    ref = plain.attention(q, k, v, w, **kw)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        for at in [(0, 0, 0, 0), (0, 3, 1, 5), (0, 4, 1, 2), (0, 1, 0, 3)]:
            e = torch.zeros_like(t)
            e[at] = 1e-5
            i = ("dq", "dk", "dv").index(name)
            up = [x + e if n == i else x for n, x in enumerate((q, k, v))]
            dn = [x - e if n == i else x for n, x in enumerate((q, k, v))]
            slope = ((plain.attention(*up, **kw)["out"] - plain.attention(*dn, **kw)["out"]) * w).sum() / 2e-5
            assert abs(float(slope - ref[name][at])) < 1e-7, (name, at)


# ------------------------------------------------------------------- on the GPU --
@pytest.fixture(scope="module")
def ctx():
    c = gr.Context()
    yield c
    c.close()


def normal(seed, *shape, dtype=F32, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * by).to(dtype).cuda()


def case(B, N, M, H, HK, D, dtype, grad=True, **kw):
    name = "-".join(str(x) for x in (B, N, M, H, HK, D)) + "-" + NAMES[dtype] + "".join(f"-{k}{'' if v is True else v}" for k, v in kw.items())
    return pytest.param(dict(B=B, N=N, M=M, H=H, HK=HK, D=D, dtype=dtype, grad=grad, **kw), id=name)


def options(c, seed=0):
    """The tensors that a case's options name."""
    g = torch.Generator().manual_seed(1000 + seed)
    B, N, M = c["B"], c["N"], c["M"]
    kw = dict(cap=c.get("cap", 0.0), causal=c.get("causal", False), position=c.get("position", 0))
    if "scale" in c:
        kw["scale"] = c["scale"]
    if c.get("slopes"):
        kw["slopes"] = torch.tensor([2.0 ** -(1 + i % 7) for i in range(c["H"])])
    if c.get("prefix"):
        kw["prefix"] = torch.randint(0, M + 2, (B,), generator=g, dtype=torch.int32)
    if c.get("lengths"):
        kw["lengths"] = torch.randint(-1, M + 3, (B,), generator=g, dtype=torch.int32)
    if c.get("documents"):
        ids = torch.sort(torch.randint(-1, c["documents"], (B, M), generator=g, dtype=torch.int32), 1)[0]
        if c.get("shuffled"):
            ids = ids[:, torch.randperm(M, generator=g)]
        kw["documents"] = (ids[:, M - N:].contiguous() if N <= M else torch.randint(-1, c["documents"], (B, N), generator=g, dtype=torch.int32), ids)
    return kw


def on_gpu(ctx, kw):
    got = {}
    for w, t in kw.items():
        if w == "documents":
            t = tuple(ctx.array(x.cuda()) for x in t)
        elif isinstance(t, torch.Tensor):
            t = ctx.array(t.cuda())
        got[w] = t
    return ctx.scores(**got)


def run_case(ctx, c, q, k, v, dout, kw, results=None):
    """Through the entry points; returns torch tensors."""
    sc = on_gpu(ctx, kw)
    A = ctx.array
    out = torch.empty_like(q) if results is None else results["out"]
    out.fill_(7.0)
    lse = torch.full((c["B"], c["H"], c["N"]), 7.0, device="cuda")
    rest = A(torch.empty_like(q)) if c["dtype"] == BF16 and c["grad"] else None
    gr.attention(A(q), A(k), A(v), sc, out=A(out), lse=A(lse), rest=rest)
    got = dict(out=out, lse=lse)
    if c["grad"]:
        for w, t in (("dq", q), ("dk", k), ("dv", v)):
            got[w] = torch.empty_like(t) if results is None else results[w]
            got[w].fill_(7.0)
        gr.attention_grad(A(dout), A(q), A(k), A(v), sc, A(out), A(lse), rest=rest, dq=A(got["dq"]), dk=A(got["dk"]), dv=A(got["dv"]))
    torch.cuda.synchronize()
    return got


def tensors(c, seed=0):
    by = 3.0 if c.get("cap") else 1.0
    q, k, v, d = (normal(seed + i, c["B"], n, h, c["D"], dtype=c["dtype"], by=f)
                  for i, (n, h, f) in enumerate(((c["N"], c["H"], by), (c["M"], c["HK"], 1.0), (c["M"], c["HK"], 1.0), (c["N"], c["H"], 1.0))))
    return q, k, v, d


CASES = [
    case(1, 1, 1, 1, 1, 64, F32), case(1, 1, 1, 1, 1, 64, BF16),
    case(2, 5, 7, 2, 1, 8, F32), case(2, 5, 7, 2, 1, 8, BF16),
    case(1, 32, 32, 1, 1, 32, BF16, causal=True), case(1, 33, 31, 3, 1, 64, F32),
    case(2, 64, 64, 4, 2, 64, F32, causal=True), case(2, 64, 64, 4, 2, 64, BF16, causal=True),
    case(1, 129, 129, 2, 2, 128, BF16, causal=True), case(1, 129, 129, 2, 2, 128, F32, causal=True),
    case(2, 65, 200, 8, 2, 96, BF16, causal=True, position=135), case(2, 65, 200, 8, 2, 96, F32, causal=True, position=135),
    case(1, 70, 70, 2, 1, 80, F32, causal=True, slopes=True), case(1, 70, 70, 2, 1, 80, BF16, causal=True, slopes=True),
    case(1, 100, 130, 6, 3, 256, BF16, cap=5.0), case(1, 100, 130, 6, 3, 256, F32, cap=5.0),
    case(2, 77, 77, 4, 4, 100, BF16, cap=20.0, causal=True, prefix=True), case(2, 77, 77, 4, 4, 100, F32, cap=20.0, causal=True, prefix=True),
    case(2, 150, 150, 4, 1, 64, BF16, causal=True, documents=4), case(2, 150, 150, 4, 1, 64, F32, documents=3),
    case(1, 90, 260, 2, 1, 128, BF16, documents=5, shuffled=True, causal=True, position=100), case(1, 90, 260, 2, 1, 128, F32, documents=2, shuffled=True),
    case(3, 40, 300, 4, 2, 64, BF16, lengths=True), case(3, 40, 300, 4, 2, 64, F32, lengths=True, cap=10.0, slopes=True, causal=True, position=200),
    case(2, 200, 60, 2, 2, 64, BF16, causal=True, position=-100), case(2, 50, 60, 2, 2, 72, F32, causal=True, position=-30, prefix=True),
    case(1, 3, 1000, 8, 1, 128, BF16, causal=True, position=990, grad=False), case(2, 2, 700, 4, 4, 256, F32, grad=False),
    case(1, 4, 5, 32, 1, 160, BF16, cap=3.0, slopes=True), case(1, 3, 40, 16, 1, 192, F32, cap=3.0, slopes=True, causal=True, position=37),
    case(1, 300, 300, 1, 1, 1, F32), case(1, 50, 50, 2, 1, 3, BF16, causal=True),
    case(1, 600, 600, 16, 2, 64, BF16, causal=True), case(1, 16, 2100, 2, 1, 64, F32, causal=True, position=2084),
    case(1, 64, 64, 2, 2, 64, F32, scale=40.0), case(1, 64, 64, 2, 2, 64, BF16, scale=1e-4),
    case(2, 0, 5, 2, 1, 64, F32), case(2, 5, 0, 2, 1, 64, BF16), case(0, 5, 5, 2, 1, 64, F32),
]


@pytest.mark.gpu
@pytest.mark.parametrize("c", CASES)
def test_against_plain(ctx, c):
    q, k, v, d = tensors(c)
    kw = options(c)
    got = run_case(ctx, c, q, k, v, d, kw)
    ref = plain.attention(q, k, v, d if c["grad"] else None, **kw)
    plain.check(got, ref, c["dtype"], c["D"], c["M"], c["N"], c["H"] // c["HK"], "plain", cap=c.get("cap", 0.0))


LAYOUTS = ["heads_first", "packed", "odd_address", "odd_rows", "backwards", "broadcast"]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_strides(ctx, layout, dtype):
    c = dict(B=2, N=75, M=75, H=4, HK=4, D=64, dtype=dtype, grad=True, causal=True)
    shape = (2, 75, 4, 64)

    def lay(seed, part):
        t = normal(seed, *shape, dtype=dtype)
        if layout == "heads_first":
            r = torch.empty(2, 4, 75, 64, dtype=dtype, device="cuda").transpose(1, 2)
        elif layout == "packed":
            r = packs[part // 3][:, :, part % 3]
        elif layout == "odd_address":
            r = torch.empty(2 * 75 * 256 + 1, dtype=dtype, device="cuda")[1:].view(shape)
        elif layout == "odd_rows":
            r = torch.empty(2, 75, 4, 65, dtype=dtype, device="cuda")[..., :64]
        elif layout == "backwards":
            n = 2 * 75 * 256
            r = None
            base = torch.empty(n, dtype=dtype, device="cuda")
            a = ctx.from_device(base.data_ptr() + base.element_size() * (n - 256), {F32: gr.GR_F32, BF16: gr.GR_BF16}[dtype], shape, (-256, -512, 64, 1), owner=base)
            back = base.view(75, 2, 4, 64).flip(0, 1).transpose(0, 1)   # (a copy: what the view shows)
            return a, back, base
        else:
            r = torch.empty(2, 75, 1, 64, dtype=dtype, device="cuda").expand(shape) if part in (1, 2) else torch.empty(shape, dtype=dtype, device="cuda")
            if part in (1, 2):
                r[:, :, :1].copy_(t[:, :, :1])
                return r
        r.copy_(t)
        return r

    packs = [torch.zeros(2, 75, 3, 4, 64, dtype=dtype, device="cuda") for _ in range(3)]
    kw = options(c)
    if layout == "backwards":
        arrays, shown, bases = [], [], []
        for i in range(8):
            a, _, base = lay(i, i)
            base.copy_(normal(i, base.numel(), dtype=dtype))
            arrays.append(a)
            bases.append(base)
        show = lambda b: b.view(75, 2, 4, 64).flip(0, 1).transpose(0, 1)  # noqa: E731
        q, k, v, d = (show(b).clone() for b in bases[:4])
        sc = on_gpu(ctx, kw)
        lse = ctx.array(torch.empty(2, 4, 75, device="cuda"))
        gr.attention(*arrays[:3], sc, out=arrays[4], lse=lse)
        gr.attention_grad(arrays[3], *arrays[:3], sc, arrays[4], lse, dq=arrays[5], dk=arrays[6], dv=arrays[7])
        torch.cuda.synchronize()
        got = dict(zip(("out", "dq", "dk", "dv"), (show(b) for b in bases[4:])))
    else:
        q, k, v, d = (lay(i, i) for i in range(4))
        res = dict(zip(("out", "dq", "dk", "dv"), (torch.empty_like(d) if layout == "broadcast" else lay(9 + i, (3, 6, 7, 8)[i]) for i in range(4))))
        if layout == "packed":
            res["out"] = torch.empty_like(d)
        got = run_case(ctx, c, q, k, v, d, kw, results=res)
    ref = plain.attention(q, k, v, d, **kw)
    plain.check({w: t for w, t in got.items()}, ref, dtype, 64, 75, 75, 1, layout)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_what_is_not_seen_has_no_say(ctx, dtype):
    """Infinities and NaN behind the lengths, in keys that belong to no document, in masked scores."""
    c = dict(B=2, N=40, M=200, H=4, HK=2, D=64, dtype=dtype, grad=True)
    q, k, v, d = tensors(c)
    lengths = torch.tensor([130, 0], dtype=torch.int32)
    clean = run_case(ctx, c, q, k, v, d, dict(lengths=lengths))
    for t, bad in ((k, math.nan), (v, math.inf)):
        t[0, 130:] = bad
        t[1] = bad
    dirty = run_case(ctx, c, q, k, v, d, dict(lengths=lengths))
    for w in clean:
        assert torch.equal(clean[w], dirty[w]), w
    assert (dirty["out"][1] == 0).all() and (dirty["lse"][1] == -math.inf).all() and (dirty["dk"][0, 130:] == 0).all() and (dirty["dq"][1] == 0).all()
    # a query far to the left of everything: its scores are the type's lowest numbers, not masked ones
    low = run_case(ctx, dict(c, grad=False), (q.float() * 0 + 1e15).to(dtype), (k.float() * 0 - 1e15).nan_to_num(-1e15).to(dtype), torch.ones_like(v), d, {})
    assert torch.isfinite(low["out"]).all() and ((low["out"].float() - 1).abs() < 0.01).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("B,M,H,HK,D,kw", [
    (1, 1, 1, 1, 64, {}), (3, 40, 4, 4, 64, {}), (2, 300, 8, 1, 128, dict(cap=10.0)), (4, 1000, 16, 2, 96, dict(slopes=True)),
    (1, 5000, 32, 1, 64, dict(cap=30.0, slopes=True)), (2, 777, 40, 1, 80, {}), (2, 129, 6, 3, 256, dict(cap=5.0)), (1, 33, 2, 2, 5, {}), (2, 0, 2, 1, 64, {}),
])
def test_single_tokens(ctx, B, M, H, HK, D, kw, dtype):
    q, k, v = normal(1, B, H, D, dtype=dtype, by=2.0), normal(2, B, M, HK, D, dtype=dtype), normal(3, B, M, HK, D, dtype=dtype)
    g = torch.Generator().manual_seed(5)
    kw = dict(kw, lengths=torch.randint(0, M + 1, (B,), generator=g, dtype=torch.int32))
    kw["lengths"][0] = M
    if kw.pop("slopes", None):
        kw["slopes"] = torch.tensor([2.0 ** -(1 + i % 9) for i in range(H)])
    for b in range(B):
        k[b, int(kw["lengths"][b]):] = math.nan
        v[b, int(kw["lengths"][b]):] = math.nan
    out = torch.full_like(q, 7.0)
    gr.attention_step(ctx.array(q), ctx.array(k), ctx.array(v), on_gpu(ctx, kw), out=ctx.array(out))
    torch.cuda.synchronize()
    ref = plain.attention(q[:, None], k.nan_to_num(0.0), v.nan_to_num(0.0), step=True, **kw)
    plain.check(dict(out=out[:, None]), ref, dtype, D, M, 1, H // HK, "step", cap=kw.get("cap", 0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,N,H,D,part", [(1, 1, 1, 64, 64), (2, 33, 3, 80, 32), (1, 7, 2, 5, 4), (3, 100, 32, 128, 128), (2, 9, 1, 256, 256), (1, 5, 4, 96, 90), (1, 3, 2, 8, 0)])
def test_rotary(ctx, B, N, H, D, part, interleaved, dtype):
    x = normal(1, B, N, H, D, dtype=dtype)
    f = gr.rotary_frequencies(part)
    g = torch.Generator().manual_seed(2)
    pos = torch.randint(-5, 2_000_000_000, (B, N), generator=g, dtype=torch.int32)
    for inverse, factor in ((False, 1.0), (True, 1.25)):
        ref = plain.rotary(x, f, pos.numpy(), interleaved, inverse, factor)
        # two products, each of a sine off by half a step and a few of the polynomial's roundings; angles: positions below 2^31 in 64 bits leave 2e-7 of a turn's last place
        size = plain.rotary(x.abs(), [0.0] * (part // 2), pos.numpy())
        bar = plain.HALF[dtype] * ref.abs() + (6 * 2.0 ** -24 + 1e-6) * factor * 2 * size.amax(-1, keepdim=True)
        y = gr.rotary(ctx.array(x), f, ctx.array(pos.cuda()), interleaved, inverse, factor).torch().cpu().double()
        assert ((y - ref).abs() <= bar).all(), float(((y - ref).abs() / bar).max())
        z = x.clone()
        gr.rotary(ctx.array(z), f, ctx.array(pos.cuda()), interleaved, inverse, factor, out=ctx.array(z))   # in place
        assert torch.equal(z.cpu().double(), y)
    # small positions: right to a few roundings
    ref = plain.rotary(x, f, torch.arange(N).numpy()[None] + 3, interleaved)
    y = gr.rotary(ctx.array(x), f, 3, interleaved).torch().cpu().double()
    assert ((y - ref).abs() <= plain.HALF[dtype] * ref.abs() + 8 * 2.0 ** -24 * x.abs().amax().item()).all()
    # strided, unaligned, into a strided place
    wide = torch.empty(B, H, N, D + 3, dtype=dtype, device="cuda")
    src, dst = wide[..., 1:D + 1].transpose(1, 2), torch.zeros(B, N, H, 2 * D + 1, dtype=dtype, device="cuda")
    src.copy_(x)
    gr.rotary(ctx.array(src), f, 3, interleaved, out=ctx.array(dst[..., D:2 * D]))
    assert torch.equal(dst[..., D:2 * D].cpu().double(), y) and (dst[..., :D] == 0).all() and (dst[..., 2 * D:] == 0).all()


@pytest.mark.gpu
def test_gradient_against_differences(ctx):
    """dq, dk, dv of the kernels against differences of the kernels' own output: f32, one direction at a time."""
    c = dict(B=1, N=40, M=40, H=4, HK=2, D=64, dtype=F32, grad=True, cap=4.0, causal=True, slopes=True)
    q, k, v, d = tensors(c)
    kw = options(c)
    got = run_case(ctx, c, q, k, v, d, kw)
    fwd = dict(c, grad=False)
    for name, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        ts = [q, k, v]
        e = normal(50 + i, *ts[i].shape)
        h = 2.0 ** -6
        up, dn = list(ts), list(ts)
        up[i], dn[i] = ts[i] + h * e, ts[i] - h * e
        slope = ((run_case(ctx, fwd, *up, d, kw)["out"].double() - run_case(ctx, fwd, *dn, d, kw)["out"].double()) * d.double()).sum() / (2 * h)
        # the difference is off by h^2 / 6 of a third derivative and 2^-24 / h of the output's size
        want = (got[name].double() * e.double()).sum()
        size = (got[name].double().norm() * e.double().norm())
        assert abs(float(slope - want)) <= 2e-3 * float(size) + 1e-2, (name, float(slope), float(want))


@pytest.mark.gpu
def test_same_bits_every_time(ctx):
    c = dict(B=1, N=500, M=900, H=8, HK=1, D=64, dtype=BF16, grad=True, causal=True, position=400)
    q, k, v, d = tensors(c)
    first = run_case(ctx, c, q, k, v, d, options(c))
    for _ in range(3):
        again = run_case(ctx, c, q, k, v, d, options(c))
        for w in first:
            assert torch.equal(first[w], again[w]), w


@pytest.mark.gpu
def test_lazy_operands_and_pending_readers(ctx):
    """Operands that are still expressions are evaluated; what was recorded over a result's storage keeps the old values."""
    x = normal(1, 24, 32)
    w = [normal(2 + i, 32, 64) for i in range(3)]
    lx = ctx.array(x)
    q, k, v = (gr.reshape(gr.dot(lx, ctx.array(t)) * 0.5, (1, 24, 4, 16)) for t in w)
    out = torch.full((1, 24, 4, 16), 3.0, device="cuda")
    lo = ctx.array(out)
    pending = lo * 2.0
    o, lse = gr.attention(q, k, v, ctx.scores(causal=True), out=lo)
    after = lo + 1.0
    ref = plain.attention(*((x @ t * 0.5).view(1, 24, 4, 16) for t in w), causal=True)
    assert (pending.torch() == 6.0).all()
    assert (after.torch().cpu().double() - 1.0 - ref["out"]).abs().max() < 1e-4
    assert (lse.torch().cpu().double() - ref["lse"]).abs().max() < 1e-4
    assert o is lo


@pytest.mark.gpu
def test_graph_replays(ctx):
    """Forward, gradient and a step captured together and replayed on new data, with eager work in between."""
    stream = torch.cuda.Stream()
    c2 = gr.Context(stream=stream.cuda_stream)
    c = dict(B=1, N=100, M=100, H=4, HK=1, D=64, dtype=BF16, grad=True, causal=True)
    with torch.cuda.stream(stream):
        q, k, v, d = tensors(c)
        docs = torch.arange(100, device="cuda", dtype=torch.int32)[None] // 40
        lens = torch.tensor([70], device="cuda", dtype=torch.int32)
        res = dict(out=torch.empty_like(q), rest=torch.empty_like(q), lse=torch.empty(1, 4, 100, device="cuda"), dq=torch.empty_like(q), dk=torch.empty_like(k),
                   dv=torch.empty_like(v), tok=torch.empty(1, 4, 64, dtype=BF16, device="cuda"))

        def go(r):
            A = c2.array
            sc = c2.scores(causal=True, documents=A(docs))
            gr.attention(A(q), A(k), A(v), sc, out=A(r["out"]), lse=A(r["lse"]), rest=A(r["rest"]))
            gr.attention_grad(A(d), A(q), A(k), A(v), sc, A(r["out"]), A(r["lse"]), rest=A(r["rest"]), dq=A(r["dq"]), dk=A(r["dk"]), dv=A(r["dv"]))
            gr.attention_step(A(q[:, 5]), A(k), A(v), c2.scores(lengths=A(lens)), out=A(r["tok"]))

        go(res)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            go(res)
        for rep in range(3):
            for t, s in ((q, 1), (k, 2), (v, 3), (d, 4)):
                t.copy_(normal(100 * rep + s, *t.shape, dtype=BF16))
            eager = {w: torch.empty_like(t) for w, t in res.items()}
            for t in res.values():
                t.zero_()
            graph.replay()
            stream.synchronize()
            go(eager)
            stream.synchronize()
            for w in res:
                assert torch.equal(res[w], eager[w]), (rep, w)
    # a call that would have to allocate during a capture says so
    c3 = gr.Context(stream=stream.cuda_stream)
    with torch.cuda.stream(stream):
        one = [normal(7, 1, 4, 1, 64, dtype=BF16), normal(8, 1, 6000, 1, 64, dtype=BF16), torch.empty(1, 4, 1, 64, dtype=BF16, device="cuda")]
        graph2 = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph2, stream=stream):
            refused("GR_ERR_OOM", gr.attention, c3.array(one[0]), c3.array(one[1]), c3.array(one[1]), c3.scores(), out=c3.array(one[2]), lse=False)
            one[2].zero_()
    c3.close()
    del graph, graph2
    c2.close()


@pytest.mark.gpu
def test_far_offsets(ctx):
    """Rows behind 2^32 elements of a buffer, and rows whose steps are too long for the fast loads."""
    step = (1 << 31) // 64 + 64            # elements between rows: 64 rows pass 2^31, 129 pass 2^32
    k = torch.zeros(130 * step, dtype=BF16, device="cuda")
    v = torch.zeros(130 * step, dtype=BF16, device="cuda")
    kv = normal(1, 2, 130, 64, dtype=BF16)
    for i, t in enumerate((k, v)):
        t.as_strided((130, 64), (step, 1)).copy_(kv[i])
    q = normal(2, 1, 4, 2, 64, dtype=BF16)
    for shape, strides in (((1, 130, 1, 64), (0, step, 0, 1)), ((130, 1, 1, 64), (step, 0, 0, 1))):
        B = shape[0]
        lk, lv = (ctx.from_device(t.data_ptr(), gr.GR_BF16, shape, strides, owner=t) for t in (k, v))
        qb = q.expand(B, 4, 2, 64).contiguous()
        out = torch.empty_like(qb)
        gr.attention(ctx.array(qb), lk, lv, ctx.scores(), out=ctx.array(out), lse=False)
        ref = plain.attention(qb, kv[0].view(shape), kv[1].view(shape))
        plain.check(dict(out=out), ref, BF16, 64, shape[1], 4, 2, "far")


@pytest.mark.gpu
def test_layer_trains_and_generates():
    """The example layer against the same layer in binary64 torch with automatic differentiation."""
    from paper_1901_03771_amd import attention_layer as al
    c = gr.Context()
    layer = al.AttentionLayer(c, width=48, heads=4, shared=2, values=24, cap=8.0, seed=4)
    ids, places = al.packed_documents(2, 70, "cuda", seed=5)
    g = torch.Generator().manual_seed(6)
    x, target = torch.randn(2, 70, 48, generator=g).cuda(), torch.randn(2, 70, 48, generator=g).cuda()
    w = {n: t.cpu().double().requires_grad_() for n, t in layer.weights.items()}

    def turned(t):
        a = places.cpu().double()[..., None, None] * torch.tensor(list(layer.frequencies), dtype=torch.float64)
        lo, hi = t[..., :12], t[..., 12:]
        return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)

    xd = x.cpu().double()
    q, k, v = turned((xd @ w["q"]).view(2, 70, 4, 24)), turned((xd @ w["k"]).view(2, 70, 2, 24)), (xd @ w["v"]).view(2, 70, 2, 24)
    k, v = k.repeat_interleave(2, 2), v.repeat_interleave(2, 2)
    s = torch.einsum("bihd,bjhd->bhij", q, k) * 24 ** -0.5
    s = 8.0 * torch.tanh(s / 8.0)
    d = ids.cpu()
    see = (torch.arange(70)[:, None] >= torch.arange(70)) & (d[:, :, None] == d[:, None, :])
    p = torch.softmax(s.masked_fill(~see[:, None], -math.inf), -1)
    y = torch.einsum("bhij,bjhd->bihd", p, v).reshape(2, 70, 96) @ w["o"]
    loss = ((y - target.cpu().double()) ** 2).mean()
    loss.backward()
    before = {n: t.cpu().double() for n, t in layer.weights.items()}
    got = layer.train_step(x, target, c.array(places), c.array(ids), rate=1.0)
    # sums of up to 140 rows or 96 values in a handful of products one after another: each is off by at most (rows + values) 2^-24 of its terms' sizes,
    # which are below 16 times the result's norm here
    bar = 6 * (140 + 96) * 2.0 ** -24 * 16
    assert abs(got - loss.item()) <= bar * loss.item()
    for n, t in layer.weights.items():
        step = before[n] - t.cpu().double()
        assert (step - w[n].grad).norm() <= bar * w[n].grad.norm() + 2.0 ** -24 * before[n].norm(), n
    # generation: the same rows as a forward pass over one sequence, with a cache that holds NaN where nothing was written
    one = x[:, :20].contiguous()
    whole = layer.forward(one, 0, None)[0].torch().view(2, 20, 48)
    cache = [torch.full((2, 30, 2, 24), math.nan, device="cuda") for _ in range(2)]
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    for i in range(20):
        y1 = layer.step(one[:, i].contiguous(), *cache, lengths)
        assert (y1 - whole[:, i]).norm() <= bar * whole[:, i].norm(), i
    c.close()


def test_random_calls_are_refused_or_run(dry):
    """Random, mostly invalid arguments: every call answers with a status, and what is refused launches nothing."""
    import random
    r = random.Random(11)
    L, P = gr.lib(), dry._p
    s = Specs(dry)

    def tensor(rank=None):
        rank = r.choice([3, 4, 4, 4, 2, 1]) if rank is None else rank
        shape = [r.choice([0, 1, 2, 2, 2, 4, 64, 300]) for _ in range(rank)]
        shape[-1] = r.choice([0, 1, 8, 64, 64, 100, 256, 257])
        strides = None
        if r.random() < 0.3:
            strides = [r.choice([0, 1, -64, 64, 4096, 1 << 31]) for _ in range(rank)]
            if r.random() < 0.7:
                strides[-1] = 1
        return s(shape, r.choice([gr.GR_F32, gr.GR_F32, gr.GR_BF16, gr.GR_I32]), strides)

    whole = [s((2, 2, 2, 64), d) for d in (gr.GR_F32, gr.GR_BF16) for _ in range(8)]
    pool = [tensor() for _ in range(60)] + whole + \
        [s((2, 2, 2)) for _ in range(3)] + [s((2,), gr.GR_I32), s((2, 2), gr.GR_I32), s((2,)), s((2, 2, 2, 64)) + 1.0, dry.scalar(3.0)]
    whole = [a.h for a in whole[:8]]
    h = lambda: r.choice([0, 1 << 50] + [a.h for a in pool] * 4)  # noqa: E731
    fine = lambda x: x if r.random() < 0.9 else r.choice([math.nan, math.inf, -1.0, 0.0, 1e300])  # noqa: E731
    f = (ctypes.c_double * 300)(*[r.choice([0.0, 1.0, 1e300]) for _ in range(300)])
    codes = set()
    for _ in range(6000):
        sc = gr._Scores(fine(0.5), fine(r.choice([0.0, 30.0])), r.choice([0, 0, h()]), r.choice([0, 1, 1, 7]), r.choice([0, 5, -(1 << 40)]),
                        r.choice([0, 0, 0, h()]), r.choice([0, 0, 0, h()]), r.choice([0, 0, 0, h()]), r.choice([0, 0, h()]))
        ref = ctypes.byref(sc) if r.random() < 0.98 else None
        before = dry.stats()["kernel_launches"]
        k = r.randrange(4)
        g = (lambda: r.choice(whole)) if r.random() < 0.5 else h
        if k == 0:
            st = L.gr_attention(P, ref, g(), g(), g(), g(), r.choice([0, h()]), r.choice([0, 0, h()]))
        elif k == 1:
            st = L.gr_attention_grad(P, ref, g(), g(), g(), g(), r.choice([0, 0, h()]), h(), g(), g(), g(), g())
        elif k == 2:
            st = L.gr_attention_step(P, ref, h(), g(), g(), h())
        else:
            st = L.gr_rotary(P, g(), r.choice([0, h()]), r.choice([0, 7, 1 << 50]), f if r.random() < 0.95 else None, r.choice([-1, 0, 4, 32, 128, 257]), r.choice([0, 1, 5]),
                             r.choice([0, 1]), fine(1.0), g())
        assert 0 <= st <= 11
        codes.add(st)
        assert st == 0 or dry.stats()["kernel_launches"] == before or st == 9
    assert {0, 1, 2, 3, 5, 6, 10} <= codes, codes


@pytest.mark.gpu
@pytest.mark.parametrize("N,M", [(40, 17003), (17003, 40)])
def test_documents_far_apart(ctx, N, M):
    """Documents whose pieces lie more than 256 tiles apart, in heads enough that no split shortens the walk; the heads share their inputs."""
    H = 256
    g = torch.Generator().manual_seed(9)
    q, k, v, d = (normal(70 + i, 1, n, 1, 64, dtype=BF16) for i, n in enumerate((N, M, M, N)))
    qd, kd = torch.full((1, N), 3, dtype=torch.int32), torch.full((1, M), 3, dtype=torch.int32)
    long, n = (kd, M) if M > N else (qd, N)
    long[:] = torch.randint(10, 20, (1, n), generator=g, dtype=torch.int32)
    long[0, 50:70] = 3
    long[0, 16500:16510] = 3
    long[0, -1] = 3
    wide = lambda t: t.expand(t.shape[0], t.shape[1], H, 64)  # noqa: E731
    sc = ctx.scores(documents=(ctx.array(qd.cuda()), ctx.array(kd.cuda())))
    A = ctx.array
    out, rest = (torch.empty(1, N, H, 64, dtype=BF16, device="cuda") for _ in range(2))
    lse = torch.empty(1, H, N, device="cuda")
    dq, dk, dv = (torch.empty(1, m, H, 64, dtype=BF16, device="cuda") for m in (N, M, M))
    gr.attention(A(wide(q)), A(wide(k)), A(wide(v)), sc, out=A(out), lse=A(lse), rest=A(rest))
    gr.attention_grad(A(wide(d)), A(wide(q)), A(wide(k)), A(wide(v)), sc, A(out), A(lse), rest=A(rest), dq=A(dq), dk=A(dk), dv=A(dv))
    torch.cuda.synchronize()
    ref = plain.attention(q, k, v, d, documents=(qd, kd))
    for h in (0, 100, 255):
        got = dict(out=out[:, :, h:h + 1], lse=lse[:, h:h + 1], dq=dq[:, :, h:h + 1], dk=dk[:, :, h:h + 1], dv=dv[:, :, h:h + 1])
        plain.check(got, ref, BF16, 64, M, N, 1, f"head {h}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_strided_masks_and_no_rest(ctx, dtype):
    """Masks, lengths, slopes and positions with steps of their own, and a gradient without what out lost in rounding."""
    B, N, H, HK, D = 2, 130, 4, 2, 64
    c = dict(B=B, N=N, M=N, H=H, HK=HK, D=D, dtype=dtype)
    q, k, v, d = tensors(c)
    g = torch.Generator().manual_seed(21)
    ids = torch.sort(torch.randint(0, 3, (B, N), generator=g, dtype=torch.int32), 1)[0]
    lengths, prefix = torch.tensor([100, 130], dtype=torch.int32), torch.tensor([7, 50], dtype=torch.int32)
    slopes = torch.tensor([0.5, 0.25, 0.0, -0.01])

    def spread(t, steps):
        big = torch.zeros([n * s for n, s in zip(t.shape, steps)], dtype=t.dtype, device="cuda")
        view = big[tuple(slice(None, None, s) for s in steps)]
        view.copy_(t)
        return ctx.array(view)

    sc = ctx.scores(causal=True, prefix=spread(prefix, (3,)), lengths=spread(lengths, (2,)), slopes=spread(slopes, (5,)), documents=spread(ids, (1, 3)))
    A = ctx.array
    out, lse = gr.attention(A(q), A(k), A(v), sc)
    dq, dk, dv = gr.attention_grad(A(d), A(q), A(k), A(v), sc, out, lse)
    ref = plain.attention(q, k, v, d, causal=True, prefix=prefix, lengths=lengths, slopes=slopes, documents=ids)
    got = dict(out=out.torch(), lse=lse.torch(), dq=dq.torch(), dk=dk.torch(), dv=dv.torch())
    plain.check(got, ref, dtype, D, N, N, H // HK, "strided masks")
    # positions transposed, and rotary through them
    pos = torch.randint(0, 5000, (N, B), generator=g, dtype=torch.int32).cuda().T
    f = gr.rotary_frequencies(D)
    y = gr.rotary(A(q), f, A(pos)).torch().cpu().double()
    want = plain.rotary(q, f, pos.cpu().numpy())
    assert ((y - want).abs() <= plain.HALF[dtype] * want.abs() + 1e-5 * q.abs().max().item()).all()


@pytest.mark.gpu
def test_many_rows_against_plain(ctx):
    """A long row whose walks have many tiles, heads shared and not, every option at once."""
    for dtype, D, H, HK in ((BF16, 128, 4, 2), (F32, 64, 2, 2)):
        c = dict(B=1, N=2500, M=2500, H=H, HK=HK, D=D, dtype=dtype, grad=True, cap=15.0, causal=True, slopes=True, prefix=True, documents=3)
        q, k, v, d = tensors(c)
        kw = options(c)
        got = run_case(ctx, c, q, k, v, d, kw)
        ref = plain.attention(q, k, v, d, **kw)
        plain.check(got, ref, dtype, D, 2500, 2500, H // HK, f"{D}", cap=15.0)


@pytest.mark.gpu
def test_new_results_belong_to_the_stream_of_the_context():
    """A context on a stream of its own, called while torch's is another: the memory of its results is not what torch's stream still works on."""
    x = normal(5, 2, 64, 4, 64)
    torch.cuda.synchronize()
    f = gr.rotary_frequencies(64)
    side = torch.cuda.Stream()
    for ours, theirs in ((side, torch.cuda.default_stream()), (torch.cuda.default_stream(), side)):
        with torch.cuda.stream(ours):
            c = gr.Context()
        with torch.cuda.stream(theirs):
            big = torch.ones(4096, 4096, device="cuda")
            old = torch.empty_like(x)
            at = old.data_ptr()
            for _ in range(20):
                big = big @ big * 2.0 ** -12
            old.fill_(9.0)   # still queued when the memory goes back to torch
            del old
            y = gr.rotary(c.array(x), f, 3)
            q = c.array(x)
            out, lse = gr.attention(q, q, q, c.scores())
            assert at not in (y.data_ptr()[0], out.data_ptr()[0])   # (torch() would copy, into memory of its own)
        torch.cuda.synchronize()
        ref = plain.rotary(x, f, torch.arange(64).numpy()[None] + 3)
        assert ((y.torch().cpu().double() - ref).abs() <= plain.HALF[F32] * ref.abs() + 8 * 2.0 ** -24 * x.abs().amax().item()).all()
        plain.check(dict(out=out.torch(), lse=lse.torch()), plain.attention(x, x, x), F32, 64, 64, 64, 1, "stream")
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_masked_scores_are_replaced(ctx, dtype, bad):
    """Keys that are not numbers where documents, causal order and capped or plain scores leave them unseen."""
    c = dict(B=1, N=96, M=96, H=4, HK=2, D=64, dtype=dtype, grad=False)
    q, k, v, d = tensors(c)
    ids = torch.zeros(1, 96, dtype=torch.int32)
    ids[0, 20:50] = -1
    late = torch.tensor([90], dtype=torch.int32)
    for kw in (dict(documents=(torch.zeros(1, 96, dtype=torch.int32), ids)), dict(documents=(torch.zeros(1, 96, dtype=torch.int32), ids), cap=10.0),
               dict(causal=True, position=-10), dict(causal=True, position=-10, cap=10.0, prefix=late - 10)):
        clean = run_case(ctx, c, q, k, v, d, kw)
        dirty = k.clone()
        if "documents" in kw:
            dirty[0, 20:50] = bad
        else:
            dirty[0, 86:] = bad
        got = run_case(ctx, c, q, dirty, v, d, kw)
        for w in clean:
            assert torch.equal(clean[w], got[w]), (kw, w)


# rows of queries, keys, heads, heads of k: calls of one part, of 2 to 16, of more, with a join of waves and without
PARTS = [(40, 40, 4, 2), (40, 500, 4, 2), (3, 90, 2, 2), (3, 1500, 64, 8), (3, 6000, 2, 1), (150, 6000, 2, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("N,M,H,HK", PARTS)
def test_nan_that_is_seen_stays(ctx, N, M, H, HK, dtype):
    """A query, a key or a stretch of keys that is not a number: NaN in out and lse of the rows that see it, the same bits as before in all others,
    however many parts the keys are divided into."""
    D = 64
    c = dict(B=2, N=N, M=M, H=H, HK=HK, D=D, dtype=dtype, grad=False)
    q, k, v, d = tensors(c)
    kw = dict(causal=True, position=M - N)
    clean = run_case(ctx, c, q, k, v, d, kw)
    assert torch.isfinite(clean["out"]).all() and torch.isfinite(clean["lse"]).all()
    G = H // HK

    def check(got, hit, what):   # hit (B, N, H): rows that have to be NaN
        assert torch.isnan(got["out"][hit]).all() and torch.isnan(got["lse"].transpose(1, 2)[hit]).all(), what
        assert torch.equal(got["out"][~hit], clean["out"][~hit]), what
        assert torch.equal(got["lse"].transpose(1, 2)[~hit], clean["lse"].transpose(1, 2)[~hit]), what

    for bad in (math.nan, math.inf):
        t = q.clone()
        t[1, N - 2, 1, 5] = bad
        hit = torch.zeros(2, N, H, dtype=torch.bool, device="cuda")
        hit[1, N - 2, 1] = True
        check(run_case(ctx, c, t, k, v, d, kw), hit, f"query {bad}")
    place = torch.arange(N, device="cuda") + M - N
    for first, last in ((M - 2, M - 1), (0, 1), (M // 2, M - N)):   # a late key, the first one, and a stretch that fills whole parts
        if first >= last:
            continue
        t = k.clone()
        t[0, first:last, HK - 1] = math.nan
        hit = torch.zeros(2, N, H, dtype=torch.bool, device="cuda")
        hit[0, :, (HK - 1) * G:] = (place >= first)[:, None]
        check(run_case(ctx, c, q, t, v, d, kw), hit, f"keys {first} .. {last}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("M", [40, 700, 40000])
def test_nan_in_single_tokens_stays(ctx, M, dtype):
    q, k, v = normal(1, 2, 4, 64, dtype=dtype), normal(2, 2, M, 1, 64, dtype=dtype), normal(3, 2, M, 1, 64, dtype=dtype)
    lengths = torch.tensor([M, M - 3], dtype=torch.int32)

    def step(q, k):
        out = torch.full_like(q, 7.0)
        gr.attention_step(ctx.array(q), ctx.array(k), ctx.array(v), on_gpu(ctx, dict(lengths=lengths)), out=ctx.array(out))
        return out

    clean = step(q, k)
    assert torch.isfinite(clean).all()
    t = q.clone()
    t[1, 2, 9] = math.nan
    got = step(t, k)
    assert torch.isnan(got[1, 2]).all()
    got[1, 2] = clean[1, 2]
    assert torch.equal(got, clean)
    t = k.clone()
    t[0, M // 3:M // 2] = math.nan
    got = step(q, t)
    assert torch.isnan(got[0]).all() and torch.equal(got[1], clean[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
def test_gradient_of_a_nan_row(ctx, dtype):
    """The rows and keys that a NaN query reaches are NaN in the gradient, the others are as they were; queries split and not."""
    for N, M, H in ((40, 40, 2), (40, 2500, 1)):
        c = dict(B=2, N=N, M=M, H=H, HK=H, D=64, dtype=dtype, grad=True)
        q, k, v, d = tensors(c)
        clean = run_case(ctx, c, q, k, v, d, {})
        q[1, 7, 0] = math.nan
        got = run_case(ctx, c, q, k, v, d, {})
        assert torch.isnan(got["dq"][1, 7, 0]).all() and torch.isnan(got["dk"][1, :, 0]).all() and torch.isnan(got["dv"][1, :, 0]).all()
        for w in ("dq", "dk", "dv"):
            assert torch.equal(got[w][0], clean[w][0]), w
            assert torch.equal(got[w][1, :, 1:], clean[w][1, :, 1:]), w
        keep = torch.arange(N) != 7
        assert torch.equal(got["dq"][1][keep], clean["dq"][1][keep])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("cap", [1e3, 1024.0, 1025.0, 1e5, 1e7, 1e20])
@pytest.mark.parametrize("N,M,H,HK,slopes", [(70, 200, 4, 2, False), (5, 900, 4, 2, True), (33, 70, 2, 2, True)])
def test_caps_far_above_the_scores(ctx, N, M, H, HK, slopes, cap, dtype):
    """A large cap leaves scores as they are: no error of the tanh is to be multiplied by it.  The score itself may be off by 2^-12 (a sixteenth of what rounding a
    probability to bfloat16 may do) in bfloat16, whatever the cap, and by nothing but its own roundings in float32."""
    c = dict(B=1, N=N, M=M, H=H, HK=HK, D=64, dtype=dtype, grad=True, cap=cap, slopes=slopes, causal=True, position=M - N)
    q, k, v, d = tensors(c)
    kw = options(c)
    got = run_case(ctx, c, q, k, v, d, kw)
    ref = plain.attention(q, k, v, d, **kw)
    lse, low = got.pop("lse").cpu().double(), 2.0 ** -12 if dtype == BF16 else 0.0
    off = (64 + 10) * 2.0 ** -24 * float(ref["score"].max())
    bar = off + low + (M + 16) * 2.0 ** -24 + 4 * 2.0 ** -24 * ref["lse"].abs()
    assert ((lse - ref["lse"]).abs() <= bar).all(), float((lse - ref["lse"]).abs().max())
    plain.check(got, ref, dtype, 64, M, N, H // HK, f"cap {cap}")


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [500.0, 1e4, 1e7])
def test_single_tokens_with_large_caps(ctx, cap):
    q, k, v = normal(1, 2, 8, 128, dtype=BF16, by=2.0), normal(2, 2, 1000, 2, 128, dtype=BF16), normal(3, 2, 1000, 2, 128, dtype=BF16)
    kw = dict(cap=cap, lengths=torch.tensor([1000, 333], dtype=torch.int32))
    out = torch.full_like(q, 7.0)
    gr.attention_step(ctx.array(q), ctx.array(k), ctx.array(v), on_gpu(ctx, kw), out=ctx.array(out))
    plain.check(dict(out=out[:, None]), plain.attention(q[:, None], k, v, step=True, **kw), BF16, 128, 1000, 1, 4, "step")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("kw", [dict(scale=1e-27), dict(scale=1e25), dict(scale=1e25, cap=1e-8), dict(scale=1e-7, cap=9e29), dict(cap=1e-25)])
def test_scales_and_caps_at_the_ends(ctx, kw, dtype):
    """Scores of one sign of zero, of a cap's size, or so far apart that one key has all: nothing but numbers, and masked keys have no say."""
    c = dict(B=1, N=70, M=70, H=2, HK=1, D=64, dtype=dtype, grad=True, causal=True)
    q, k, v, d = tensors(c)
    got = run_case(ctx, c, q, k, v, d, dict(kw, causal=True))
    for w, t in got.items():
        assert torch.isfinite(t).all(), w
    # the first query sees the first key alone
    assert torch.equal(got["out"][:, 0], v[:, 0].expand(1, 2, 64))
    if kw.get("cap", 1.0) < 1e-20 or kw.get("scale", 1.0) < 1e-20:   # all scores as good as zero: means of v
        mean = v.double().cumsum(1) / torch.arange(1, 71, device="cuda").view(1, 70, 1, 1)
        assert ((got["out"].double() - mean).abs() <= 2 * plain.HALF[dtype] * v.double().abs().cumsum(1) / torch.arange(1, 71, device="cuda").view(1, 70, 1, 1) + 1e-5).all()


@pytest.mark.gpu
def test_the_largest_floats(ctx):
    """float32 values up to 2^128 - 2^119 are numbers, seen and unseen; those beyond count as infinite."""
    c = dict(B=1, N=40, M=40, H=2, HK=1, D=64, dtype=F32, grad=False, causal=True)
    q, k, v, d = tensors(c)
    most = 2.0 ** 128 - 2.0 ** 119 - 2.0 ** 104   # the last float below
    clean = run_case(ctx, c, q, k, v, d, options(c))
    last = v.clone()
    last[0, 39] = -most                            # seen by the last query alone
    got = run_case(ctx, c, q, k, last, d, options(c))
    assert torch.equal(got["out"][:, :39], clean["out"][:, :39])
    plain.check(got, plain.attention(q, k, last, causal=True), F32, 64, 40, 40, 2, "largest")
    last[0, 39, :, 3] = 2.0 ** 128 - 2.0 ** 119
    got = run_case(ctx, c, q, k, last, d, options(c))
    assert torch.isnan(got["out"][0, 39, :, 3]).all() and torch.equal(got["lse"], clean["lse"])


@pytest.mark.gpu
@pytest.mark.parametrize("slopes", [False, True])
def test_probabilities_of_the_float32_gradient(ctx, slopes):
    """Every query sees one key, at a score of exactly zero, under an lse that the test gives: dv, dq and dk are single products with p = exp(-lse).  Roundings of
    p, in units of 2^-24: lse in binary logarithms 0.7, a power of two of half the exponent, off by a unit in the last place at most, taken twice 4, two
    products 1 each; of the result: two products more.  In the mean, a rounding of e at most being e / sqrt(3): sqrt(0.5 + 16 + 4) / sqrt(3) = 2.6, and the bar is 4, that is
    2^-22.  An exponent rounded as a number near 32 would be off by 16 ln 2 / sqrt(3) = 6.4."""
    N, D = 512, 64
    g = torch.Generator().manual_seed(31)
    q, k, v = torch.zeros(3, 1, N, 1, D).unbind(0)
    q[..., :32], k[..., 32:], v[..., 0] = torch.randn(1, N, 1, 32, generator=g), torch.randn(1, N, 1, 32, generator=g), 1.0
    do, lse = torch.randn(1, N, 1, D, generator=g), torch.rand(1, 1, N, generator=g) * 0.5 + 0.5
    ids = torch.arange(N, dtype=torch.int32)[None]
    A = lambda t: ctx.array(t.cuda())  # noqa: E731
    sc = ctx.scores(scale=1.0, documents=A(ids), slopes=A(torch.tensor([3.0])) if slopes else None)   # (a key at the query's own place)
    got = gr.attention_grad(A(do), A(q), A(k), A(v), sc, A(torch.zeros_like(q)), A(lse))
    p = torch.exp(-lse.double())[0, 0].view(1, N, 1, 1)
    ds = p * do.double()[..., :1]
    for name, x, want in zip(("dq", "dk", "dv"), got, (ds * k.double(), ds * q.double(), p * do.double())):
        x = x.torch().cpu().double()
        some = want != 0
        assert (x[~some] == 0).all(), name
        off = x[some] / want[some] - 1
        assert off.square().mean().sqrt() <= 2.0 ** -22, (name, float(off.square().mean().sqrt()))


@pytest.mark.gpu
@pytest.mark.parametrize("B,M,H,HK,D,kw", [(4, 500, 16, 16, 64, {}), (2, 3000, 8, 2, 128, dict(cap=30.0)), (1, 6000, 8, 1, 96, {}), (2, 700, 4, 2, 256, {})])
def test_single_tokens_are_as_near_as_bfloat16_is(ctx, B, M, H, HK, D, kw):
    """A step's result is as far from binary64, in norm, as its own rounding to bfloat16, and a tenth more: probabilities of 16 bits leave 2^-17 of the
    sizes of the terms, up to 30 times those of the results here, whose square is a fiftieth of the rounding's."""
    q, k, v = normal(61, B, H, D, dtype=BF16), normal(62, B, M, HK, D, dtype=BF16), normal(63, B, M, HK, D, dtype=BF16)
    kw = dict(kw, lengths=torch.full((B,), M, dtype=torch.int32))
    out = torch.empty_like(q)
    gr.attention_step(ctx.array(q), ctx.array(k), ctx.array(v), on_gpu(ctx, kw), out=ctx.array(out))
    ref = plain.attention(q[:, None], k, v, step=True, **kw)["out"][:, 0]
    rounding = (ref.to(BF16).double() - ref).norm()
    off = (out.cpu().double() - ref).norm()
    assert off <= 1.1 * rounding, float(off / rounding)
