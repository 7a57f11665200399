"""Gated feed-forward step and its backward pass against the formulas in 64 bits.

Bounds before the output's own rounding (u: half a step of the type, U = 2^-24): the tensor cores add exact products
into fp32 accumulators, at worst truncating each of K / 16 partial sums and the final few (2^-23 each): a projection is off by
(K / 16 + 8) 2^-23 of the sum of magnitudes.  SiLU and the logistic function add 2^-20 of their values.  dG and
dV are rounded to the type once (u of each, 2^-25 absolute below fp16's normal range) before they are multiplied
into dx and dw, whose bounds sum those errors over the products' magnitudes.  That worst case is loose where signs mix, so
the relative L2 error is held too: one rounding of each operand's and of the output's elements, independent and at most u
each, is below 1.2 u in the mean square (each is u / sqrt(3) or less), with K 2^-23-sized sums far below."""
import pytest
import torch

from block_testutil import TORCH_DT, assert_close, guarded, half_step, rel_l2
from paper_2609_26590_gb300 import build as gbuild
from paper_2609_26590_gb300 import gla

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    gbuild.build()
    gla.load()


def _inputs(M, D, F, dtype, seed, x_stride=None, o_stride=None):
    g, dt = torch.Generator(device="cuda").manual_seed(seed), TORCH_DT[dtype]

    def wide(rows, cols, stride, scale=1.0):
        t = torch.full((rows, stride or cols), float("nan"), dtype=dt, device="cuda")[:, :cols]
        t.copy_(torch.randn(rows, cols, device="cuda", generator=g) * scale)
        return t

    return (wide(M, D, x_stride), wide(F, D, None, D ** -0.5), wide(F, D, None, D ** -0.5), wide(M, F, o_stride))


def _sum_bound(K):
    return (K / 16 + 8) * 2.0 ** -23


def _forward64(x, wg, wv):
    x, wg, wv = x.double(), wg.double(), wv.double()
    g, v = x @ wg.t(), x @ wv.t()
    eg = _sum_bound(x.shape[1]) * (x.abs() @ wg.abs().t())
    ev = _sum_bound(x.shape[1]) * (x.abs() @ wv.abs().t())
    return g, v, eg, ev


def _check_forward(x, wg, wv, out, what):
    g, v, eg, ev = _forward64(x, wg, wv)
    s = g * torch.sigmoid(g)
    ref = s * v
    bound = 1.1 * eg * (v.abs() + ev) + s.abs() * ev + 2.0 ** -20 * ref.abs()
    assert_close(out, ref, bound, what)


SHAPES = [(1, 8, 8), (1, 64, 128), (3, 72, 200), (7, 16, 136), (31, 128, 64), (64, 200, 120), (128, 64, 128), (129, 96, 264),
          (255, 192, 256), (256, 384, 512), (257, 136, 1000), (600, 320, 72), (1000, 1024, 40), (20, 2048, 640), (2000, 264, 2304),
          # up to eight tokens: each instantiation, inputs wider than a CTA takes at once, many channels
          (2, 264, 40), (4, 2056, 72), (5, 496, 136), (6, 8, 16), (8, 4104, 24), (1, 5000, 96), (2, 64, 20000), (9, 64, 72),
          # the weights stay resident over several tiles; the gradients' tiles of 384 and 512 columns, whole and cut
          (5000, 384, 520), (3000, 448, 1200), (300, 1544, 2600), (20000, 384, 264), (2500, 2040, 1000),
          # ... and dx's sums cut with and without dW's
          (276, 32, 3160), (1662, 56, 3088), (2016, 248, 5456), (65, 608, 3208), (67, 848, 4224), (4032, 1960, 88),
          (3196, 976, 64)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,D,F", SHAPES, ids=lambda v: str(v))
def test_forward(M, D, F, dtype):
    x, wg, wv, _ = _inputs(M, D, F, dtype, M + D + F)
    out, check = guarded((M, F), x.dtype)
    gla.swiglu_ffn(x, wg, wv, out=out)
    torch.cuda.synchronize()
    assert gla.sync_status() == 0
    check("ffn")
    _check_forward(x, wg, wv, out, f"ffn {M}x{D}x{F} {dtype}")
    assert torch.equal(out, gla.swiglu_ffn(x, wg, wv))


def _check_backward(x, wg, wv, do, dx, dwg, dwv, what):
    u = half_step(x.dtype)
    tiny = 2.0 ** -25 if x.dtype == torch.float16 else 0.0
    g, v, eg, ev = _forward64(x, wg, wv)
    d = do.double()
    s = torch.sigmoid(g)
    dv, slope = d * g * s, s * (1 + g * (1 - s))
    dg = d * v * slope
    # slopes: |silu'| <= 1.1, |silu''| <= 0.5
    edv = 1.1 * eg * d.abs() + 2.0 ** -20 * dv.abs()
    edg = d.abs() * (1.1 * ev + 0.5 * eg * (v.abs() + ev)) + 2.0 ** -19 * (d * v).abs()
    edv, edg = edv + u * (dv.abs() + edv) + tiny, edg + u * (dg.abs() + edg) + tiny
    X, Wg, Wv = x.double(), wg.double(), wv.double()
    ref = dg @ Wg + dv @ Wv
    k = _sum_bound(2 * wg.shape[0])
    bound = edg @ Wg.abs() + edv @ Wv.abs() + k * ((dg.abs() + edg) @ Wg.abs() + (dv.abs() + edv) @ Wv.abs())
    assert_close(dx, ref, bound, what + " dx")
    k = _sum_bound(x.shape[0]) + 64 * 2.0 ** -24
    for got, e, o, n in ((dwg, edg, dg, "dw_gate"), (dwv, edv, dv, "dw_value")):
        assert_close(got, o.t() @ X, e.t() @ X.abs() + k * ((o.abs() + e).t() @ X.abs()), f"{what} {n}")
    if x.shape[0] >= 128 and x.shape[1] >= 64 and wg.shape[0] >= 64:
        for got, r, n in ((dx, ref, "dx"), (dwg, dg.t() @ X, "dw_gate"), (dwv, dv.t() @ X, "dw_value")):
            assert rel_l2(got, r) <= 1.2 * u, f"{what} {n}: relative L2 {rel_l2(got, r):.3g}"


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,D,F", SHAPES, ids=lambda v: str(v))
def test_backward(M, D, F, dtype):
    x, wg, wv, do = _inputs(M, D, F, dtype, 1 + M + D + F)
    ws = torch.full((gla.swiglu_ffn_backward_workspace_bytes(M, D, F),), 255, dtype=torch.uint8, device="cuda")
    got = gla.swiglu_ffn_backward(do, x, wg, wv, workspace=ws)
    torch.cuda.synchronize()
    assert gla.sync_status() == 0
    _check_backward(x, wg, wv, do, *got, f"ffn {M}x{D}x{F} {dtype}")
    assert all(torch.equal(a, b) for a, b in zip(got, gla.swiglu_ffn_backward(do, x, wg, wv)))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_strides(dtype):
    x, wg, wv, do = _inputs(300, 72, 136, dtype, 5, x_stride=160, o_stride=144)
    _check_forward(x, wg, wv, gla.swiglu_ffn(x, wg, wv), "strided")
    _check_backward(x, wg, wv, do, *gla.swiglu_ffn_backward(do, x, wg, wv), "strided")
    one = torch.cat([wg, wv])  # both weights of one projection
    assert torch.equal(gla.swiglu_ffn(x, one[:136], one[136:]), gla.swiglu_ffn(x, wg, wv))


def test_backward_against_differences():
    """The 64-bit formulas' own check: central differences of the forward formula."""
    x, wg, wv, do = (t.double() for t in _inputs(3, 8, 8, "f16", 8))

    def loss(x, wg, wv):
        g = x @ wg.t()
        return (g * torch.sigmoid(g) * (x @ wv.t()) * do).sum()

    g, v = x @ wg.t(), x @ wv.t()
    s = torch.sigmoid(g)
    dv, dg = do * g * s, do * v * s * (1 + g * (1 - s))
    grads = (dg @ wg + dv @ wv, dg.t() @ x, dv.t() @ x)
    h = 1e-6
    for k, grad in enumerate(grads):
        for i in range(grad.numel()):
            a, b = [t.clone() for t in (x, wg, wv)], [t.clone() for t in (x, wg, wv)]
            a[k].view(-1)[i] += h
            b[k].view(-1)[i] -= h
            num = float(loss(*a) - loss(*b)) / (2 * h)
            assert abs(num - float(grad.view(-1)[i])) <= 1e-7 * (1 + abs(num))


def test_values_at_the_ends():
    """Gates far from zero, zeros, and a token of NaN and infinities that must stay alone."""
    x, wg, wv, do = _inputs(200, 64, 128, "bf16", 12)
    x[3] *= 40.0
    x[4] = 0.0
    clean = gla.swiglu_ffn(x, wg, wv)
    _check_forward(x, wg, wv, clean, "large gates")
    assert not clean[4].any()
    _check_backward(x, wg, wv, do, *gla.swiglu_ffn_backward(do, x, wg, wv), "large gates")
    x2 = x.clone()
    x2[7, 0] = float("nan")
    x2[8, 1] = float("inf")
    out = gla.swiglu_ffn(x2, wg, wv)
    keep = [i for i in range(200) if i not in (7, 8)]
    assert torch.equal(out[keep], clean[keep]) and bool(out[7].isnan().all())


def test_empty_and_refusals():
    w = torch.ones(16, 64, device="cuda", dtype=torch.float16)
    x = torch.empty(0, 64, device="cuda", dtype=torch.float16)
    assert gla.swiglu_ffn(x, w, w.clone()).shape == (0, 16)
    dx, dg, dv = gla.swiglu_ffn_backward(torch.empty(0, 16, device="cuda", dtype=torch.float16), x, w, w.clone())
    assert dx.shape == (0, 64) and not dg.any() and not dv.any()
    y = torch.zeros(4, 64, device="cuda", dtype=torch.float16)
    with pytest.raises(ValueError):
        gla.swiglu_ffn(y, w, w[:8])
    with pytest.raises(ValueError):
        gla.swiglu_ffn(y, w, w.bfloat16())
    with pytest.raises(ValueError):
        gla.swiglu_ffn_backward(y, y, w, w)
    with pytest.raises(gla.GLAError):
        gla.swiglu_ffn(y[:, :60].contiguous(), w[:, :60].contiguous(), w[:, :60].contiguous())
    with pytest.raises(gla.GLAError) as e:
        gla.swiglu_ffn(y.float(), w.float(), w.float())
    assert e.value.status == 2
    with pytest.raises(gla.GLAError) as e:
        gla.swiglu_ffn_backward(y[:, :16].contiguous(), y, w, w.clone(),
                                workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3


def test_streams_and_graph():
    x, wg, wv, do = _inputs(700, 192, 768, "bf16", 21)
    ref = (gla.swiglu_ffn(x, wg, wv), *gla.swiglu_ffn_backward(do, x, wg, wv))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = (gla.swiglu_ffn(x, wg, wv, stream=s), *gla.swiglu_ffn_backward(do, x, wg, wv, stream=s))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = (gla.swiglu_ffn(x, wg, wv), *gla.swiglu_ffn_backward(do, x, wg, wv))
    x2, _, _, do2 = _inputs(700, 192, 768, "bf16", 22)
    x.copy_(x2)
    do.copy_(do2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((gla.swiglu_ffn(x, wg, wv), *gla.swiglu_ffn_backward(do, x, wg, wv)), res))
    assert gla.sync_status() == 0
