"""Layer norm and its backward pass against the formulas in 64 bits.

Bounds before the output's own rounding, from fp32 arithmetic (U = 2^-24, half a step): a row's sums add at most
16 elements in a thread, then trees of at most 10 levels, so a mean is off by at most 26 U of the mean magnitude;
the centred value by that and one rounding, r by 15 U or so; 64 U of the magnitudes covers them with the products
after.  A column sum adds one row at a time in at most n / (CTAs) + 64 steps."""
import pytest
import torch

from block_testutil import TORCH_DT, U32, assert_close, guarded
from paper_2609_26590_gb300 import build as gbuild
from paper_2609_26590_gb300 import gla

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _built():
    gbuild.build()
    gla.load()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inputs(rows, D, dtype, seed, stride=None, offset=0.5):
    g = _gen(seed)
    wide = torch.full((rows, stride or D), float("nan"), dtype=TORCH_DT[dtype], device="cuda")
    x = wide[:, :D]
    x.copy_(torch.randn(rows, D, device="cuda", generator=g) * 1.5 + offset)
    dwide = torch.full((rows, stride or D), float("nan"), dtype=TORCH_DT[dtype], device="cuda")
    dy = dwide[:, :D]
    dy.copy_(torch.randn(rows, D, device="cuda", generator=g))
    w = 1 + 0.2 * torch.randn(D, device="cuda", generator=g)
    b = 0.3 * torch.randn(D, device="cuda", generator=g)
    return x, dy, w, b


def _forward64(x, w, b, eps=EPS):
    x = x.double()
    m = x.mean(1, keepdim=True)
    r = 1 / torch.sqrt((x - m).square().mean(1, keepdim=True) + eps)
    w = torch.ones(x.shape[1], device="cuda", dtype=torch.float64) if w is None else w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    return (x - m) * r * w + b, m[:, 0], r[:, 0]


def _check_forward(x, w, b, out, mean, rstd, what):
    ref, m, r = _forward64(x, w, b)
    amp = (x.double().abs().amax(1) * r)[:, None]  # largest |x| r of the row
    wm = 1.0 if w is None else w.double().abs()
    bm = 0.0 if b is None else b.double().abs()
    assert_close(out, ref, 64 * U32 * ((amp + 1) * wm + bm), what)
    if mean is not None:
        assert_close(mean, m, 64 * U32 * x.double().abs().amax(1), what + " mean")
        assert_close(rstd, r, 64 * U32 * r * (1 + amp[:, 0] ** 2), what + " rstd")


# every team (8 lanes, a warp, a CTA), full and ragged vectors, single elements and single rows
SHAPES = [(1, 1), (3, 2), (5, 7), (1, 64), (33, 64), (17, 127), (130, 128), (7, 130), (1600, 192), (77, 384), (2, 512),
          (9, 513), (65, 1000), (41, 1001), (3, 4096), (2, 4099), (5, 8192), (1, 16384), (2, 16383),
          (130, 300), (65, 320), (33, 380), (9, 460), (41, 1004), (3, 8196), (1, 16380), (19, 4), (7, 12),
          (701, 640), (613, 1004), (650, 2052), (609, 4096), (620, 4088), (1300, 516), (2500, 384), (2433, 300), (2441, 264),
          (2433, 955), (2440, 1022), (2500, 2046), (2437, 510), (2500, 514), (1300, 1), (1217, 33), (1301, 129), (1220, 333), (1219, 767)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,D", SHAPES, ids=[f"{r}x{d}" for r, d in SHAPES])
def test_forward(rows, D, dtype):
    x, _, w, b = _inputs(rows, D, dtype, 100 + rows + D)
    out, check = guarded((rows, D), x.dtype)
    got, mean, rstd = gla.layernorm(x, w, b, EPS, stats=True, out=out)
    assert got is out
    check("layernorm")
    _check_forward(x, w, b, out, mean, rstd, f"{rows}x{D} {dtype}")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D,stride", [(64, 192), (64, 65), (200, 208), (33, 40), (1000, 2000)])
def test_strides_and_no_affine(D, stride, dtype):
    x, dy, w, b = _inputs(37, D, dtype, 7 + D + stride, stride)
    out, mean, rstd = gla.layernorm(x, None, None, EPS, stats=True)
    _check_forward(x, None, None, out, mean, rstd, "no affine")
    _check_forward(x, w, None, gla.layernorm(x, w, None, EPS), None, None, "no bias")
    dx, dw, db = gla.layernorm_backward(dy, x, None, mean, rstd)
    assert dw is None and db is None
    _check_backward(x, dy, None, mean, rstd, dx, None, None, "no affine, strided")


def test_leading_dimensions():
    x = torch.randn(3, 5, 96, device="cuda", generator=_gen(1)).half()
    w, b = torch.ones(96, device="cuda"), torch.zeros(96, device="cuda")
    out, mean, rstd = gla.layernorm(x, w, b, EPS, stats=True)
    assert out.shape == x.shape and mean.shape == (3, 5)
    assert torch.equal(out.view(15, 96), gla.layernorm(x.view(15, 96), w, b, EPS))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_constant_rows_and_far_offsets(dtype):
    # a constant row normalises to its bias; rows far from zero keep their spread
    x, _, w, b = _inputs(6, 256, dtype, 3, offset=0.0)
    x[0] = 0.0
    x[1] = 3.0
    x[2] += 100.0
    out, mean, rstd = gla.layernorm(x, w, b, EPS, stats=True)
    _check_forward(x, w, b, out, mean, rstd, "offsets")
    assert torch.equal(out[0], b.to(x.dtype))


def test_a_nan_row_stays_alone():
    x, dy, w, b = _inputs(40, 192, "f16", 5)
    clean, mean, rstd = gla.layernorm(x, w, b, EPS, stats=True)
    x2 = x.clone()
    x2[7, 3] = float("nan")
    x2[9, 0] = float("inf")
    out = gla.layernorm(x2, w, b, EPS)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[7, 9]] = False
    assert torch.equal(out[keep], clean[keep])
    assert bool(out[7].isnan().all()) and bool(out[9].isnan().all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,D,stride", [(640, 1000, 2000), (640, 1004, 1012), (700, 2056, 4112), (2500, 384, 1152), (2500, 300, 308),
                                           (2500, 955, 957), (2500, 1022, 1030), (1300, 333, 335)])
def test_many_strided_rows(rows, D, stride, dtype):
    """Enough rows for a warp to hold each: strides, no weights, no bias, statistics, and a NaN that stays in its row."""
    x, _, w, b = _inputs(rows, D, dtype, 11 + D, stride)
    out, mean, rstd = gla.layernorm(x, None, None, EPS, stats=True)
    _check_forward(x, None, None, out, mean, rstd, "no affine")
    _check_forward(x, w, None, gla.layernorm(x, w, None, EPS), None, None, "no bias")
    clean = gla.layernorm(x, w, b, EPS)
    _check_forward(x, w, b, clean, None, None, "affine")
    x[7, 3] = float("nan")
    x[rows - 1, D - 1] = float("inf")
    out = gla.layernorm(x, w, b, EPS)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[[7, rows - 1]] = False
    assert torch.equal(out[keep], clean[keep])
    assert bool(out[7].isnan().all()) and bool(out[rows - 1].isnan().all())


def _check_backward(x, dy, w, mean, rstd, dx, dw, db, what):
    n, D = x.shape
    x64, d64, m, r = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x64 - m) * r
    d = d64 if w is None else d64 * w.double()
    c1, c2 = d.mean(1, keepdim=True), (d * xh).mean(1, keepdim=True)
    ref = r * (d - c1 - xh * c2)
    amp = (x64.abs().amax(1, keepdim=True) + m.abs()) * r  # a centred value is off by U of this
    mag = r * (d.abs() + d.abs().mean(1, keepdim=True) + xh.abs() * (d * xh).abs().mean(1, keepdim=True))
    assert_close(dx, ref, 64 * U32 * mag * (1 + amp), what + " dx")
    if dw is not None:
        steps = n / 152 + 128
        s = (d64 * xh).abs().sum(0) + (d64.abs() * amp).sum(0)
        assert_close(dw, (d64 * xh).sum(0), steps * U32 * s, what + " dweight")
        assert_close(db, d64.sum(0), steps * U32 * d64.abs().sum(0), what + " dbias")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,D", SHAPES + [(5000, 64), (20000, 24), (24577, 264), (25001, 300), (4867, 256)], ids=lambda v: str(v))
def test_backward(rows, D, dtype):
    x, dy, w, b = _inputs(rows, D, dtype, 200 + rows + D)
    _, mean, rstd = gla.layernorm(x, w, b, EPS, stats=True)
    ws = torch.full((gla.layernorm_backward_workspace_bytes(rows, D),), 255, dtype=torch.uint8, device="cuda")
    dx, dw, db = gla.layernorm_backward(dy, x, w, mean, rstd, workspace=ws)
    _check_backward(x, dy, w, mean, rstd, dx, dw, db, f"{rows}x{D} {dtype}")
    again = gla.layernorm_backward(dy, x, w, mean, rstd)
    assert all(torch.equal(a, c) for a, c in zip((dx, dw, db), again))  # fixed order: the same bits


def test_backward_against_differences():
    # the 64-bit formula's own check: central differences of the forward formula
    g = _gen(11)
    x = torch.randn(3, 10, device="cuda", dtype=torch.float64, generator=g)
    w = torch.randn(10, device="cuda", dtype=torch.float64, generator=g)
    b = torch.randn(10, device="cuda", dtype=torch.float64, generator=g)
    dy = torch.randn(3, 10, device="cuda", dtype=torch.float64, generator=g)
    x32, dy32 = x.float(), dy.float()
    _, mean, rstd = gla.layernorm(x32, w.float(), b.float(), EPS, stats=True)
    dx, dw, db = gla.layernorm_backward(dy32, x32, w.float(), mean, rstd)

    def loss(x, w, b):
        return (_forward64(x, w, b)[0] * dy32.double()).sum()

    h = 1e-6
    for t, grad in ((x32.double(), dx), (w.float().double(), dw), (b.float().double(), db)):
        for i in range(t.numel()):
            args = [x32.double(), w.float().double(), b.float().double()]
            k = 0 if grad is dx else 1 if grad is dw else 2
            up, dn = args[k].clone(), args[k].clone()
            up.view(-1)[i] += h
            dn.view(-1)[i] -= h
            a1, a2 = list(args), list(args)
            a1[k], a2[k] = up, dn
            num = float(loss(*a1) - loss(*a2)) / (2 * h)
            # central differences: h^2 and 2^-52 / h terms, a few 1e-9; fp32 gradients: a few 1e-6
            assert abs(num - float(grad.view(-1)[i])) <= 2e-5 * (1 + abs(num))


def test_empty_and_refusals():
    w = torch.ones(64, device="cuda")
    x = torch.empty(0, 64, device="cuda", dtype=torch.float16)
    out, mean, rstd = gla.layernorm(x, w, w, EPS, stats=True)
    assert out.shape == (0, 64) and mean.shape == (0,)
    dx, dw, db = gla.layernorm_backward(x, x, w, mean, rstd)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    y = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError):
        gla.layernorm(y, w[:32], w, EPS)
    with pytest.raises(ValueError):
        gla.layernorm(y, w.half(), w, EPS)
    with pytest.raises(ValueError):
        gla.layernorm(y[0:1].expand(4, 64), w, w, EPS)
    with pytest.raises(ValueError):
        gla.layernorm_backward(y.half(), y, w, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"))
    with pytest.raises(gla.GLAError):
        gla.layernorm(y, w, w, EPS, out=y)
    with pytest.raises(gla.GLAError):
        gla.layernorm(torch.zeros(1, 16385, device="cuda"), None, None, EPS)
    with pytest.raises(gla.GLAError) as e:
        gla.layernorm_backward(y, y, w, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"),
                               workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3


def test_streams_and_graph():
    x, dy, w, b = _inputs(700, 384, "bf16", 21)
    ref, mean, rstd = gla.layernorm(x, w, b, EPS, stats=True)
    grads = gla.layernorm_backward(dy, x, w, mean, rstd)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = gla.layernorm(x, w, b, EPS, stream=s)
    g2 = gla.layernorm_backward(dy, x, w, mean, rstd, stream=s)
    s.synchronize()
    assert torch.equal(out, ref) and all(torch.equal(a, c) for a, c in zip(grads, g2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, m2, r2 = gla.layernorm(x, w, b, EPS, stats=True)
        g3 = gla.layernorm_backward(dy, x, w, m2, r2)
    for seed in (31, 32):
        x3, dy3, _, _ = _inputs(700, 384, "bf16", seed)
        x.copy_(x3)
        dy.copy_(dy3)
        graph.replay()
        torch.cuda.synchronize()
        ref, mean, rstd = gla.layernorm(x, w, b, EPS, stats=True)
        assert torch.equal(o, ref)
        assert all(torch.equal(a, c) for a, c in zip(g3, gla.layernorm_backward(dy, x, w, mean, rstd)))
