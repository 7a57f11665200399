"""The operators around the mixer where an element's offset passes 32 bits: tokens a long way apart in inputs, and
inputs, outputs and states of more than 2^31 elements.

What lies past the border is compared with the same rows in a call of their own, whose offsets are small.  Rows of
layer norm, tokens of the convolution and of the feed-forward step do not depend on how many there are: the same
bits, except where another kernel takes few rows or tokens.  The scan and the weights' gradients cut their sums by the size
of the problem, so there both calls' errors count."""
import pytest
import torch

from block_testutil import half_step
from paper_2609_26590_gb300 import build as gbuild
from paper_2609_26590_gb300 import gla

pytestmark = pytest.mark.gpu
FAR = (1 << 30) + 64  # elements between tokens: the third lies past 2^31


@pytest.fixture(scope="module", autouse=True)
def _built():
    gbuild.build()
    gla.load()


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("less than 60 GB of device memory free")
    yield
    torch.cuda.empty_cache()


def _far(t):
    """t [n, width] with its rows FAR elements apart."""
    n, width = t.shape
    buf = torch.empty((n - 1) * FAR + width, dtype=t.dtype, device="cuda")
    view = buf.as_strided((n, width), (FAR, 1))
    view.copy_(t)
    return view


def _randn(*s, dtype=torch.float16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(s, device="cuda", generator=g).to(dtype)


def test_far_tokens_layernorm():
    x, dy = _randn(4, 64), _randn(4, 64, seed=1)
    w, b = torch.rand(64, device="cuda"), torch.rand(64, device="cuda")
    y, m, r = gla.layernorm(x, w, b, 1e-5, stats=True)
    assert torch.equal(gla.layernorm(_far(x), w, b, 1e-5), y)
    for got, want in zip(gla.layernorm_backward(_far(dy), _far(x), w, m, r), gla.layernorm_backward(dy, x, w, m, r)):
        assert torch.equal(got, want)


def test_far_tokens_ffn():
    """Four tokens (the few-token kernel) and, with wide weights, the tensor cores' kernel."""
    for D, F in ((64, 72), (2048, 4104)):
        x, dh = _randn(4, D), _randn(4, F, seed=1)
        wg, wv = _randn(F, D, seed=2) / D ** 0.5, _randn(F, D, seed=3) / D ** 0.5
        assert torch.equal(gla.swiglu_ffn(_far(x), wg, wv), gla.swiglu_ffn(x, wg, wv))
        for got, ref in zip(gla.swiglu_ffn_backward(_far(dh), _far(x), wg, wv), gla.swiglu_ffn_backward(dh, x, wg, wv)):
            assert torch.equal(got, ref)
    assert gla.sync_status() == 0


@pytest.mark.parametrize("order", range(4))
def test_far_tokens_conv_and_scan(order):
    gh, gw, E, N = 2, 2, 64, 16
    x, dl, z = (_randn(4, E, seed=s) for s in range(3))
    Bm, C = _randn(4, N, seed=3), _randn(4, N, seed=4)
    w, A = _randn(E, 4, dtype=torch.float32), -torch.rand(E, N, device="cuda") - 0.1
    got = gla.causal_conv(_far(x)[None], w, None, gh, gw, order, final_state=True)
    want = gla.causal_conv(x[None], w, None, gh, gw, order, final_state=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = gla.ssm_scan(_far(x)[None], _far(dl)[None], A, _far(Bm)[None], _far(C)[None], gh, gw, order, z=_far(z)[None])
    want = gla.ssm_scan(x[None], dl[None], A, Bm[None], C[None], gh, gw, order, z=z[None])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_far_tokens_steps():
    E, N, B = 64, 16, 4
    x, dl = _randn(B, E), _randn(B, E, seed=1)
    Bm, C = _randn(B, N, seed=2), _randn(B, N, seed=3)
    w, A = _randn(E, 4, dtype=torch.float32), -torch.rand(E, N, device="cuda") - 0.1
    cs, hs = _randn(B, 3, E, seed=4), _randn(B, E, N, dtype=torch.float32, seed=5)
    got, want = gla.causal_conv_step(_far(x), cs.clone(), w, None), gla.causal_conv_step(x, cs.clone(), w, None)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = gla.ssm_step(_far(x), _far(dl), A, _far(Bm), _far(C), hs.clone())
    want = gla.ssm_step(x, dl, A, Bm, C, hs.clone())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_many_rows_layernorm():
    n, D = (1 << 21) + 77, 1024
    x = torch.empty(n, D, dtype=torch.float16, device="cuda").normal_()
    w, b = torch.rand(D, device="cuda"), torch.rand(D, device="cuda")
    y, m, r = gla.layernorm(x, w, b, 1e-5, stats=True)
    tail = slice(n - 2000, n)  # (enough rows for the same kernel)
    y1, m1, r1 = gla.layernorm(x[tail], w, b, 1e-5, stats=True)
    assert torch.equal(y[tail], y1) and torch.equal(m[tail], m1) and torch.equal(r[tail], r1)
    dx = gla.layernorm_backward(y, x, w, m, r)[0]
    assert torch.equal(dx[tail], gla.layernorm_backward(y1, x[tail], w, m1, r1)[0])


def test_many_outputs_ffn():
    M, D, F = (1 << 20) + 129, 64, 2056
    x = torch.empty(M, D, dtype=torch.bfloat16, device="cuda").normal_()
    wg, wv = _randn(F, D, dtype=torch.bfloat16, seed=2) / 8, _randn(F, D, dtype=torch.bfloat16, seed=3) / 8
    y = gla.swiglu_ffn(x, wg, wv)
    tail = slice(M - 600, M)
    assert torch.equal(y[tail], gla.swiglu_ffn(x[tail], wg, wv))
    dx = gla.swiglu_ffn_backward(y, x, wg, wv)[0]
    del y
    # one fp32 sum of 2 F terms each, in two orders, rounded once: a step of the result and 2 F half steps of fp32
    # of its terms' size at the worst
    d64 = x[tail].double()
    G, V = d64 @ wg.double().t(), d64 @ wv.double().t()
    s = torch.sigmoid(G)
    dh = (G * s * V).to(torch.bfloat16).double()
    terms = (dh * V * s * (1 + G * (1 - s))).abs() @ wg.double().abs() + (dh * G * s).abs() @ wv.double().abs()
    ref = gla.swiglu_ffn_backward(gla.swiglu_ffn(x[tail], wg, wv), x[tail], wg, wv)[0]
    limit = 2 * half_step(torch.bfloat16) * ref.double().abs() + 2 * 2 * F * 2.0 ** -24 * 1.02 * terms + 2.0 ** -120
    assert bool(((dx[tail].double() - ref.double()).abs() <= limit).all())
    assert gla.sync_status() == 0


def test_long_grid_conv_and_scan():
    gh, gw, E, N = 1024, 1024, 1032, 4
    T = gh * gw
    x = torch.empty(2, T, E, dtype=torch.float16, device="cuda").normal_()
    w = _randn(E, 3, dtype=torch.float32)
    y, st = gla.causal_conv(x, w, None, gh, gw, gla.COL_REV, final_state=True)
    y1, st1 = gla.causal_conv(x[1:], w, None, gh, gw, gla.COL_REV, final_state=True)
    assert torch.equal(y[1:], y1) and torch.equal(st[1:], st1)
    del y, y1
    Bm, C = (torch.empty(2, T, N, dtype=torch.float16, device="cuda").normal_() for _ in range(2))
    A = -torch.rand(E, N, device="cuda") - 0.5
    bias = torch.full((E,), -1.0, device="cuda")
    y, h = gla.ssm_scan(x, x, A, Bm, C, gh, gw, gla.COL_REV, delta_bias=bias)
    y1, h1 = gla.ssm_scan(x[1:], x[1:], A, Bm[1:], C[1:], gh, gw, gla.COL_REV, delta_bias=bias)
    # a state forgets within tens of positions (dt A is -0.2 or less on average), so a value's relative error is below
    # a hundred half steps of fp32 of its terms; of 4e9 normal products dt x B the largest is below 150 and |C| below 6.5
    eps = 100 * 2.0 ** -24 * 150
    assert float((h[1] - h1[0]).abs().max()) <= eps
    for t in range(0, T, 1 << 18):
        a, b = y[1, t:t + (1 << 18)].float(), y1[0, t:t + (1 << 18)].float()
        limit = 2 * half_step(torch.float16) * torch.maximum(a.abs(), b.abs()) + N * 6.5 * eps
        assert bool(((a - b).abs() <= limit).all())


def test_many_states_step():
    B, E, N = (1 << 17) + 5, 1024, 32
    h = torch.empty(B, E, N, device="cuda").normal_()
    x, dl = _randn(B, E), _randn(B, E, seed=1)
    Bm, C = _randn(B, N, seed=2), _randn(B, N, seed=3)
    A = -torch.rand(E, N, device="cuda") - 0.1
    tail = slice(B - 9, B)
    want = gla.ssm_step(x[tail], dl[tail], A, Bm[tail], C[tail], h[tail].clone())
    got = gla.ssm_step(x, dl, A, Bm, C, h)
    assert torch.equal(got[0][tail], want[0]) and torch.equal(got[1][tail], want[1])
