"""The operators together, as a pre-norm block runs them: layer norm, projections, the causal convolution and the
selective scan along one scan order, a residual, layer norm, the gated feed-forward step and its down projection.

The reference makes the same steps in 64 bits and rounds where the block stores 16-bit values, so the two differ where
fp32 arithmetic moves a value across a rounding border.  Eleven steps round; if each moves up to a sixteenth of its
values by one step (2 u, u half a step), that is u / 2 in the mean square each, behind gains of up to 2: below
4 u together.  The training chain compares with 64-bit autograd without those roundings: five of them (the norm's
output, dG and dV, the step's gradient, the norm's gradient), each u / sqrt(3) or less in the mean square: below 3 u."""
import pathlib
import subprocess
import sys

import pytest
import torch

from block_testutil import TORCH_DT, half_step, rel_l2, scan_tokens
from paper_2609_26590_gb300 import build as gbuild
from paper_2609_26590_gb300 import gla

pytestmark = pytest.mark.gpu
EPS = 1e-5
D, E, N, W, F = 64, 128, 16, 4, 200


@pytest.fixture(scope="module", autouse=True)
def _built():
    gbuild.build()
    gla.load()


def _weights(dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*s):
        return torch.randn(s, device="cuda", generator=g)

    return {
        "n1": 1 + 0.1 * randn(D), "b1": 0.1 * randn(D), "n2": 1 + 0.1 * randn(D), "b2": 0.1 * randn(D),
        "w_in": (randn(D, 2 * E) / D ** 0.5).to(dt), "conv": randn(E, W) / W ** 0.5, "conv_b": 0.1 * randn(E),
        "w_x": (randn(E, E + 2 * N) / E ** 0.5).to(dt), "A": -torch.exp(randn(E, N)), "skip": 1 + 0.1 * randn(E),
        "dt_b": -3 + randn(E), "w_out": (randn(E, D) / E ** 0.5).to(dt), "wg": (randn(F, D) / D ** 0.5).to(dt),
        "wv": (randn(F, D) / D ** 0.5).to(dt), "w_down": (randn(F, D) / F ** 0.5).to(dt)}


def _block(x, w, gh, gw, order, state=None):
    """The block on the GPU; state: (convolution, scan) of the tokens before, for single tokens (x [B, D])."""
    step = state is not None
    h = gla.layernorm(x, w["n1"], w["b1"], EPS)
    xz = h @ w["w_in"]
    if step:
        u, conv = gla.causal_conv_step(xz[..., :E], state[0], w["conv"], w["conv_b"])
    else:
        u, conv = gla.causal_conv(xz[..., :E], w["conv"], w["conv_b"], gh, gw, order, final_state=True)
    p = u @ w["w_x"]
    args = (u, p[..., :E], w["A"], p[..., E:E + N], p[..., E + N:])
    kw = dict(D=w["skip"], z=xz[..., E:], delta_bias=w["dt_b"])
    if step:
        y, scan = gla.ssm_step(*args, state[1], **kw)
    else:
        y, scan = gla.ssm_scan(*args, gh, gw, order, **kw)
    x1 = x + y @ w["w_out"]
    h2 = gla.layernorm(x1, w["n2"], w["b2"], EPS)
    return x1 + gla.swiglu_ffn(h2, w["wg"], w["wv"]) @ w["w_down"], (conv, scan)


def _block64(x, w, gh, gw, order):
    dt = x.dtype

    def r(t):  # a 16-bit tensor in between
        return t.to(dt).double()

    def norm(t, n, b):
        m = t.mean(-1, keepdim=True)
        return r((t - m) / torch.sqrt((t - m).square().mean(-1, keepdim=True) + EPS) * w[n].double() + w[b].double())

    v = {n: t.double() for n, t in w.items()}
    x0 = x.double()
    T = gh * gw
    tok = scan_tokens(gh, gw, order)
    xz = r(norm(x0, "n1", "b1") @ v["w_in"])
    a = torch.nn.functional.pad(xz[:, tok, :E], (0, 0, W - 1, 0))
    acc = v["conv_b"] + sum(v["conv"][:, j] * a[:, j:j + T] for j in range(W))
    u = r(acc * torch.sigmoid(acc))
    p = r(u @ v["w_x"])
    dt_ = torch.nn.functional.softplus(p[..., :E] + v["dt_b"], threshold=1e9)
    h = torch.zeros(x.shape[0], E, N, dtype=torch.float64, device="cuda")
    ys = []
    for t in range(T):
        s = dt_[:, t, :, None]
        h = torch.exp(s * v["A"]) * h + s * u[:, t, :, None] * p[:, t, None, E:E + N]
        ys.append((h * p[:, t, None, E + N:]).sum(-1))
    y = torch.stack(ys, 1) + v["skip"] * u
    z = xz[:, tok, E:]
    out = torch.empty_like(y)
    out[:, tok] = y * z * torch.sigmoid(z)
    x1 = r(x0 + r(r(out) @ v["w_out"]))
    h2 = norm(x1, "n2", "b2")
    g = h2 @ v["wg"].t()
    f = r(g * torch.sigmoid(g) * (h2 @ v["wv"].t()))
    return r(x1 + r(f @ v["w_down"])), h


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("order", range(4))
def test_block(order, dtype):
    dt = TORCH_DT[dtype]
    w = _weights(dt, 31)
    x = torch.randn(2, 11 * 13, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(32 + order)).to(dt)
    out, (conv, scan) = _block(x, w, 11, 13, order)
    ref, h = _block64(x, w, 11, 13, order)
    u = half_step(dt)
    assert rel_l2(out, ref) <= 4 * u, f"{rel_l2(out, ref) / u:.2f} u"
    assert rel_l2(scan, h) <= 4 * u, f"{rel_l2(scan, h) / u:.2f} u"
    assert gla.sync_status() == 0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_prompt_then_tokens(dtype):
    """A prompt, then single tokens from its states, give the longer prompt's outputs."""
    dt = TORCH_DT[dtype]
    w = _weights(dt, 41)
    T, cut = 40, 35
    x = torch.randn(3, T, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(42)).to(dt)
    whole, _ = _block(x, w, 1, T, 0)
    _, state = _block(x[:, :cut].contiguous(), w, 1, cut, 0)
    for t in range(cut, T):
        out, state = _block(x[:, t].contiguous(), w, 1, 1, 0, state)
        assert rel_l2(out, whole[:, t].double()) <= 4 * half_step(dt)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_training_chain(dtype):
    """Norm, feed-forward step and down projection forward and back, against 64-bit autograd."""
    dt = TORCH_DT[dtype]
    w = _weights(dt, 51)
    g = torch.Generator(device="cuda").manual_seed(52)
    x = torch.randn(500, D, device="cuda", generator=g).to(dt)
    dy = torch.randn(500, D, device="cuda", generator=g).to(dt)
    h, mean, rstd = gla.layernorm(x, w["n2"], w["b2"], EPS, stats=True)
    f = gla.swiglu_ffn(h, w["wg"], w["wv"])
    df = dy @ w["w_down"].t()
    dh, dwg, dwv = gla.swiglu_ffn_backward(df, h, w["wg"], w["wv"])
    dx, dn, db = gla.layernorm_backward(dh, x, w["n2"], mean, rstd)

    leaves = {n: t.double().requires_grad_() for n, t in (("x", x), ("n2", w["n2"]), ("b2", w["b2"]), ("wg", w["wg"]), ("wv", w["wv"]))}
    h64 = torch.nn.functional.layer_norm(leaves["x"], (D,), leaves["n2"], leaves["b2"], EPS)
    f64 = torch.nn.functional.silu(h64 @ leaves["wg"].t()) * (h64 @ leaves["wv"].t())
    grads = dict(zip(leaves, torch.autograd.grad(f64, list(leaves.values()), df.double())))
    u = half_step(dt)
    assert rel_l2(f, f64.detach()) <= 3 * u
    for n, got in (("x", dx), ("n2", dn), ("b2", db), ("wg", dwg), ("wv", dwv)):
        assert rel_l2(got, grads[n]) <= 3 * u, f"{n}: {rel_l2(got, grads[n]) / u:.2f} u"


def test_block_captured():
    """The block captured into a CUDA graph and replayed on other tokens."""
    w = _weights(torch.float16, 61)
    gen = torch.Generator(device="cuda").manual_seed(62)
    x = torch.randn(1, 64, D, device="cuda", generator=gen).half()
    _block(x, w, 8, 8, 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, (conv, scan) = _block(x, w, 8, 8, 3)
    x.copy_(torch.randn(1, 64, D, device="cuda", generator=gen).half())
    graph.replay()
    torch.cuda.synchronize()
    again, (conv2, scan2) = _block(x, w, 8, 8, 3)
    assert torch.equal(out, again) and torch.equal(conv, conv2) and torch.equal(scan, scan2)


def test_two_streams_at_once():
    """Two blocks on two streams, nothing ordering them: each its own results."""
    w = _weights(torch.bfloat16, 71)
    xs = [torch.randn(2, 400, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(72 + i)).bfloat16()
          for i in range(2)]
    ref = [_block(x, w, 20, 20, i)[0] for i, x in enumerate(xs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append(_block(xs[i], w, 20, 20, i)[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


FIRST_CALLS = {
    "layernorm": "lambda: gla.layernorm(x, v, v, 1e-5)",
    "layernorm_backward": "lambda: gla.layernorm_backward(x, x, v, s, s)[0]",
    "causal_conv": "lambda: gla.causal_conv(x[None], w, v, 8, 8)[0]",
    "causal_conv_step": "lambda: gla.causal_conv_step(x, c, w, v, state_out=c2)[0]",
    "ssm_scan": "lambda: gla.ssm_scan(x[None], x[None], a, b[None], b[None], 8, 8)[0]",
    "ssm_step": "lambda: gla.ssm_step(x, x, a, b, b, h, state_out=h2)[0]",
    "swiglu_ffn": "lambda: gla.swiglu_ffn(x, f, f)",
    "swiglu_ffn_few": "lambda: gla.swiglu_ffn(x[:1], f, f)",
    "swiglu_ffn_backward": "lambda: gla.swiglu_ffn_backward(x, x, q, q)[0]",
}


@pytest.mark.parametrize("name", sorted(FIRST_CALLS))
def test_first_call_captured(name):
    """The first call of a process inside a capture: what an operator asks the device once is legal there."""
    code = f"""
import torch
from paper_2609_26590_gb300 import gla
gla.load()
g = torch.Generator(device="cuda").manual_seed(5)
def r(*n, dt=torch.float16): return torch.randn(n, device="cuda", generator=g).to(dt)
x, f, q, b = r(64, 128), r(200, 128) / 11, r(128, 128) / 11, r(64, 16)
v, s, w, a = torch.rand(128, device="cuda"), torch.rand(64, device="cuda"), r(128, 4, dt=torch.float32), -torch.rand(128, 16, device="cuda")
c, h = r(64, 3, 128), r(64, 128, 16, dt=torch.float32)
c2, h2 = torch.empty_like(c), torch.empty_like(h)
call = {FIRST_CALLS[name]}
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = call()
graph.replay()
torch.cuda.synchronize()
assert torch.equal(out, call()) and bool(torch.isfinite(out.float()).all())
assert gla.sync_status() == 0
"""
    root = pathlib.Path(__file__).resolve().parent.parent
    run = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
