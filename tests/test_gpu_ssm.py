"""Causal convolution and selective scan, whole sequences and single tokens, against the formulas in 64 bits.

Bounds before the output's own rounding (U = 2^-24).  Convolution: W multiply-adds of fp32 values, (W + 1) U of
the sum of magnitudes, through SiLU's slope (at most 1.1), and 2^-20 of the value for SiLU by the hardware's power
and reciprocal.  Scan: dt = softplus(v) comes from an exponential whose error is 2 + 1.2 |v| steps (|v| <= 10
here: 2^-19 of it); the power of a step has the argument's rounding and dt's error, |dt A| (2^-19 + 2^-22), and its own 2^-22;
errors of the state decay with it, so they follow the recurrence err = a (err + eps |h|) + 2^-18 |dt x B|, run
in 64 bits beside the values on magnitudes, as the segments' folds do (their decays' exponents are sums of dt:
covered by 4 eps).  The readout adds N terms."""
import pytest
import torch

from block_testutil import TORCH_DT, U32, assert_close, guarded, scan_tokens
from paper_2609_26590_gb300 import build as gbuild
from paper_2609_26590_gb300 import gla

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    gbuild.build()
    gla.load()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


# ------------------------------------------------------------------ convolution

def _conv64(x, w, b, tok, init, silu):
    B, T, E = x.shape
    W = w.shape[1]
    pre = torch.zeros(B, W - 1, E, dtype=torch.float64, device="cuda") if init is None else init.double()
    a = torch.cat([pre, x.double()[:, tok]], 1)
    acc = torch.zeros(B, T, E, dtype=torch.float64, device="cuda") + (0 if b is None else b.double())
    mag = acc.abs()
    for j in range(W):
        acc = acc + w.double()[:, j] * a[:, j:j + T]
        mag = mag + (w.double()[:, j] * a[:, j:j + T]).abs()
    bound = (W + 1) * U32 * mag
    if silu:
        bound = 1.1 * bound + 2.0 ** -20 * acc.abs()
        acc = acc * torch.sigmoid(acc)
    out, bnd = torch.empty_like(acc), torch.empty_like(acc)
    out[:, tok], bnd[:, tok] = acc, bound
    return out, bnd, a[:, T:]


CONV = [  # B, grid_h, grid_w, E, W, x stride (0: E)
    (1, 1, 1, 1, 4, 0), (2, 1, 2, 8, 4, 0), (1, 1, 3, 24, 4, 0), (3, 5, 7, 40, 4, 0), (2, 4, 4, 33, 3, 0), (1, 16, 1, 72, 2, 0),
    (2, 1, 17, 100, 4, 0), (1, 9, 11, 64, 3, 128), (2, 6, 5, 30, 4, 61), (1, 40, 40, 96, 4, 0), (5, 3, 33, 2056, 4, 0),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("case", CONV, ids=lambda c: "x".join(map(str, c)))
def test_conv(case, dtype):
    B, gh, gw, E, W, stride = case
    g = _gen(sum(case))
    wide = torch.full((B, gh * gw, stride or E), float("nan"), device="cuda", dtype=TORCH_DT[dtype])
    x = wide[:, :, :E]
    x.copy_(_randn(g, B, gh * gw, E))
    w, b = _randn(g, E, W) / 2, 0.2 * _randn(g, E)
    init = _randn(g, B, W - 1, E).to(x.dtype)
    for order in range(4):
        for silu, bias, st in ((True, b, None), (False, None, init)):
            tok = scan_tokens(gh, gw, order)
            out, check = guarded((B, gh * gw, E), x.dtype)
            fs, check_fs = guarded((B, W - 1, E), x.dtype)
            gla.causal_conv(x, w, bias, gh, gw, order, silu=silu, initial_state=st, final_state=fs, out=out)
            check("conv")
            check_fs("conv state")
            ref, bound, state = _conv64(x, w, bias, tok, st, silu)
            assert_close(out, ref, bound, f"conv {case} {dtype} order {order}")
            assert torch.equal(fs.double(), state)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,E,W", [(1, 1, 4), (3, 40, 4), (257, 33, 3), (2, 4096, 2), (70000, 8, 4)])
def test_conv_step(B, E, W, dtype):
    g = _gen(B + E + W)
    x, st = _randn(g, B, E).to(TORCH_DT[dtype]), _randn(g, B, W - 1, E).to(TORCH_DT[dtype])
    w, b = _randn(g, E, W) / 2, 0.2 * _randn(g, E)
    ref, bound, state = _conv64(x[:, None], w, b, torch.zeros(1, dtype=torch.long, device="cuda"), st, True)
    out, new = gla.causal_conv_step(x, st, w, b, state_out=torch.empty_like(st))
    assert_close(out, ref[:, 0], bound[:, 0], "conv step")
    assert torch.equal(new.double(), state)
    out2, same = gla.causal_conv_step(x, st, w, b)  # in place
    assert same is st and torch.equal(st, new) and torch.equal(out2, out)


def test_conv_prompt_then_tokens():
    """A prompt and then single tokens give the longer prompt's outputs (bit for bit: the same sums)."""
    g = _gen(5)
    B, T, E, W, cut = 2, 23, 48, 4, 20
    x = _randn(g, B, T, E).half()
    w, b = _randn(g, E, W) / 2, 0.1 * _randn(g, E)
    whole, fs = gla.causal_conv(x, w, b, 1, T, final_state=True)
    _, st = gla.causal_conv(x[:, :cut].contiguous(), w, b, 1, cut, final_state=True)
    for t in range(cut, T):
        out, st = gla.causal_conv_step(x[:, t], st, w, b)
        assert torch.equal(out, whole[:, t])
    assert torch.equal(st, fs)


# ------------------------------------------------------------------ scan

def _scan_inputs(seed, B, T, E, N, dtype, slices=False):
    g, dt = _gen(seed), TORCH_DT[dtype]
    s = {"A": -torch.exp(_randn(g, E, N)), "D": _randn(g, E), "delta_bias": -3 + _randn(g, E)}
    if slices:  # one projection's output, cut at offsets that no vector divides
        p = _randn(g, B, T, 3 * E + 2 * N + 5).to(dt)
        s["x"], s["z"], s["delta"] = p[..., 1:E + 1], p[..., E + 1:2 * E + 1], p[..., 2 * E + 1:3 * E + 1]
        s["Bm"], s["C"] = p[..., 3 * E + 2:3 * E + 2 + N], p[..., 3 * E + 3 + N:3 * E + 3 + 2 * N]
    else:
        for n, w in (("x", E), ("z", E), ("delta", E), ("Bm", N), ("C", N)):
            s[n] = _randn(g, B, T, w).to(dt)
    s["init"] = _randn(g, B, E, N)
    return s


def _scan64(s, tok, init, D, z, bias, softplus):
    x, A = s["x"].double()[:, tok], s["A"].double()
    Bm, C = s["Bm"].double()[:, tok], s["C"].double()[:, tok]
    v = s["delta"].double()[:, tok] + (0 if bias is None else bias.double())
    dt = torch.nn.functional.softplus(v, threshold=1e9) if softplus else v
    e_dt = 2.0 ** -19 if softplus else 2.0 ** -23
    B, T, E = x.shape
    h = torch.zeros(B, E, A.shape[1], dtype=torch.float64, device="cuda") if init is None else init.double()
    mag, err = h.abs(), torch.zeros_like(h)
    y, bnd = torch.empty_like(x), torch.empty_like(x)
    for t in range(T):
        arg = dt[:, t, :, None] * A
        a = torch.exp(arg)
        b = (dt[:, t] * x[:, t])[..., None] * Bm[:, t, None, :]
        eps = 4 * (2.0 ** -22 + arg.abs() * (e_dt + 2.0 ** -22))
        err = a * (err + eps * mag) + (e_dt + 4 * U32) * b.abs() + U32 * (a * mag)
        h, mag = a * h + b, a * mag + b.abs()
        y[:, t] = (h * C[:, t, None, :]).sum(-1)
        bnd[:, t] = (C[:, t, None, :].abs() * (err + (A.shape[1] + 4) * U32 * mag)).sum(-1)
    if D is not None:
        y = y + D.double() * x
        bnd = bnd + 4 * U32 * (D.double() * x).abs()
    bnd = bnd + 4 * U32 * y.abs()
    if z is not None:
        zz = z.double()[:, tok]
        gate = zz * torch.sigmoid(zz)
        bnd = bnd * gate.abs() + 2.0 ** -20 * (y * gate).abs()
        y = y * gate
    out, ob = torch.empty_like(y), torch.empty_like(y)
    out[:, tok], ob[:, tok] = y, bnd
    return out, ob, h, err + 4 * U32 * mag


SCAN = [  # B, grid_h, grid_w, E, N
    (1, 1, 1, 1, 1), (2, 1, 1, 40, 16), (1, 1, 15, 8, 16), (1, 1, 16, 8, 16), (1, 1, 17, 9, 16), (2, 5, 7, 24, 8), (1, 3, 33, 33, 5),
    (2, 9, 4, 40, 32), (1, 13, 9, 20, 64), (1, 6, 6, 12, 33), (1, 40, 40, 24, 16), (3, 8, 8, 100, 12), (1, 1, 700, 1, 16),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("case", SCAN, ids=lambda c: "x".join(map(str, c)))
def test_scan(case, dtype):
    B, gh, gw, E, N = case
    s = _scan_inputs(sum(case), B, gh * gw, E, N, dtype, slices=E % 2 == 1)
    for order in range(4):
        full = order % 2 == 0
        init, D, z, bias = (None, s["D"], s["z"], s["delta_bias"]) if full else (s["init"], None, None, None)
        out, check = guarded((B, gh * gw, E), s["x"].dtype)
        fs, check_fs = guarded((B, E, N), torch.float32)
        gla.ssm_scan(s["x"], s["delta"], s["A"], s["Bm"], s["C"], gh, gw, order, D=D, z=z, delta_bias=bias,
                     initial_state=init, final_state=fs, out=out)
        check("scan")
        check_fs("scan state")
        tok = scan_tokens(gh, gw, order)
        ref, bound, state, sb = _scan64(s, tok, init, D, z, bias, True)
        assert_close(out, ref, bound, f"scan {case} {dtype} order {order}")
        assert_close(fs, state, sb, f"scan state {case} {dtype} order {order}")


@pytest.mark.parametrize("E", [8, 600, 5000])
def test_scan_split_and_whole(E):
    """Launches of few and of many channels (segments a CTA folds, whole sequences): the same values."""
    s = _scan_inputs(E, 1, 150, E, 16, "f32")
    ref, bound, state, sb = _scan64(s, scan_tokens(1, 150, 0), None, s["D"], s["z"], s["delta_bias"], True)
    out, fs = gla.ssm_scan(s["x"], s["delta"], s["A"], s["Bm"], s["C"], 1, 150, D=s["D"], z=s["z"], delta_bias=s["delta_bias"])
    assert_close(out, ref, bound, "scan")
    assert_close(fs, state, sb, "scan state")
    again, fs2 = gla.ssm_scan(s["x"], s["delta"], s["A"], s["Bm"], s["C"], 1, 150, D=s["D"], z=s["z"],
                              delta_bias=s["delta_bias"])
    assert torch.equal(out, again) and torch.equal(fs, fs2)
    nofs, none = gla.ssm_scan(s["x"], s["delta"], s["A"], s["Bm"], s["C"], 1, 150, D=s["D"], z=s["z"],
                              delta_bias=s["delta_bias"], final_state=None)
    assert none is None and torch.equal(nofs, out)


def test_scan_steps_given():
    """softplus off: the steps are taken as they come, zero among them (the state stands still)."""
    s = _scan_inputs(9, 2, 40, 16, 16, "f32")
    s["delta"] = s["delta"].abs() * 0.1
    s["delta"][:, 5:9] = 0.0
    ref, bound, state, sb = _scan64(s, scan_tokens(5, 8, 2), None, None, None, None, False)
    out, fs = gla.ssm_scan(s["x"], s["delta"], s["A"], s["Bm"], s["C"], 5, 8, 2, softplus=False)
    assert_close(out, ref, bound, "scan, steps given")
    assert_close(fs, state, sb, "state, steps given")


def test_scan_extremes():
    """Steps that forget everything, steps of nearly nothing, gates at both ends; one channel's NaN stays its own."""
    s = _scan_inputs(10, 1, 64, 16, 16, "f32")
    s["delta_bias"][0], s["delta_bias"][1] = 80.0, -60.0
    s["z"][0, :, 2], s["z"][0, :, 3] = 200.0, -200.0
    args = (s["A"], s["Bm"], s["C"], 8, 8, 1)
    out, fs = gla.ssm_scan(s["x"], s["delta"], *args, D=s["D"], z=s["z"], delta_bias=s["delta_bias"])
    ref, bound, state, sb = _scan64(s, scan_tokens(8, 8, 1), None, s["D"], s["z"], s["delta_bias"], True)
    keep = [c for c in range(16) if c > 1]
    assert_close(out[..., keep], ref[..., keep], bound[..., keep], "scan, gates")
    # dt = 80: exact to 2^-19 of it, decays vanish; dt = e^-60: the library's exponential is off by 72 steps
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(fs).all())
    assert float((out[..., :2].double() - ref[..., :2]).abs().max()) <= 2.0 ** -15 * float(ref[..., :2].abs().max())
    x2 = s["x"].clone()
    x2[0, 20, 5] = float("nan")
    bad, _ = gla.ssm_scan(x2, s["delta"], *args, D=s["D"], z=s["z"], delta_bias=s["delta_bias"])
    other = [c for c in range(16) if c != 5]
    assert torch.equal(bad[..., other], out[..., other]) and bool(bad[..., 5].isnan().any())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,E,N", [(1, 1, 1), (2, 40, 16), (3, 65, 4), (2, 33, 8), (5, 12, 32), (2, 7, 64), (2, 50, 12), (300, 24, 16)])
def test_step(B, E, N, dtype):
    s = _scan_inputs(B + E + N, B, 1, E, N, dtype, slices=True)
    one = {n: (t[:, 0] if n in ("x", "z", "delta", "Bm", "C") else t) for n, t in s.items()}
    ref, bound, state, sb = _scan64(s, torch.zeros(1, dtype=torch.long, device="cuda"), s["init"], s["D"], s["z"],
                                    s["delta_bias"], True)
    st = s["init"].clone()
    kw = dict(D=s["D"], z=one["z"], delta_bias=s["delta_bias"])
    out, new = gla.ssm_step(one["x"], one["delta"], s["A"], one["Bm"], one["C"], st, state_out=torch.empty_like(st), **kw)
    assert_close(out, ref[:, 0], bound[:, 0], "step")
    assert_close(new, state, sb, "step state")
    assert torch.equal(st, s["init"])
    out2, same = gla.ssm_step(one["x"], one["delta"], s["A"], one["Bm"], one["C"], st, **kw)
    assert same is st and torch.equal(st, new) and torch.equal(out2, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_tokens(dtype):
    """A prompt's state and single tokens after it follow the longer prompt (to the bounds of both)."""
    T, cut, E, N = 61, 50, 72, 16
    s = _scan_inputs(77, 2, T, E, N, dtype)
    kw = dict(D=s["D"], delta_bias=s["delta_bias"])
    ref, bound, state, sb = _scan64(s, scan_tokens(1, T, 0), None, s["D"], s["z"], s["delta_bias"], True)
    part = {n: s[n][:, :cut].contiguous() for n in ("x", "delta", "z", "Bm", "C")}
    _, st = gla.ssm_scan(part["x"], part["delta"], s["A"], part["Bm"], part["C"], 1, cut, z=part["z"], **kw)
    for t in range(cut, T):
        out, st = gla.ssm_step(s["x"][:, t], s["delta"][:, t], s["A"], s["Bm"][:, t], s["C"][:, t], st, z=s["z"][:, t], **kw)
        assert_close(out, ref[:, t], bound[:, t], f"token {t}")
    assert_close(st, state, sb, "state after the tokens")


def test_refusals():
    s = _scan_inputs(1, 1, 16, 8, 16, "f32")
    ok = (s["x"], s["delta"], s["A"], s["Bm"], s["C"], 4, 4)
    with pytest.raises(ValueError):
        gla.ssm_scan(*ok[:5], 4, 5)
    with pytest.raises(ValueError):
        gla.ssm_scan(s["x"], s["delta"].half(), *ok[2:])
    with pytest.raises(ValueError):
        gla.ssm_scan(s["x"], s["delta"], s["A"].t(), *ok[3:])
    with pytest.raises(ValueError):
        gla.ssm_scan(*ok, z=s["z"][:, :, :4])
    with pytest.raises(gla.GLAError):
        gla.ssm_scan(*ok, out=s["x"])
    with pytest.raises(gla.GLAError):
        gla.ssm_scan(*ok, order=4)
    big = torch.zeros(8, 65, device="cuda")
    b65 = torch.zeros(1, 16, 65, device="cuda")
    with pytest.raises(gla.GLAError):
        gla.ssm_scan(s["x"], s["delta"], big, b65, b65, 4, 4)
    with pytest.raises(gla.GLAError):
        gla.causal_conv(s["x"], torch.zeros(8, 5, device="cuda"), None, 4, 4)
    with pytest.raises(ValueError):
        gla.causal_conv(s["x"], torch.zeros(8, 4, device="cuda").half(), None, 4, 4)
    empty = torch.zeros(0, 16, 8, device="cuda")
    out, fs = gla.causal_conv(empty, torch.zeros(8, 4, device="cuda"), None, 4, 4, final_state=True)
    assert out.shape == (0, 16, 8) and fs.shape == (0, 3, 8)


def test_streams_and_graph():
    s = _scan_inputs(3, 2, 144, 48, 16, "bf16")
    w, b = torch.randn(48, 4, device="cuda", generator=_gen(4)), torch.zeros(48, device="cuda")

    def block(stream=None):
        u, cs = gla.causal_conv(s["x"], w, b, 12, 12, 3, final_state=True, stream=stream)
        y, hs = gla.ssm_scan(u, s["delta"], s["A"], s["Bm"], s["C"], 12, 12, 3, D=s["D"], z=s["z"], stream=stream)
        return u, cs, y, hs

    ref = block()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = block(st)
    st.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(ref, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = block()
    s["x"].copy_(torch.randn(2, 144, 48, device="cuda", generator=_gen(6)))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(block(), res))
