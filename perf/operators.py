"""The operators around a recurrent token mixer, as timed cases: their plain form and the framework's calls.

A pre-norm block normalises its tokens (``layernorm`` and its backward pass), mixes them (the short
causal convolution and the selective state-space scan along a scan order of the patch grid, for whole
sequences and for single tokens) and passes them through a gated feed-forward step
(``swiglu_ffn`` and its backward pass).  Sizes are the repository's own stride-16 patch grids of
640^2 and 1280^2 images, widths 192 and 384, expansions 4 and 6, and generic odd, long and wide ones.

``run`` computes a case by elementary torch operations in 32 bits when ``own`` is false, and calls
``paper_2609_26590_gb300.gla`` when it is true.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_ELEM = {"f32": 4, "f16": 2, "bf16": 2}
_EPS = 1e-5
_ROW_FWD, _ROW_REV, _COL_FWD, _COL_REV = 0, 1, 2, 3


def _case(name, c):
    return dict(c, name=name) if name else c


def _ln(name, op, dtype, rows, D):
    return _case(name, {"op": op, "dtype": dtype, "rows": rows, "D": D})


def _ffn(name, op, dtype, M, D, F):
    return _case(name, {"op": op, "dtype": dtype, "M": M, "D": D, "F": F})


def _conv(name, dtype, B, grid_h, grid_w, E, W, order):
    return _case(name, {"op": "conv", "dtype": dtype, "B": B, "grid_h": grid_h, "grid_w": grid_w, "E": E, "W": W,
                        "order": order})


def _conv_step(name, dtype, B, E, W):
    return _case(name, {"op": "conv_step", "dtype": dtype, "B": B, "E": E, "W": W})


def _ssm(name, dtype, B, grid_h, grid_w, E, N, order):
    return _case(name, {"op": "ssm", "dtype": dtype, "B": B, "grid_h": grid_h, "grid_w": grid_w, "E": E, "N": N,
                        "order": order})


def _ssm_step(name, dtype, B, E, N):
    return _case(name, {"op": "ssm_step", "dtype": dtype, "B": B, "E": E, "N": N})


def listed():
    return [
        # one 640^2 image's tokens before a small model's mixer (serving latency)
        _ln("layernorm_b1_640_f16", "ln", "f16", 1600, 192),
        # a training batch of 640^2 images, the large model's width: gradients of tokens, weight and bias
        _ln("layernorm_bwd_b32_640_bf16", "ln_bwd", "bf16", 51200, 384),
        # full precision at a width and a row count that no vector or tile divides (evaluation, gradients)
        _ln("layernorm_bwd_odd_f32", "ln_bwd", "f32", 4099, 1001),
        # a batch of 640^2 images through the large model's feed-forward step (throughput inference)
        _ffn("ffn_b32_640_bf16", "ffn", "bf16", 51200, 384, 1536),
        # one token of a wide model: the weights are what has to be read (serving latency)
        _ffn("ffn_token_f16", "ffn", "f16", 1, 2048, 5632),
        # the gradients of a training batch in the widest vision model, a ragged number of tokens
        _ffn("ffn_bwd_b8_640_f16", "ffn_bwd", "f16", 12797, 384, 2304),
        # the gradients of a wide model's feed-forward step over long sequences
        _ffn("ffn_bwd_wide_bf16", "ffn_bwd", "bf16", 8192, 2048, 5632),
        # the batch of 640^2 images through the convolution before the scan, in a column order
        _conv("conv_b32_640_bf16", "bf16", 32, 40, 40, 768, 4, _COL_REV),
        # one token of each of 256 sequences being generated (convolution)
        _conv_step("conv_step_b256_f16", "f16", 256, 1536, 4),
        # one 640^2 image through a small model's scan: one sequence, few channels (latency)
        _ssm("ssm_b1_640_f16", "f16", 1, 40, 40, 384, 16, _COL_FWD),
        # 1280^2 images (6,400 tokens) through the large model's scan
        _ssm("ssm_b8_1280_bf16", "bf16", 8, 80, 80, 768, 16, _ROW_REV),
        # one token of each of 256 sequences being generated (scan; states are what has to be moved)
        _ssm_step("ssm_step_b256_bf16", "bf16", 256, 1536, 16),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ones' ranges; costs no more than the largest of them."""
    kind = rng.choice(["ln", "ln_bwd", "ffn", "ffn", "ffn_bwd", "ffn_bwd", "conv", "conv_step", "ssm", "ssm", "ssm",
                       "ssm_step"])
    dtype = rng.choice(["f16", "bf16"]) if kind.startswith("ffn") else rng.choice(["f16", "bf16", "f32"])
    while True:
        if kind in ("ln", "ln_bwd"):
            c = _ln(None, kind, dtype, _log_int(rng, 1, 51200), _log_int(rng, 64, 8192))
            if work(c)["bytes"] <= 3e8:
                return c
        elif kind in ("ffn", "ffn_bwd"):
            c = _ffn(None, kind, dtype, _log_int(rng, 1, 51200), 8 * _log_int(rng, 8, 256), 8 * _log_int(rng, 8, 704))
            if work(c)["flops"] <= (4e11 if kind == "ffn" else 1.1e12) and work(c)["bytes"] <= 6e8:
                return c
        elif kind == "conv":
            c = _conv(None, dtype, _log_int(rng, 1, 32), _log_int(rng, 1, 128), _log_int(rng, 1, 128),
                      _log_int(rng, 48, 2048), rng.choice([2, 3, 4, 4]), rng.randrange(4))
            if work(c)["bytes"] <= 3e8:
                return c
        elif kind == "conv_step":
            return _conv_step(None, dtype, _log_int(rng, 1, 512), _log_int(rng, 48, 4096), rng.choice([2, 3, 4, 4]))
        elif kind == "ssm":
            c = _ssm(None, dtype, _log_int(rng, 1, 16), _log_int(rng, 1, 100), _log_int(rng, 1, 100),
                     _log_int(rng, 48, 2048), rng.choice([8, 16, 16, 16, 32]), rng.randrange(4))
            if work(c)["flops"] <= 4.5e9:
                return c
        else:
            return _ssm_step(None, dtype, _log_int(rng, 1, 256), _log_int(rng, 48, 2048), rng.choice([8, 16, 16, 16, 32]))


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, op = _DTYPES[case["dtype"]], case["op"]

    def randn(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    if op in ("ln", "ln_bwd"):
        n, D = case["rows"], case["D"]
        # a residual stream: channels of unlike scale, rows off centre
        x = (randn(n, D) * torch.exp(0.5 * randn(D)) + randn(n, 1)).to(dt)
        s = {"x": x, "weight": 1.0 + 0.1 * randn(D), "bias": 0.1 * randn(D)}
        if op == "ln_bwd":
            s["dy"] = randn(n, D).to(dt)
            x64 = x.double()  # what the forward pass left behind
            m = x64.mean(1)
            s["mean"] = m.float()
            s["rstd"] = torch.rsqrt((x64 - m[:, None]).square().mean(1) + _EPS).float()
        return s
    if op in ("ffn", "ffn_bwd"):
        M, D, F = case["M"], case["D"], case["F"]
        s = {"x": randn(M, D).to(dt), "w_gate": (randn(F, D) / math.sqrt(D)).to(dt),
             "w_value": (randn(F, D) / math.sqrt(D)).to(dt)}
        if op == "ffn_bwd":
            s["dout"] = randn(M, F).to(dt)
        return s
    B, E = case["B"], case["E"]
    if op in ("conv", "conv_step"):
        W = case["W"]
        s = {"weight": randn(E, W) / math.sqrt(W), "bias": 0.1 * randn(E)}
        if op == "conv":
            s["x"] = randn(B, case["grid_h"] * case["grid_w"], E).to(dt)
        else:
            s["x"], s["state"] = randn(B, E).to(dt), randn(B, W - 1, E).to(dt)
        return s
    N = case["N"]
    lead = (B, case["grid_h"] * case["grid_w"]) if op == "ssm" else (B,)
    s = {"A": -(torch.arange(1, N + 1, device="cuda").float() * torch.exp(0.1 * randn(E, N))), "D": 1.0 + 0.1 * randn(E)}
    # step sizes of 0.001 to 0.1 at rest, the usual start of such models
    u = torch.rand(E, device="cuda", generator=gen)
    step = torch.exp(u * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
    s["delta_bias"] = step + torch.log(-torch.expm1(-step))
    s["x"], s["z"] = randn(*lead, E).to(dt), randn(*lead, E).to(dt)
    s["delta"] = (0.5 * randn(*lead, E)).to(dt)
    s["Bm"], s["C"] = randn(*lead, N).to(dt), randn(*lead, N).to(dt)
    if op == "ssm_step":
        s["state"] = randn(B, E, N)
    return s


def prepare(case, seed):
    s = dict(case, x=_inputs(case, seed))
    if case["op"] in ("conv_step", "ssm_step"):
        s["new_state"] = torch.empty_like(s["x"]["state"])
    return s


def _tokens(T, grid_h, grid_w, order):
    """The spatial tokens in the order in which the scan visits them."""
    s = torch.arange(T, device="cuda")
    u = T - 1 - s if order in (_ROW_REV, _COL_REV) else s
    return u if order in (_ROW_FWD, _ROW_REV) else (u % grid_h) * grid_w + u // grid_h


def _softplus(t):
    return t.clamp(min=0) + torch.log1p(torch.exp(-t.abs()))


def _silu(t):
    return t / (1.0 + torch.exp(-t))


def _plain_ffn_bwd(x, dt):
    a, wg, wv, dh = (x[n].float() for n in ("x", "w_gate", "w_value", "dout"))
    g, v = a @ wg.t(), a @ wv.t()
    sg = 1.0 / (1.0 + torch.exp(-g))
    dv = dh * g * sg
    dg = dh * v * sg * (1.0 + g * (1.0 - sg))
    return (dg @ wg + dv @ wv).to(dt), (dg.t() @ a).to(dt), (dv.t() @ a).to(dt)


def _plain_ssm(s, dt):
    x, T = s["x"], s["grid_h"] * s["grid_w"]
    tok = _tokens(T, s["grid_h"], s["grid_w"], s["order"])
    u = x["x"].float()
    step = _softplus(x["delta"].float() + x["delta_bias"])
    Bm, C = x["Bm"].float(), x["C"].float()
    h = torch.zeros((s["B"], s["E"], s["N"]), device="cuda")
    y = torch.empty_like(u)
    L = 16
    for t0 in range(0, T, L):
        t = tok[t0:t0 + L]
        st = step[:, t]
        a = torch.exp(st.unsqueeze(-1) * x["A"])
        b = (st * u[:, t]).unsqueeze(-1) * Bm[:, t].unsqueeze(2)
        hs = []
        for i in range(t.numel()):
            h = a[:, i] * h + b[:, i]
            hs.append(h)
        y[:, t] = (torch.stack(hs, 1) * C[:, t].unsqueeze(2)).sum(-1)
    return ((y + x["D"] * u) * _silu(x["z"].float())).to(dt), h


def _plain(s):
    x, op, dt = s["x"], s["op"], _DTYPES[s["dtype"]]
    if op == "ln":
        a = x["x"].float()
        c = a - a.mean(1, keepdim=True)
        return (c * torch.rsqrt(c.square().mean(1, keepdim=True) + _EPS) * x["weight"] + x["bias"]).to(dt)
    if op == "ln_bwd":
        rstd, dy = x["rstd"][:, None], x["dy"].float()
        xh = (x["x"].float() - x["mean"][:, None]) * rstd
        d = dy * x["weight"]
        dx = rstd * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
        return dx.to(dt), (dy * xh).sum(0), dy.sum(0)
    if op == "ffn":
        a = x["x"].float()
        return (_silu(a @ x["w_gate"].float().t()) * (a @ x["w_value"].float().t())).to(dt)
    if op == "ffn_bwd":
        return _plain_ffn_bwd(x, dt)
    if op == "conv":
        W, T = s["W"], s["grid_h"] * s["grid_w"]
        tok = _tokens(T, s["grid_h"], s["grid_w"], s["order"])
        a = torch.cat([torch.zeros((s["B"], W - 1, s["E"]), device="cuda"), x["x"].float()[:, tok]], 1)
        acc = x["bias"] + sum(x["weight"][:, j] * a[:, j:j + T] for j in range(W))
        out = torch.empty_like(acc)
        out[:, tok] = _silu(acc)
        return out.to(dt), a[:, T:].to(dt)
    if op == "conv_step":
        a = torch.cat([x["state"], x["x"][:, None]], 1)
        acc = x["bias"] + (x["weight"].t() * a.float()).sum(1)
        return _silu(acc).to(dt), a[:, 1:]
    if op == "ssm":
        return _plain_ssm(s, dt)
    u = x["x"].float()
    step = _softplus(x["delta"].float() + x["delta_bias"])
    h = torch.exp(step.unsqueeze(-1) * x["A"]) * x["state"] + (step * u).unsqueeze(-1) * x["Bm"].float().unsqueeze(1)
    y = (h * x["C"].float().unsqueeze(1)).sum(-1) + x["D"] * u
    return (y * _silu(x["z"].float())).to(dt), h


def _own(s):
    from paper_2609_26590_gb300 import gla

    x, op = s["x"], s["op"]
    if op == "ln":
        return gla.layernorm(x["x"], x["weight"], x["bias"], _EPS)
    if op == "ln_bwd":
        return gla.layernorm_backward(x["dy"], x["x"], x["weight"], x["mean"], x["rstd"])
    if op == "ffn":
        return gla.swiglu_ffn(x["x"], x["w_gate"], x["w_value"])
    if op == "ffn_bwd":
        return gla.swiglu_ffn_backward(x["dout"], x["x"], x["w_gate"], x["w_value"])
    if op == "conv":
        return gla.causal_conv(x["x"], x["weight"], x["bias"], s["grid_h"], s["grid_w"], s["order"], final_state=True)
    if op == "conv_step":
        return gla.causal_conv_step(x["x"], x["state"], x["weight"], x["bias"], state_out=s["new_state"])
    if op == "ssm":
        return gla.ssm_scan(x["x"], x["delta"], x["A"], x["Bm"], x["C"], s["grid_h"], s["grid_w"], s["order"], D=x["D"],
                            z=x["z"], delta_bias=x["delta_bias"], final_state=True)
    return gla.ssm_step(x["x"], x["delta"], x["A"], x["Bm"], x["C"], x["state"], D=x["D"], z=x["z"],
                        delta_bias=x["delta_bias"], state_out=s["new_state"])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    es, op = _ELEM[case["dtype"]], case["op"]
    if op in ("ln", "ln_bwd"):
        n, D = case["rows"], case["D"]
        if op == "ln":
            return {"bytes": 2.0 * n * D * es + 8.0 * D, "flops": 8.0 * n * D}
        return {"bytes": 3.0 * n * D * es + 8.0 * n + 12.0 * D, "flops": 14.0 * n * D}
    if op in ("ffn", "ffn_bwd"):
        M, D, F = case["M"], case["D"], case["F"]
        if op == "ffn":
            return {"bytes": float(es * (M * D + 2 * F * D + M * F)), "flops": 4.0 * M * D * F + 6.0 * M * F}
        # both projections again, the tokens' gradient, the weights' gradients
        return {"bytes": float(es * (2 * M * D + 4 * F * D + M * F)), "flops": 12.0 * M * D * F + 14.0 * M * F}
    B, E = case["B"], case["E"]
    if op in ("conv", "conv_step"):
        W = case["W"]
        if op == "conv":
            n = B * case["grid_h"] * case["grid_w"]
            return {"bytes": float(es * (2 * n * E + B * (W - 1) * E) + 4 * E * (W + 1)), "flops": n * E * (2.0 * W + 4.0)}
        return {"bytes": float(es * B * E * 2 * W + 4 * E * (W + 1)), "flops": B * E * (2.0 * W + 4.0)}
    N = case["N"]
    if op == "ssm":
        n = B * case["grid_h"] * case["grid_w"]
        nbytes = es * n * (4 * E + 2 * N) + 4 * E * (N + 2) + 4 * B * E * N
    else:
        n = B
        nbytes = es * n * (4 * E + 2 * N) + 4 * E * (N + 2) + 8 * B * E * N
    # a token and state: the decay's product and power, the input's product, the state's and the readout's sums
    return {"bytes": float(nbytes), "flops": n * E * (7.0 * N + 16.0)}


def _exact_ssm(case, x):
    B, E, N, T = case["B"], case["E"], case["N"], case["grid_h"] * case["grid_w"]
    tok = _tokens(T, case["grid_h"], case["grid_w"], case["order"])
    step = torch.nn.functional.softplus(x["delta"] + x["delta_bias"], threshold=1e9)
    h = torch.zeros((B, E, N), dtype=torch.float64, device="cuda")
    y = torch.empty((B, T, E), dtype=torch.float64, device="cuda")
    # sum over the tokens s <= t of a block: C_t e^{A (c_t - c_s)} B_s step_s x_s, plus the state before it
    K = 8
    for t0 in range(0, T, K):
        t = tok[t0:t0 + K]
        n = t.numel()
        c = step[:, t].cumsum(1)
        w = step[:, t] * x["x"][:, t]
        Bt, Ct = x["Bm"][:, t], x["C"][:, t]
        for i in range(n):
            acc = torch.einsum("ben,bn->be", torch.exp(c[:, i].unsqueeze(-1) * x["A"]) * h, Ct[:, i])
            far = (c[:, i:i + 1] - c[:, :i + 1]).unsqueeze(-1) * x["A"]
            acc += torch.einsum("bsen,bsn,bse->be", torch.exp(far), Bt[:, :i + 1] * Ct[:, i:i + 1], w[:, :i + 1])
            y[:, t[i]] = acc
        last = (c[:, -1:] - c).unsqueeze(-1) * x["A"]
        h = torch.exp(c[:, -1].unsqueeze(-1) * x["A"]) * h + torch.einsum("bsen,bsn,bse->ben", torch.exp(last), Bt, w)
    return (y + x["D"] * x["x"]) * x["z"] * torch.sigmoid(x["z"]), h


def exact(case, seed):
    x = {n: t.double() for n, t in _inputs(case, seed).items()}
    op = case["op"]
    if op == "ln":
        var, mean = torch.var_mean(x["x"], dim=1, correction=0, keepdim=True)
        return (x["x"] - mean) / torch.sqrt(var + _EPS) * x["weight"] + x["bias"]
    if op == "ln_bwd":
        D = case["D"]
        xh = x["rstd"][:, None] * (x["x"] - x["mean"][:, None])
        g = x["dy"] * x["weight"]
        s1, s2 = g.sum(1, keepdim=True), (g * xh).sum(1, keepdim=True)
        return x["rstd"][:, None] * (g - (s1 + xh * s2) / D), torch.einsum("rd,rd->d", x["dy"], xh), x["dy"].sum(0)
    if op == "ffn":
        return torch.nn.functional.silu(torch.nn.functional.linear(x["x"], x["w_gate"])) * torch.nn.functional.linear(
            x["x"], x["w_value"])
    if op == "ffn_bwd":
        leaves = [x[n].requires_grad_() for n in ("x", "w_gate", "w_value")]
        h = torch.nn.functional.silu(torch.nn.functional.linear(x["x"], x["w_gate"])) * torch.nn.functional.linear(
            x["x"], x["w_value"])
        return torch.autograd.grad(h, leaves, x["dout"])
    if op == "conv":
        B, E, W, T = case["B"], case["E"], case["W"], case["grid_h"] * case["grid_w"]
        tok = _tokens(T, case["grid_h"], case["grid_w"], case["order"])
        a = torch.nn.functional.pad(x["x"][:, tok], (0, 0, W - 1, 0))
        acc = torch.einsum("btew,ew->bte", a.unfold(1, W, 1), x["weight"]) + x["bias"]
        out = torch.empty_like(acc)
        out[:, tok] = torch.nn.functional.silu(acc)
        return out, a[:, T:]
    if op == "conv_step":
        a = torch.cat([x["state"], x["x"][:, None]], 1)
        return torch.nn.functional.silu(torch.einsum("bwe,ew->be", a, x["weight"]) + x["bias"]), a[:, 1:]
    if op == "ssm":
        return _exact_ssm(case, x)
    step = torch.nn.functional.softplus(x["delta"] + x["delta_bias"], threshold=1e9)
    h = x["state"] * torch.exp(torch.einsum("be,en->ben", step, x["A"])) + torch.einsum("be,be,bn->ben", step, x["x"],
                                                                                       x["Bm"])
    return (torch.einsum("ben,bn->be", h, x["C"]) + x["D"] * x["x"]) * x["z"] * torch.sigmoid(x["z"]), h
