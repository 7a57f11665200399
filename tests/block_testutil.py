"""Helpers of the tests of the operators around the mixer: half a step of rounding per type, and an
elementwise comparison against 64-bit values with a bound per element."""
import torch

TORCH_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                 # half a step of fp32


def half_step(dtype: torch.dtype) -> float:
    """The largest relative error of one rounding to `dtype`."""
    return torch.finfo(dtype).eps / 2


def assert_close(got: torch.Tensor, ref: torch.Tensor, bound, what: str):
    """|got - ref| <= one rounding of ref to got's type plus `bound` (the error before that rounding).
    The rounding of a value whose error is `bound` is off by half a step of both; below the normal
    range of fp16 a step is 2^-24 whatever the value; what lies below fp32's normal range (bf16's too)
    may be flushed to zero."""
    u = half_step(got.dtype)
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 2.0 ** -126
    assert got.shape == ref.shape, f"{what}: shape {tuple(got.shape)} != {tuple(ref.shape)}"
    err = (got.double() - ref).abs()
    limit = u * (ref.abs() + bound) + bound + tiny
    bad = ~(err <= limit)
    if bad.any():
        i = int(torch.argmax(torch.where(bad, err - limit, torch.zeros_like(err) - 1).nan_to_num(nan=1e30).flatten()))
        at = tuple(int(k) for k in torch.unravel_index(torch.tensor(i), err.shape))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} elements off, the worst at {at}: got "
                             f"{float(got[at])}, want {float(ref[at])}, error {float(err[at]):.3g} > {float(limit[at] if limit.dim() else limit):.3g}")


def rel_l2(got: torch.Tensor, ref: torch.Tensor) -> float:
    return float((got.double() - ref).norm() / ref.norm().clamp(min=1e-300))


def scan_tokens(grid_h: int, grid_w: int, order: int) -> torch.Tensor:
    """Tokens in the order the scan visits them, walked position by position."""
    walk = []
    if order < 2:
        for y in range(grid_h):
            for x in range(grid_w):
                walk.append(y * grid_w + x)
    else:
        for x in range(grid_w):
            for y in range(grid_h):
                walk.append(y * grid_w + x)
    if order & 1:
        walk.reverse()
    return torch.tensor(walk, device="cuda")


def guarded(shape, dtype, fill=None):
    """A tensor of `shape` inside a larger buffer whose elements around it hold a pattern; returns the
    tensor and a check that the pattern is still there."""
    n = 1
    for s in shape:
        n *= s
    pad = 1024
    buf = torch.full((n + 2 * pad,), 7.0, dtype=dtype, device="cuda")
    t = buf[pad:pad + n].view(shape)
    t.fill_(float("nan") if fill is None else fill)

    def check(what):
        assert bool((buf[:pad] == 7.0).all()) and bool((buf[pad + n:] == 7.0).all()), f"{what}: written outside"

    return t, check
