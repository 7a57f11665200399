"""The C ABI of the operators around the mixer refuses what its documentation excludes before anything is
launched (made-up addresses, no GPU), and its Python entry points refuse tensors that are not on a GPU."""
import pytest
import torch

from paper_2609_26590_gb300 import build as gbuild

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
K = 1 << 24  # addresses K, 2K, ...: 16 MB apart, never read


@pytest.fixture(scope="module")
def lib():
    gbuild.build()
    from paper_2609_26590_gb300 import gla
    return gla.load()


def _ln(lib, x=K, xs=64, w=2 * K, b=3 * K, eps=1e-5, n=4, D=64, dt=1, out=4 * K, mean=5 * K, rstd=6 * K):
    return lib.gtr_layernorm_fwd(x, xs, w, b, eps, n, D, dt, out, mean, rstd, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(out=None), dict(x=K + 8), dict(out=4 * K + 4), dict(w=2 * K + 2),
                                 dict(mean=5 * K + 1), dict(D=0), dict(D=16385, xs=16385), dict(n=-1), dict(xs=63),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(dt=3), dict(dt=-1),
                                 dict(out=K + 256), dict(mean=4 * K), dict(rstd=5 * K), dict(n=1 << 31),
                                 dict(n=1 << 29, xs=1 << 30)])
def test_layernorm_refuses(lib, bad):
    assert _ln(lib, **bad) == INVALID


def test_layernorm_empty(lib):
    assert _ln(lib, n=0, x=None, out=None) == 0
    assert lib.gtr_layernorm_bwd_workspace_bytes(0, 64) == 0
    assert lib.gtr_layernorm_bwd_workspace_bytes(5, 0) == 0
    assert lib.gtr_layernorm_bwd_workspace_bytes(5, 64) >= 2 * 64 * 4


def _lnb(lib, dy=K, ds=64, x=2 * K, xs=64, w=3 * K, mean=4 * K, rstd=5 * K, n=4, D=64, dt=1, dx=6 * K, dw=7 * K, db=8 * K,
         ws=9 * K, wb=1 << 20):
    return lib.gtr_layernorm_bwd(dy, ds, x, xs, w, mean, rstd, n, D, dt, dx, dw, db, ws, wb, None)


@pytest.mark.parametrize("bad,status", [(dict(dy=None), INVALID), (dict(mean=None), INVALID), (dict(rstd=None), INVALID),
                                        (dict(ds=10), INVALID), (dict(dx=2 * K), INVALID), (dict(dw=8 * K), INVALID),
                                        (dict(ws=9 * K + 16), INVALID), (dict(ws=None), WORKSPACE), (dict(wb=100), WORKSPACE),
                                        (dict(ws=2 * K), INVALID), (dict(dt=7), INVALID), (dict(db=8 * K + 2), INVALID)])
def test_layernorm_backward_refuses(lib, bad, status):
    assert _lnb(lib, **bad) == status


def _conv(lib, x=K, xs=64, w=2 * K, b=3 * K, silu=1, init=None, B=2, gh=4, gw=4, E=64, W=4, order=0, dt=1, out=4 * K,
          fs=5 * K):
    return lib.gtr_causal_conv_fwd(x, xs, w, b, silu, init, B, gh, gw, E, W, order, dt, out, fs, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(w=None), dict(out=None), dict(x=K + 2), dict(init=6 * K + 8),
                                 dict(fs=5 * K + 8), dict(W=1), dict(W=5), dict(E=0), dict(E=(1 << 20) + 1), dict(gh=0),
                                 dict(gw=-1), dict(B=-1), dict(order=4), dict(order=-1), dict(dt=3), dict(silu=2), dict(xs=60),
                                 dict(out=K), dict(fs=K), dict(fs=4 * K), dict(init=5 * K), dict(gh=1 << 16, gw=1 << 16),
                                 dict(gh=1 << 15, gw=1 << 15, B=1 << 20)])
def test_conv_refuses(lib, bad):
    assert _conv(lib, **bad) == INVALID


def test_conv_empty(lib):
    assert _conv(lib, B=0, x=None, out=None) == 0


def _cstep(lib, x=K, xs=64, st=2 * K, w=3 * K, b=None, silu=1, B=2, E=64, W=4, dt=1, out=4 * K, so=5 * K):
    return lib.gtr_causal_conv_step(x, xs, st, w, b, silu, B, E, W, dt, out, so, None)


@pytest.mark.parametrize("bad", [dict(st=None), dict(so=None), dict(so=2 * K + 256), dict(out=2 * K), dict(so=K), dict(W=9),
                                 dict(out=2 * K, so=2 * K)])
def test_conv_step_refuses(lib, bad):
    assert _cstep(lib, **bad) == INVALID


def _ssm(lib, x=K, xs=64, dl=2 * K, ds=64, A=3 * K, b=4 * K, bs=16, c=5 * K, cs=16, D=6 * K, z=7 * K, zs=64, bias=8 * K, sp=1,
         init=None, B=2, gh=4, gw=4, E=64, N=16, order=0, dt=1, out=9 * K, fs=10 * K):
    return lib.gtr_ssm_scan_fwd(x, xs, dl, ds, A, b, bs, c, cs, D, z, zs, bias, sp, init, B, gh, gw, E, N, order, dt, out, fs,
                                None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(dl=None), dict(A=None), dict(b=None), dict(c=None), dict(out=None),
                                 dict(x=K + 1), dict(A=3 * K + 4), dict(out=9 * K + 8), dict(fs=10 * K + 4), dict(D=6 * K + 2),
                                 dict(N=0), dict(N=65), dict(E=0), dict(xs=63), dict(ds=1), dict(zs=3), dict(bs=15), dict(cs=0),
                                 dict(sp=2), dict(order=5), dict(dt=4), dict(B=-3), dict(gh=0), dict(out=K), dict(fs=3 * K),
                                 dict(fs=9 * K), dict(init=10 * K), dict(gh=1 << 20, gw=1 << 20)])
def test_ssm_refuses(lib, bad):
    assert _ssm(lib, **bad) == INVALID


def test_ssm_empty_and_no_gate(lib):
    assert _ssm(lib, B=0, x=None, out=None) == 0
    assert _ssm(lib, B=0, z=None, zs=0) == 0  # no gate, no stride of it


def _sstep(lib, x=K, xs=64, dl=2 * K, ds=64, A=3 * K, b=4 * K, bs=16, c=5 * K, cs=16, D=None, z=None, zs=0, bias=None, sp=1,
           st=6 * K, B=2, E=64, N=16, dt=1, out=7 * K, so=8 * K):
    return lib.gtr_ssm_step(x, xs, dl, ds, A, b, bs, c, cs, D, z, zs, bias, sp, st, B, E, N, dt, out, so, None)


@pytest.mark.parametrize("bad", [dict(st=None), dict(so=None), dict(so=6 * K + 16), dict(out=6 * K), dict(so=3 * K),
                                 dict(out=6 * K, so=6 * K), dict(st=6 * K + 8), dict(N=70)])
def test_ssm_step_refuses(lib, bad):
    assert _sstep(lib, **bad) == INVALID


def _ffn(lib, x=K, xs=64, wg=2 * K, wv=3 * K, M=4, D=64, F=128, dt=1, out=4 * K):
    return lib.gtr_swiglu_ffn_fwd(x, xs, wg, wv, M, D, F, dt, out, None)


@pytest.mark.parametrize("bad,status", [(dict(x=None), INVALID), (dict(wg=None), INVALID), (dict(wv=3 * K + 8), INVALID),
                                        (dict(D=60), INVALID), (dict(F=12), INVALID), (dict(D=0), INVALID), (dict(xs=68), INVALID),
                                        (dict(xs=56), INVALID), (dict(M=-1), INVALID), (dict(dt=5), INVALID), (dict(out=K), INVALID),
                                        (dict(out=3 * K), INVALID), (dict(dt=0), UNSUPPORTED), (dict(M=1 << 31), INVALID),
                                        (dict(M=1 << 30, F=1 << 20), INVALID)])
def test_ffn_refuses(lib, bad, status):
    assert _ffn(lib, **bad) == status


def _ffnb(lib, do=K, ds=128, x=2 * K, xs=64, wg=3 * K, wv=4 * K, M=4, D=64, F=128, dt=1, dx=5 * K, dg=6 * K, dv=7 * K,
          ws=8 * K, wb=None):
    if wb is None:
        wb = lib.gtr_swiglu_ffn_bwd_workspace_bytes(M, D, F)
    return lib.gtr_swiglu_ffn_bwd(do, ds, x, xs, wg, wv, M, D, F, dt, dx, dg, dv, ws, wb, None)


@pytest.mark.parametrize("bad,status", [(dict(do=None), INVALID), (dict(dx=None), INVALID), (dict(dg=None), INVALID),
                                        (dict(ds=120), INVALID), (dict(ds=132), INVALID), (dict(dx=2 * K), INVALID),
                                        (dict(dg=7 * K), INVALID), (dict(ws=8 * K + 128), INVALID), (dict(ws=None), WORKSPACE),
                                        (dict(wb=64), WORKSPACE), (dict(ws=5 * K), INVALID), (dict(dt=0), UNSUPPORTED)])
def test_ffn_backward_refuses(lib, bad, status):
    assert _ffnb(lib, **bad) == status


def test_ffn_empty(lib):
    assert _ffn(lib, M=0, x=None, out=None) == 0
    assert lib.gtr_swiglu_ffn_bwd_workspace_bytes(4, 60, 128) == 0
    assert lib.gtr_swiglu_ffn_bwd_workspace_bytes(4, 64, 128) >= 2 * 4 * 128 * 2


def test_python_entry_points_refuse_cpu_tensors(lib):
    from paper_2609_26590_gb300 import gla
    x, w = torch.zeros(4, 64), torch.ones(64)
    s = torch.zeros(1, 4, 64)
    h = torch.zeros(4, 64, dtype=torch.float16)
    wg = torch.zeros(16, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        gla.layernorm(x, w, w, 1e-5)
    with pytest.raises(ValueError):
        gla.layernorm_backward(x, x, w, torch.zeros(4), torch.zeros(4))
    with pytest.raises(ValueError):
        gla.causal_conv(s, torch.zeros(64, 4), None, 2, 2)
    with pytest.raises(ValueError):
        gla.causal_conv_step(x, torch.zeros(4, 3, 64), torch.zeros(64, 4), None)
    with pytest.raises(ValueError):
        gla.ssm_scan(s, s, torch.zeros(64, 16), torch.zeros(1, 4, 16), torch.zeros(1, 4, 16), 2, 2)
    with pytest.raises(ValueError):
        gla.ssm_step(x, x, torch.zeros(64, 16), torch.zeros(4, 16), torch.zeros(4, 16), torch.zeros(4, 64, 16))
    with pytest.raises(ValueError):
        gla.swiglu_ffn(h, wg, wg)
    with pytest.raises(ValueError):
        gla.swiglu_ffn_backward(h[:, :16], h, wg, wg)
    with pytest.raises(gla.GLAError) as e:
        gla.swiglu_ffn(x, torch.zeros(16, 64), torch.zeros(16, 64))
    assert e.value.status == UNSUPPORTED
    with pytest.raises(ValueError):
        gla.layernorm(torch.zeros(4, 64, dtype=torch.float64), w, w, 1e-5)


def test_row_strides():
    from paper_2609_26590_gb300.gla import _row_stride
    t = torch.zeros(2, 3, 40)
    assert _row_stride(t, "t") == 40
    assert _row_stride(t[:, :, 8:24], "t") == 40
    assert _row_stride(t[:1, :1, 8:24], "t") == 16        # one token: the stride says nothing
    assert _row_stride(t[:, :1], "t") == 120
    for bad in (t[:, :2], t.transpose(0, 1), t[:, :, ::2], torch.zeros(1, 40).expand(3, 40), t.transpose(1, 2)):
        with pytest.raises(ValueError):
            _row_stride(bad, "t")
    assert _row_stride(torch.zeros(5, 1), "t") == 1
    assert _row_stride(torch.zeros(0, 7), "t") == 7


@pytest.mark.parametrize("E,N,per", [(8, 16, 32), (16, 32, 16), (8, 64, 8), (33, 16, 32)])
def test_ssm_refuses_more_groups_than_documented(lib, E, N, per):
    far = 1 << 44  # nothing overlaps
    groups = -(-E // per)
    B = (1 << 27) // groups + 1
    assert _ssm(lib, x=far, dl=2 * far, A=3 * far, b=4 * far, c=5 * far, D=None, z=None, bias=None, out=6 * far, fs=None,
                xs=E, ds=E, bs=N, cs=N, B=B, gh=1, gw=1, E=E, N=N) == INVALID
