"""The gated feed-forward step's backward pass deals every block of its sums exactly once (host arithmetic, no GPU),
and the sizes that tests/test_gpu_ffn.py runs cover each way of dealing them."""
import random

import pytest

from paper_2609_26590_gb300 import build as gbuild

GB300_SMS = 152


@pytest.fixture(scope="module")
def gla():
    gbuild.build()
    from paper_2609_26590_gb300 import gla
    gla.load()
    return gla


def _tiles(n, size):
    return (n + size - 1) // size


def _check(gla, M, D, F, n_sm):
    columns, cut, w, x = gla.swiglu_ffn_backward_plan(M, D, F, n_sm)
    what = (M, D, F, n_sm, columns, cut)
    assert columns in (128, 256, 384, 512) and (columns == 128 or columns < D + 128), what
    assert len(w) == min(n_sm // 2, 128) + 1, what
    tn = _tiles(D, columns)
    w_nk, x_nk = _tiles(M, 64), 2 * _tiles(F, 64)
    w_all, x_all = 2 * _tiles(F, 256) * tn * w_nk, _tiles(M, 256) * tn * x_nk
    for start, total, nk, is_cut in ((w, w_all, w_nk, cut >= 1), (x, x_all if cut == 2 else 0, x_nk, cut == 2)):
        assert start[0] == 0 and start[-1] == total, what
        for a, b in zip(start, start[1:]):
            assert a <= b, what
            # whole tiles, or cuts that leave at least eight blocks at a tile's ends
            assert b % nk == 0 or (is_cut and b % nk >= 8 and nk - b % nk >= 8), what
    return columns, cut, w_all + x_all, max((b - a) + (d - c) for a, b, c, d in zip(w, w[1:], x, x[1:]))


def test_plan_covers_every_block_once(gla):
    rng = random.Random(7)
    for _ in range(4000):
        M = int(2 ** rng.uniform(0, 20))
        D, F = 8 * int(2 ** rng.uniform(0, 9)), 8 * int(2 ** rng.uniform(0, 10))
        _check(gla, M, D, F, rng.choice([2, 3, 16, 132, 148, GB300_SMS, GB300_SMS, 264, 400]))


def test_plan_evens_out(gla):
    # few tokens: dx's one tile column of long sums is spread over the pairs
    columns, cut, total, most = _check(gla, 72, 72, 2528, GB300_SMS)
    assert cut == 2 and most <= 12
    # a training batch of narrow tokens: dW's sums over 12,797 tokens are cut, no pair has 1.2 times its share
    columns, cut, _, _ = _check(gla, 12797, 384, 2304, GB300_SMS)
    assert columns == 384 and cut == 1
    # a wide model: whole tiles fit the pairs
    columns, cut, _, _ = _check(gla, 8192, 2048, 5632, GB300_SMS)
    assert columns == 512 and cut == 0


def test_gpu_sizes_cover_the_plan(gla):
    from test_gpu_ffn import SHAPES
    seen = {gla.swiglu_ffn_backward_plan(M, D, F, GB300_SMS)[:2] for M, D, F in SHAPES}
    assert {c for c, _ in seen} == {128, 256, 384, 512}
    assert {k for _, k in seen} == {0, 1, 2}


def test_plan_refuses(gla):
    for bad in ((0, 64, 64, 152), (4, 60, 64, 152), (4, 64, 4, 152), (4, 64, 64, 1), (-1, 64, 64, 152)):
        with pytest.raises(ValueError):
            gla.swiglu_ffn_backward_plan(*bad)


def test_limits_of_a_stride(gla):
    lib = gla.load()
    K = 1 << 24
    assert lib.gtr_swiglu_ffn_fwd(K, 1 << 39, 2 * K, 3 * K, 1, 64, 128, 1, 4 * K, None) == 1
    assert lib.gtr_swiglu_ffn_bwd(K, 1 << 39, 2 * K, 64, 3 * K, 4 * K, 1, 64, 128, 1, 5 * K, 6 * K, 7 * K, 8 * K, 1 << 30, None) == 1
