"""Attention whose scores are large, or all but nothing (GPU)."""
import numpy as np
import pytest
import torch

import cache_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from test_gpu_cache import f64, put, rng_rows

pytestmark = pytest.mark.gpu


def pages_of(k, v, d):
    """One unit's rows [n, d] in pages: pool and table."""
    pages = -(-len(k) // 64)
    pool = tk.cache_pool(pages, d, device())
    table = put(np.arange(pages, dtype=np.int32).reshape(1, 1, pages))
    shape = (1, 1, len(k), d)
    out = tk.twinkv_cache_pack(k.view(shape).to(device()), v.view(shape).to(device()), None, pool,
                               table)
    assert out["status"].eq(0).all()
    return pool, table, out["lens"]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 8, 16])
@pytest.mark.parametrize("length", [2, 64, 200, 60000])
@pytest.mark.parametrize("e", [10, 30, 100])
def test_one_key_far_above_the_others(d, G, length, e):
    """Keys are multiples of one direction, the top one's twice the next: scores differ by
    d^0.5 2^(e - 1) and more, so that the output is the value of the top slot, rounded as a product
    (2^-11) and as an output (2^-8).  Even rows see positive scores, odd ones negative, where the
    smallest multiple is on top.  The denominator's logarithm is the score: a row's at most eight products
    of 16 values are float32 sums, off by 2^-21 of at most four times its size each."""
    rng = np.random.default_rng([d, G, length, e])
    u = rng.choice([-1.0, 1.0], d)
    level = rng.uniform(0.3, 0.5, length)
    most, least = rng.choice(length, 2, replace=False)
    level[most], level[least] = 1.0, 0.15
    k = torch.from_numpy(np.ldexp(level[:, None] * u, e)).to(torch.bfloat16)
    v = rng_rows(rng, length, d)
    sign = np.where(np.arange(G) % 2, -1.0, 1.0)
    q = torch.from_numpy(sign[:, None] * u).to(torch.bfloat16)
    pool, table, lens = pages_of(k, v, d)
    got = tk.twinkv_cache_attend(q.view(1, 1, G, d).to(device()), pool, table, lens, want_lse=True)
    want = R.round_trip(f64(v))[np.where(sign > 0, most, least)]
    out = f64(got["out"])[0, 0]
    assert (np.abs(out - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want)).all()
    score = (R.round_trip(f64(k))[np.where(sign > 0, most, least)] * f64(q)).sum(-1) * d ** -0.5
    lse = f64(got["lse"])[0, 0]
    assert (np.abs(lse - score) <= 2.0 ** -16 * np.abs(score)).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 8, 16])
@pytest.mark.parametrize("scale", [1e-38, 1e-25, 1e-12])
def test_scores_that_are_all_but_nothing(d, G, scale):
    """Rows of zeros (a padded head) and of tiny queries with a tiny scale: every slot that a row sees has the
    same probability, and the others none."""
    rng = np.random.default_rng([d, G])
    for length, n in ((3, 1), (200, 3), (5000, 2)):
        k, v = rng_rows(rng, length, d, outliers=False), rng_rows(rng, length, d)
        pool, table, lens = pages_of(k, v, d)
        q = rng_rows(rng, 1, n, G, d)
        q[:, :, ::2] = 0
        q[:, :, 1::4] *= 2.0 ** -90
        kk, vv = R.round_trip(f64(k)), R.round_trip(f64(v))
        for window in (0, 50):
            got = tk.twinkv_cache_attend(q.to(device()), pool, table, lens, scale=scale, window=window,
                                         want_lse=True)
            want, lse, *sizes = R.attend(f64(q)[0], kk, vv, np.arange(length), scale, window, 0,
                                         R.quantize(f64(v))[1])
            bound = R.attend_bound(want, *sizes, length)
            assert (np.abs(f64(got["out"])[0] - want) <= bound).all()
            assert (np.abs(f64(got["lse"])[0] - lse) <= 5e-4).all()


@pytest.mark.parametrize("kw", [{"window": 2 ** 32 + 5}, {"window": 5, "n_sink": 2 ** 32},
                                {"window": 2 ** 31}])
def test_a_window_beyond_32_bits_is_refused(kw):
    x = torch.randn(100, 64).to(torch.bfloat16)
    pool, table, lens = pages_of(x, x, 64)
    q = torch.randn(1, 1, 4, 64, device=device()).to(torch.bfloat16)
    with pytest.raises(ValueError):
        tk.twinkv_cache_attend(q, pool, table, lens, **kw)
