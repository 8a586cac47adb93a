"""Windowed attention over units with page numbers outside the pool (GPU)."""
import numpy as np
import pytest
import torch

import cache_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from test_gpu_cache import f64, make_cache, put, rng_rows

pytestmark = pytest.mark.gpu


def windowed(q, k, v, pos, gone, scale, window, n_sink, v_scales):
    """R.attend of one unit whose slots in `gone` are unseen; a token's own position is that of the
    last slot up to its own whose page is in the pool."""
    n, G, d = q.shape
    out, size, steps = (np.zeros((n, G, d)) for _ in range(3))
    length = len(k)
    for i in range(n):
        last = length - n + i
        known = np.flatnonzero(~gone[:last + 1])
        see = (np.arange(length) <= last) & ~gone
        own = pos[known[-1]] if len(known) else -1
        see &= (pos > own - window) | (pos < n_sink)
        if not see.any():
            continue
        x = q[i] @ k[see].T * scale
        p = np.exp(x - x.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        s = np.repeat(v_scales[see], 64, axis=1)
        out[i], size[i], steps[i] = p @ v[see], p @ np.abs(v[see]), p @ s
    return out, size, steps


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("bad", [[7], [10], [5, 6, 7, 8], [0], [0, 1], [11], [10, 11],
                                 list(range(12))])
def test_a_window_over_pages_outside_the_pool(d, n, bad):
    """Slots of such pages count as unseen, and the others are seen as they were."""
    rng = np.random.default_rng([d, n, len(bad), bad[0]])
    length = 12 * 64 - 10
    pool, ids, units = make_cache(rng, [length], d, n_new=n)
    ids[0, bad] = torch.tensor([-1, 10 ** 6] * 6, dtype=torch.int32, device=device())[:len(bad)]
    k, v, pos, vs = units[0]
    gone = np.isin(np.arange(length) // 64, bad)
    q = rng_rows(rng, 1, n, 4, d)
    lens = put(np.array([[length]], np.int32))
    for window, n_sink in ((1, 0), (90, 4), (300, 70), (500, 0), (600, 200), (100000, 4)):
        got = tk.twinkv_cache_attend(q.to(device()), pool, ids.view(1, 1, -1), lens, window=window,
                                     n_sink=n_sink)
        assert got["status"].tolist() == [[1]]
        want, *sizes = windowed(f64(q)[0], k, v, pos, gone, d ** -0.5, window, n_sink, vs)
        err = np.abs(f64(got["out"])[0] - want)
        assert (err <= R.attend_bound(want, *sizes, length)).all(), (window, n_sink)
