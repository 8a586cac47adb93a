"""Weights from large scores, up to what the header allows (GPU): exact scores, as in
test_gpu_prompt_scores."""
import numpy as np
import pytest
import torch

import cache_reference as C
import prompt_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from test_gpu_cache import make_cache, put
from test_gpu_prompt_scores import attend, prompt
from test_gpu_weights import C_STEP

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e", [0, 4, 8, 12, 15])
@pytest.mark.parametrize("window,n_sink,last", [(0, 0, 0), (500, 4, 0), (0, 0, 16)])
def test_large_scores(d, e, window, n_sink, last):
    """Scores of either sign up to d^0.5 2^e (2^18.5), beside ordinary ones.  With x the score and lse as it is
    given, in float32, the exponent is off by 2^-24 |x| for the factor of a score, 2^-23 |lse| for
    that of lse and its rounding, 2^-24 |x - lse| for the difference's, and the exponential by 2^-22."""
    for n, m in ((150, 150), (100, 3000)):
        p = prompt(n, m, d, e, [0, 0, -e, -e], e, more=[(3, 40)])
        lse = np.full((p.T, p.Hq), np.nan, np.float32)
        want, off = np.zeros((1, p.Tk)), np.zeros((1, p.Tk))
        assert np.nanmax(np.abs(p.k64)) * d ** 0.5 < 2.0 ** 20
        for t, j, h, kv in p.heads():
            q, k, v = p.q64[t, h], p.k64[j, kv], p.v64[j, kv]
            lse[t, h] = attend(q, k, v, d ** -0.5, window, n_sink)[1]
            log = lse[t, h].astype(np.float64)[:, None]
            see = R.sees(len(q), len(k), window, n_sink)
            if last > 0:
                see[:max(0, len(q) - last)] = False
            x = np.where(see, q @ k.T * d ** -0.5, 0.0)
            log = np.where(see, log, 0.0)
            w = np.where(see, np.exp(x - log), 0.0)
            far = (2.0 ** -24 * np.abs(x) + 2.0 ** -23 * np.abs(log) + 2.0 ** -24 * np.abs(x - log)
                   + 2.0 ** -22)
            want[kv, j] += w.sum(0)
            off[kv, j] += (w * np.expm1(far)).sum(0) + (len(q) * p.Hq + 4) * 2.0 ** -23 * w.sum(0) + 1e-37
        given = {"score": torch.full((1, p.Tk), 7.0, device=device())}
        got = tk.twinkv_prompt_weights(p.q, p.k, put(lse), **p.where, window=window, n_sink=n_sink,
                                       last=last, out=given)
        assert got["status"].eq(0).all() and tk.twinkv_get_last_error() == tk.OK
        score = got["score"].double().cpu().numpy()
        assert (score[:, ~p.key] == 7.0).all()
        bad = np.abs(score - want) > off
        assert not bad[:, p.key].any(), (np.abs(score - want) / np.maximum(off, 1e-37))[:, p.key].max()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 2), (8, 5)])
def test_large_scores_over_pages(d, G, n):
    """Queries of up to 64 times the usual size.  A score's float32 sums are off as test_gpu_weights derives
    (d + 8 steps over terms of 31 |q| s, one of 128 a group), the rest as above."""
    rng = np.random.default_rng([d, G, n])
    lens = [700, 130]
    pool, table, units = make_cache(rng, lens, d, n_new=n)
    q = torch.from_numpy(rng.standard_normal((2, n, G, d)) * 2.0 ** rng.integers(0, 7, (2, n, G, 1)))
    q = q.to(torch.bfloat16)
    q64, scale = q.double().numpy(), d ** -0.5
    lse = np.zeros((2, n, G), np.float32)
    want, off = np.zeros((2, 700)), np.zeros((2, 700))
    for u, (k, v, pos, _) in enumerate(units):
        length = len(pos)
        for i in range(n):
            log = C.attend(q64[u, i:i + 1], k[:length - n + 1 + i], v[:length - n + 1 + i], pos, scale)[1]
            lse[u, i] = log[0]
            see = np.arange(length)[:, None] <= length - n + i
            x = k @ q64[u, i].T * scale
            y = lse[u, i].astype(np.float64)
            w = np.where(see, np.exp(np.where(see, x - y, 0.0)), 0.0)
            steps = np.abs(q64[u, i]).sum(-1) * C_STEP(k)
            far = ((31 * (d + 8) + 256) * 2.0 ** -23 * scale * steps + 2.0 ** -23 * (np.abs(x) + np.abs(y))
                   + 2.0 ** -24 * np.abs(x - y) + 2.0 ** -22)
            want[u, :length] += w.sum(-1)
            off[u, :length] += (w * np.expm1(far)).sum(-1) + (n * G + 2) * 2.0 ** -23 * w.sum(-1) + 1e-37
    score = torch.zeros(2, 1, 700, device=device())
    got = tk.twinkv_cache_weights(q.to(device()), put(lse), pool, table.view(2, 1, -1),
                                  put(np.array(lens, np.int32)).view(2, 1), score)
    assert got["status"].eq(0).all() and tk.twinkv_get_last_error() == tk.OK
    for u, length in enumerate(lens):
        a = got["score"][u, 0, :length].double().cpu().numpy()
        assert (np.abs(a - want[u, :length]) <= off[u, :length]).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [1e-12, 1e-38, 1e-40, 1e-45])
def test_scales_down_to_the_smallest(d, scale):
    """Scores that are all but nothing, also where the scale has few bits or none beside log 2: a token pays
    alike to every key that it sees, and nothing to the others.  Off by lse's rounding and its
    product's, 2^-23 |lse| with |lse| < 8, the exponential's 2^-22, and the sum's 2^-23 a step; the
    scores themselves are below 2^-21."""
    p = prompt(100, 700, d, 0, [0, 0, -3, 2], 1, more=[(33, 33)])
    lse = np.full((p.T, p.Hq), np.nan, np.float32)
    want, steps = np.zeros(p.Tk), np.zeros(p.Tk)
    for (n, m), t, j in zip(p.seqs, p.t0, p.j0):
        see = R.sees(n, m)
        lse[t:t + n] = np.log(see.sum(1))[:, None]
        want[j:j + m] = p.Hq * (see / see.sum(1)[:, None]).sum(0)
        steps[j:j + m] = n * p.Hq
    off = want * (8 * 2.0 ** -22 + 2.0 ** -21 + 2.0 ** -22 + (steps + 4) * 2.0 ** -23)
    got = tk.twinkv_prompt_weights(p.q, p.k, put(lse), **p.where, scale=scale)
    score = got["score"].double().cpu().numpy()[0]
    assert (np.abs(score - want) <= off)[p.key].all()

    pool, table, _ = make_cache(np.random.default_rng(d), [300], d)
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((1, 1, 4, d))).to(torch.bfloat16)
    log = torch.full((1, 1, 4), float(np.log(300)), device=device())
    score = tk.twinkv_cache_weights(q.to(device()), log, pool, table.view(1, 1, -1),
                                    torch.full((1, 1), 300, dtype=torch.int32, device=device()),
                                    torch.zeros(1, 1, 300, device=device()), scale=scale)["score"]
    assert (score.double() - 4 / 300).abs().max() <= 4 / 300 * (8 * 2.0 ** -22 + 2.0 ** -20)
