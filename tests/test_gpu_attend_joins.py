"""Attention over units that the grid's warps and blocks share, with windows, many tokens and large
groups, and what its roundings come to (GPU), against the definition in 64 bits.

Queries are made to tell slots apart.  Most rows have three slots of their own (any, and those at
the ends of what the row sees), on which nearly all of the probability lies, in equal parts: a page that is
lost, taken twice or read from another place changes the output by a third of its size.  The others
point at a slot that they must not see: if they did, it would be all of their output.

bound() derives how far an output may be off.  With |x| <= y meaning "off by y at most":
  score      2^-21 per multiplication of 16 values, four a group, of sums that stay within
             30 s sum|q| (codes and zeros are below 16); and 2^-21 of the scores' size and 1 for what
             follows in float32.  A ratio of sums is off by twice that, relatively
  product    probability times value scale, as f16 in units of 2^(e - 7), of which half of the slots enter
             divided by 16: 2^-11 relatively, or 2^-28 of the largest scale's power of two, 2^e
  sums       of codes and of zeros, up to 15 p s each: 2^-20 per multiplication of 16 slots and rescaling, five
             a page; 2^-23 per part that is joined, of which there are less than 170
  output     2^-8, bf16 having 8 significant bits
"""
import numpy as np
import pytest
import torch

import cache_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from test_gpu_cache import f64, put

pytestmark = pytest.mark.gpu


class Units:
    """Units of lens[u] slots at random ascending positions, in pages of their own in any order."""

    def __init__(self, seed, lens, d, gap=2, k=None, v=None):
        rng = np.random.default_rng(seed)
        self.lens, self.d = [int(x) for x in lens], d
        U, N = len(lens), max(1, gap * max(lens))
        g = torch.Generator(device=device()).manual_seed(seed)
        shape = (1, U, N, d)
        mask = np.zeros((1, U, N), np.uint8)
        self.pos = []
        for u, n in enumerate(self.lens):
            self.pos.append(np.sort(rng.choice(N, n, replace=False)))
            mask[0, u, self.pos[u]] = 1

        def rows(given):
            x = torch.randn(shape, generator=g, device=device()).to(torch.bfloat16)
            for u, y in enumerate(given or []):
                x[0, u, put(self.pos[u])] = torch.from_numpy(y).to(torch.bfloat16).to(device())
            return x

        self._k, self._v = rows(k), rows(v)
        pages = max(1, -(-max(self.lens) // 64))
        ids = rng.permutation(U * pages).astype(np.int32).reshape(1, U, pages)
        self.pool = tk.cache_pool(U * pages, d, device())
        self.table = put(ids)
        out = tk.twinkv_cache_pack(self._k, self._v, put(mask), self.pool, self.table)
        assert out["status"].eq(0).all() and out["lens"].view(-1).tolist() == self.lens
        self.device_lens = out["lens"]

    def rows(self, u):
        """Keys, values and value scales of a unit, as its pages stand for them."""
        at = put(self.pos[u])
        k, v = (f64(x[0, u, at]) for x in (self._k, self._v))
        if not len(k):
            return k, v, np.zeros((0, self.d // 64)), np.zeros((0, self.d // 64))
        return R.round_trip(k), R.round_trip(v), R.quantize(k)[1], R.quantize(v)[1]

    def attend(self, q, **kw):
        """q [U][n][G][d] (numpy) over the units, each a sequence of its own."""
        U = len(self.lens)
        t = torch.from_numpy(q).to(torch.bfloat16).to(device())
        res = tk.twinkv_cache_attend(t, self.pool, self.table.view(U, 1, -1),
                                     self.device_lens.view(U, 1), want_lse=True, **kw)
        assert res["status"].eq(0).all()
        return f64(t), f64(res["out"]), f64(res["lse"])

    def pages(self, rows):
        """Pages of all parts of all units, windows not counted."""
        per = 8 if rows <= 8 else 16
        return sum(-(-n // 64) for n in self.lens) * -(-rows // per)


def seen(pos, n, window, n_sink):
    """[n][len] whether a unit's newest tokens see its slots."""
    length = len(pos)
    last = length - n + np.arange(n)
    see = np.arange(length)[None] <= last[:, None]
    if window > 0 and length:
        own = pos[np.maximum(last, 0)][:, None]
        see &= (pos[None] > own - window) | (pos[None] < n_sink)
    return see


def definition(q, k, v, see, scale, key_scales, value_scales, pages):
    """Outputs and log denominators of q [n][G][d] over a unit, and how far the kernel's may be off."""
    n, G, d = q.shape
    groups = d // 64
    out, bound = np.zeros((n, G, d)), np.zeros((n, G, d))
    lse, lse_bound = np.full((n, G), -np.inf), np.zeros((n, G))
    steps = 5 * (-(-pages // (152 * 8)) + 1)
    for i in range(n):
        at = np.flatnonzero(see[i])
        if not len(at):
            continue
        kk, vv = k[at], v[at]
        vs = np.repeat(value_scales[at], 64, axis=1)
        x = q[i] @ kk.T * scale
        m = x.max(-1, keepdims=True)
        p = np.exp(x - m)
        total = p.sum(-1, keepdims=True)
        p /= total
        sums = np.abs(q[i]).reshape(G, groups, 64).sum(-1)
        score = (scale * 30 * 4 * 2.0 ** -21 * (sums * key_scales[at].max(0)).sum(-1)
                 + 2.0 ** -21 * (np.abs(x).max(-1) + 1))[:, None]
        out[i] = p @ vv
        top = 2.0 ** np.floor(np.log2(np.maximum(value_scales.max(0), 2.0 ** -126)))
        codes = (np.abs(vv) / np.where(vs > 0, vs, 1)).sum(0) * np.repeat(top, 64)
        rest = ((2.0 ** -11 + 2.1 * score) * (p @ np.abs(vv)) + 2.0 ** -28 * codes / total
                + 30 * (steps * 2.0 ** -20 + 170 * 2.0 ** -23) * (p @ vs)
                + 2.0 ** -18 * np.abs(out[i]))
        bound[i] = rest + 2.0 ** -8 * (np.abs(out[i]) + rest)
        lse[i] = (m + np.log(total))[:, 0]
        lse_bound[i] = (2.1 * score)[:, 0] + 2.0 ** -20 * (1 + np.abs(lse[i])) \
            + (4 * steps + 170) * 2.0 ** -23
    return out, bound, lse, lse_bound


def check(units, q, n, window=0, n_sink=0):
    d, scale = units.d, units.d ** -0.5
    q, got, got_lse = units.attend(q, window=window, n_sink=n_sink)
    pages = units.pages(q.shape[1] * q.shape[2])
    widest = 0.0
    for u in range(len(units.lens)):
        k, v, ks, vs = units.rows(u)
        see = seen(units.pos[u], n, window, n_sink)
        out, bound, lse, lse_bound = definition(q[u], k, v, see, scale, ks, vs, pages)
        err = np.abs(got[u] - out)
        assert (err <= bound).all(), (u, units.lens[u], np.argwhere(err > bound)[:4].tolist(),
                                      (err / np.maximum(bound, 1e-30)).max())
        assert np.array_equal(np.isneginf(got_lse[u]), np.isneginf(lse)), u
        fine = np.isfinite(lse)
        assert (np.abs(got_lse[u][fine] - lse[fine]) <= lse_bound[fine]).all(), u
        widest = max(widest, np.sqrt((bound ** 2).mean()))
    return widest


def pointing_queries(seed, units, n, G, window, n_sink, level=25.0):
    rng = np.random.default_rng([seed, 1])
    d = units.d
    q = rng.standard_normal((len(units.lens), n, G, d)) * 0.1
    for u, length in enumerate(units.lens):
        if not length:
            continue
        k = units.rows(u)[0]
        see = seen(units.pos[u], n, window, n_sink)
        for i in range(n):
            ins, outs = np.flatnonzero(see[i]), np.flatnonzero(~see[i])
            edge = np.flatnonzero(np.diff(see[i].astype(int)))
            near = sorted({int(x) for e in edge for x in (e, e + 1)})
            for g in range(G):
                if g % 4 == 3 and len(outs):
                    at = [x for x in near if not see[i][x]] if g % 8 == 3 else outs
                    at = [int(rng.choice(at if len(at) else outs))]
                elif len(ins):
                    at = rng.choice(ins, min(3, len(ins)), replace=False).tolist()
                    mine = [x for x in near if see[i][x]]
                    if mine and g % 2:
                        at[0] = mine[int(rng.integers(len(mine)))]
                    at = sorted(set(at))
                else:
                    continue
                q[u, i, g] = np.linalg.pinv(k[at]) @ np.full(len(at), level * d ** 0.5)
    return q


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n,units,least,most", [
    (4, 1, 3, 50000, 90000), (8, 1, 2, 50000, 90000), (2, 8, 2, 40000, 60000),
    (4, 1, 300, 0, 900), (8, 1, 300, 0, 900), (4, 4, 250, 0, 600), (6, 4, 100, 0, 1500),
    (4, 64, 6, 0, 1500), (1, 64, 8, 30, 700), (64, 1, 20, 0, 1000), (256, 2, 3, 1, 400),
    (7, 33, 5, 0, 900)])
def test_units_over_the_grid(d, G, n, units, least, most):
    seed = 1000 * G + 10 * n + d
    lens = np.random.default_rng(seed).integers(least, most + 1, units)
    if least == 0:
        lens[units // 2:units // 2 + max(1, units // 20)] = 0
    c = Units(seed, lens, d)
    for turn in range(6 if units < 4 and n < 64 and G < 64 else 1):   # more slots of long units
        widest = check(c, pointing_queries(seed + turn, c, n, G, 0, 0), n)
        assert widest < 0.05              # against values of size 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n,units,least,most,window,n_sink", [
    (4, 1, 100, 2500, 5000, 4000, 130), (8, 1, 100, 2500, 5000, 4000, 4),
    (4, 4, 100, 2500, 5000, 4000, 130), (4, 6, 60, 2500, 5000, 4000, 4),
    (4, 1, 500, 100, 1200, 300, 0), (4, 4, 300, 100, 1200, 300, 4), (5, 7, 200, 0, 1200, 300, 130),
    (5, 64, 10, 0, 1500, 300, 130), (40, 2, 30, 0, 2500, 2000, 4), (4, 1, 3, 50000, 70000, 90000, 4),
    (4, 2, 4, 30000, 50000, 2000, 130)])
def test_windows_over_the_grid(d, G, n, units, least, most, window, n_sink):
    """Spans of warps that go from a unit's sinks to its window and on to the next unit."""
    seed = 1000 * G + 10 * n + d + window
    lens = np.random.default_rng(seed).integers(least, most + 1, units)
    c = Units(seed, lens, d)
    widest = check(c, pointing_queries(seed, c, n, G, window, n_sink), n, window, n_sink)
    assert widest < 0.05


@pytest.mark.parametrize("gap", [1, 100])
@pytest.mark.parametrize("window", [1, 2, 64, 65, 4096, 10 ** 6])
def test_windows_over_gaps_between_positions(gap, window):
    c = Units(gap, [1, 64, 65, 700, 1300], 64, gap=gap)
    check(c, pointing_queries(window, c, 5, 4, window, 4), 5, window, 4)


# ---------------------------------------------------------------- roundings

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 8, 16])
@pytest.mark.parametrize("length", [500, 20000])
@pytest.mark.parametrize("above", [8, 12, 14, 16])
def test_one_key_with_a_value_of_0_above_all_others(d, G, length, above):
    """As a sink often is: the output is what the small probabilities of the others come to."""
    rng = np.random.default_rng([d, G, length, above])
    u = rng.choice([-1.0, 1.0], d)
    k = rng.standard_normal((length, d)) * 0.05
    v = 1.0 + 0.2 * rng.standard_normal((length, d))
    first = int(rng.integers(length))
    k[first], v[first] = u, 0.0
    c = Units(above, [length], d, gap=1, k=[k], v=[v])
    q = np.broadcast_to(u * above * d ** -0.5, (1, 1, G, d)) * rng.uniform(0.9, 1.1, (1, 1, G, 1))
    check(c, q, 1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 8, 16])
def test_probabilities_have_11_bits(d, G):
    """Pairs of opposite values under nearly equal scores: outputs are near 0, and what the
    probabilities lose stays visible beside the output's own rounding."""
    rng = np.random.default_rng([d, G])
    lens = [2, 4, 8] * 40
    k = [rng.standard_normal((n, d)) * 0.3 for n in lens]
    v = []
    for n in lens:
        half = rng.standard_normal((n // 2, d))
        v.append(np.stack([half, -half], 1).reshape(n, d))
    c = Units(d + G, lens, d, gap=1, k=k, v=v)
    check(c, rng.standard_normal((len(lens), 1, G, d)) * 0.3, 1)
