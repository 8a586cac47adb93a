"""What the bound of test_gpu_attend_joins.py can see, without a GPU: mistakes planted in the
definition itself have to exceed it."""
import numpy as np
import pytest

import cache_reference as R
import test_gpu_attend_joins as J


class Rows:
    """One unit's rows, as Units has them."""

    def __init__(self, seed, length, d):
        rng = np.random.default_rng(seed)
        self.lens, self.d = [length], d
        self.pos = [np.arange(length) * 2]
        k, v = (R.to_bf16(rng.standard_normal((length, d))) for _ in range(2))
        self._rows = R.round_trip(k), R.round_trip(v), R.quantize(k)[1], R.quantize(v)[1]

    def rows(self, u):
        return self._rows


def setting(d, length, window=0, n_sink=0, n=2, G=8):
    c = Rows(length + d, length, d)
    q = R.to_bf16(J.pointing_queries(3, c, n, G, window, n_sink))[0]
    return c, q, J.seen(c.pos[0], n, window, n_sink), d ** -0.5


def shares(c, q, see, scale):
    """Probabilities of each row over all slots."""
    x = np.where(see[:, None], q @ c.rows(0)[0].T * scale, -np.inf)
    p = np.exp(x - x.max(-1, keepdims=True))
    return p / p.sum(-1, keepdims=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [200, 5000, 90000])
def test_a_page_lost_taken_twice_or_read_elsewhere(d, length):
    c, q, see, scale = setting(d, length)
    k, v, ks, vs = c.rows(0)
    pages = -(-length // 64)
    out, bound, *_ = J.definition(q, k, v, see, scale, ks, vs, pages)
    p = shares(c, q, see, scale)
    pointed = [g for g in range(8) if g % 4 != 3]
    for g in pointed:
        for page in np.unique(np.argsort(p[0, g])[-3:] // 64):
            at = np.arange(length) // 64 == page
            lost = (p[0, g, ~at] @ v[~at]) / p[0, g, ~at].sum()
            twice = (out[0, g] + p[0, g, at] @ v[at]) / (1 + p[0, g, at].sum())
            other = v.copy()
            other[at] = v[(np.flatnonzero(at) + 64) % length]
            for wrong in (lost, twice, p[0, g] @ other):
                if p[0, g, at].sum() < 0.1 or pages < 2:
                    continue
                assert (np.abs(wrong - out[0, g]) > bound[0, g]).mean() > 0.3
    assert np.sqrt((bound ** 2).mean()) < 0.05


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,n_sink", [(300, 0), (300, 4), (2000, 130)])
def test_a_slot_seen_that_must_not_be(d, window, n_sink):
    c, q, see, scale = setting(d, 5000, window, n_sink)
    k, v, ks, vs = c.rows(0)
    out, bound, *_ = J.definition(q, k, v, see, scale, ks, vs, 80)
    more = see.copy()
    edge = np.flatnonzero(np.diff(see[0].astype(int)))
    more[:, edge], more[:, edge + 1] = True, True
    wide, *_ = J.definition(q, k, v, more, scale, ks, vs, 80)
    err = np.abs(wide - out)
    assert (err > bound).any(-1).any(0)[3] and (err[:, 3].max(-1) > 0.5).any()
    everything, *_ = J.definition(q, k, v, np.ones_like(see), scale, ks, vs, 80)
    for g in (3, 7):
        assert (np.abs(everything - out)[:, g] > bound[:, g]).mean() > 0.3


@pytest.mark.parametrize("d", [64, 128])
def test_probabilities_of_8_bits(d):
    """Products of probabilities and value scales rounded to bf16 instead of f16."""
    rng = np.random.default_rng(d)
    beyond = 0
    for n in (2, 4, 8) * 20:
        half = rng.standard_normal((n // 2, d))
        v0 = R.to_bf16(np.stack([half, -half], 1).reshape(n, d))
        k0 = R.to_bf16(rng.standard_normal((n, d)) * 0.3)
        k, v, ks, vs = R.round_trip(k0), R.round_trip(v0), R.quantize(k0)[1], R.quantize(v0)[1]
        q = R.to_bf16(rng.standard_normal((1, 4, d)) * 0.3)
        see = np.ones((1, n), bool)
        out, bound, *_ = J.definition(q, k, v, see, d ** -0.5, ks, vs, 1)
        x = q[0] @ k.T * d ** -0.5
        p = np.exp(x - x.max(-1, keepdims=True))
        for bits, least in ((R.to_bf16, True), (lambda y: y.astype(np.float16).astype(float), False)):
            got = np.zeros((4, d))
            for e in range(d):
                s = vs[:, e // 64]
                got[:, e] = bits(p * s) @ (v[:, e] / np.where(s > 0, s, 1)) / p.sum(-1)
            wrong = (np.abs(R.to_bf16(got) - out[0]) > bound[0]).any()
            if least:
                beyond += wrong
            else:
                assert not wrong
    assert beyond > 30
