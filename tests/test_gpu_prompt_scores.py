"""Attention over prompts whose scores are large, or far apart (GPU).

Keys are multiples of one direction of +-1, and so are the queries, so that a score's partial sums are
whole multiples of one power of two with at most 15 significant bits: float32 holds them exactly,
and the reference's scores are the kernel's.  What is left to be off is derived at `bound`."""
import numpy as np
import pytest
import torch

import prompt_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from prompt_cases import Prompts

pytestmark = pytest.mark.gpu


def levels(rng, m):
    """Multiples that seldom rise above, or fall below, all those before them."""
    x = rng.uniform(0.45, 0.55, m)
    at = np.unique(np.concatenate([[0], np.geomspace(2, max(3, m - 1), 8).astype(int)]))
    at = at[at < m]
    x[at] = 0.6 + 0.05 * np.arange(len(at))
    down = at[at + 1 < m] + 1
    x[down] = 0.4 - 0.03 * np.arange(len(down))
    return x


def prompt(n, m, d, key_exponent, q_exponents, seed, more=()):
    """Sequence (n, m), and others, whose keys are levels times 2^key_exponent of one direction (an
    exponent for each key, or one), and whose query head i is sign (-1)^i of it times
    2^q_exponents[i]."""
    rng = np.random.default_rng([n, m, d, seed])
    p = Prompts([(n, m), *more], len(q_exponents), 1, d, device(), gap=1, seed=seed)
    u = rng.choice([-1.0, 1.0], d)
    for (_, m_), j in zip(p.seqs, p.j0):
        e = np.broadcast_to(key_exponent, m)[:m_]
        p.k64[j:j + m_, 0] = np.ldexp(levels(rng, m_), e)[:, None] * u
    sign = np.where(np.arange(len(q_exponents)) % 2, -1.0, 1.0)
    p.q64[p.token] = (np.ldexp(sign, q_exponents)[:, None] * u)[None]
    p.k, p.q = (torch.from_numpy(x).to(torch.bfloat16) for x in (p.k64, p.q64))
    p.k64, p.q64 = p.k.double().numpy(), p.q.double().numpy()
    p.k, p.q = p.k.to(device()), p.q.to(device())
    return p


def attend(q, k, v, scale, window=0, n_sink=0):
    """One sequence and query head in 64 bits with exact scores: outputs, lse, and how far they may be
    off:
      2^-8 p |v|       a probability is rounded to bf16 for its product
      2^-8 |out|       so is the output
      m 2^-22 p |v|    float32 sums over m keys, twice, as in prompt_reference.attend
      2^-22 p |x - x_top| |v|, twice: a score's distance from the top is rounded, and multiplied
                       with a rounded factor, 2^-24 each at most, for the numerator and the denominator
      2^-11 p |v|      the row's top enters rounded, below 2^12 in units of log 2: what a row has when its
                       top rises beyond that is off by half of that top's last bit, 2^-13
    and for lse the sum's m 2^-23, and 2^-22 of itself for its factors and its roundings."""
    n, m = len(q), len(k)
    see = R.sees(n, m, window, n_sink)
    x = np.where(see, q @ k.T * scale, -np.inf)
    top = x.max(1, initial=-np.inf)
    some = np.isfinite(top)
    gap = np.where(see, x - np.where(some, top, 0)[:, None], -np.inf)
    p = np.exp(gap)
    total = p.sum(1)
    lse = np.where(some, top + np.log(np.where(some, total, 1)), -np.inf)
    p /= np.where(some, total, 1)[:, None]
    out, size = p @ v, p @ np.abs(v)
    far = (p * np.where(see, -gap, 0)) @ np.abs(v) + (p * np.where(see, -gap, 0)).sum(1)[:, None] * size
    off = (2.0 ** -8 * (size + np.abs(out)) + ((m + 8) * 2.0 ** -22 + 2.0 ** -11) * size
           + 2.0 ** -21 * far + 1e-30)
    return out, lse, off, (m + 8) * 2.0 ** -23 + np.abs(np.where(some, lse, 0)) * 2.0 ** -22


def check(p, scale=None, v_size=1.0, **kw):
    dev = device()
    given = {"out": torch.full((p.T, p.Hq, p.d), 7.0, dtype=torch.bfloat16, device=dev),
             "lse": torch.full((p.T, p.Hq), 7.0, device=dev)}
    got = tk.twinkv_prompt_attend(p.q, p.k, p.v, **p.where, scale=scale, want_lse=True, out=given,
                                  **kw)
    assert tk.twinkv_get_last_error() == tk.OK and got["status"].eq(0).all()
    out, lse = got["out"].double().cpu().numpy(), got["lse"].double().cpu().numpy()
    assert (out[~p.token] == 7.0).all() and (lse[~p.token] == 7.0).all()
    scale = p.d ** -0.5 if scale is None else float(np.float32(scale))
    for t, j, h, kv in p.heads():
        want, log, off, off_log = attend(p.q64[t, h], p.k64[j, kv], p.v64[j, kv], scale, **kw)
        a, b = out[t, h], lse[t, h]
        assert np.isfinite(a).all(), (t, h)
        assert (np.abs(a - want) <= off).all(), (t, h, (np.abs(a - want) / off).max())
        none = np.isinf(log)
        assert (b[none] == -np.inf).all() and (a[none] == 0).all()
        assert (np.abs(b[~none] - log[~none]) <= off_log[~none]).all(), (t, h)
    return got


# q . k of d 2^e: e = 8 or so is where scores pass 2^12 in units of log 2, 28 where their rounding passes 2^7
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e", [2, 8, 9, 16, 28, 31, 36, 60, 100])
def test_large_scores(d, e):
    """Large scores of either sign beside ordinary ones in other rows of the same warp, in items that
    one block does and in items that are cut; windows that leave the largest behind."""
    heads = [0, 0, -e, -e, -e // 2]
    check(prompt(150, 150, d, e, heads, 1))
    p = prompt(100, 3000, d, e, heads, 2, more=[(3, 40), (5, 3)])
    assert tk.prompt_attend_workspace(p.q.shape, p.k.shape, 3, "cpu").numel() > 256
    check(p)
    check(p, window=500, n_sink=4)
    check(p, window=40)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_tops_of_random_size(d, seed):
    """Rows whose largest scores are of all sizes up to 2^119."""
    heads = list(np.random.default_rng(seed).integers(0, 100, 16))
    check(prompt(64, 3000, d, 10, heads, seed))
    check(prompt(150, 150, d, 0, heads, seed))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e", [12, 40, 100])
@pytest.mark.parametrize("down", [False, True])
def test_scores_that_pass_from_small_to_large(d, e, down):
    """Keys that grow, or shrink, by 2^(e + 4) along the sequence, a little with every few of them."""
    for n, m in ((300, 300), (90, 2500)):
        exponents = np.linspace(-4, e, m).round().astype(int)
        check(prompt(n, m, d, exponents[::-1] if down else exponents, [0, 0, -e, -2], e))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale,k,q", [(1.0, 80, 0), (2.0 ** 20, 80, 0), (2.0 ** 100, 0, 0),
                                       (2.0 ** 110, -56, -56), (2.0 ** 126, -60, -60),
                                       (1e-30, 100, 0), (1e-38, 0, 0), (1e-40, 0, 0),
                                       (1e-45, 60, 0)])
def test_scales(d, scale, k, q):
    """From scores that are alike to the largest ones, by the scale."""
    check(prompt(40, 200, d, k, [q] * 4, 1), scale=scale)


@pytest.mark.parametrize("d", [64, 128])
def test_equal_large_scores_share_the_output(d):
    """The top key twice: half of either's value."""
    p = prompt(30, 200, d, 60, [0, 0], 5)
    p.k64[p.j0[0] + 90] = p.k64[p.j0[0] + 40] = 2 * p.k64[p.j0[0]]
    p.k = torch.from_numpy(p.k64).to(torch.bfloat16).to(device())
    got = check(p)
    want = (p.v64[p.j0[0] + 90, 0] + p.v64[p.j0[0] + 40, 0]) / 2
    out = got["out"][:30, 0].double().cpu().numpy()
    assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("d", [64, 128])
def test_large_values(d):
    """Values up to the largest that the header allows, whose products with probabilities of up to
    2^15 (a tile's sum before the top follows) and their sums stay finite."""
    size = 2.0 ** 92
    for n, m in ((300, 300), (64, 3000)):
        p = Prompts([(n, m)], 2, 1, d, device(), seed=d)
        p.k64[:] = 0
        p.k64[:, 0, 0] = np.linspace(0, 60, m)         # rises by less than the top follows at, for long
        p.q64[:] = 0
        p.q64[:, 0, 0], p.q64[:, 1, 0] = d ** 0.5, -d ** 0.5
        p.k, p.q = (torch.from_numpy(x).to(torch.bfloat16).to(device()) for x in (p.k64, p.q64))
        p.k64, p.q64 = p.k.double().cpu().numpy(), p.q.double().cpu().numpy()
        p.v64 = p.v64 * size
        p.v = torch.from_numpy(p.v64).to(torch.bfloat16).to(device())
        assert np.abs(p.v64).max() < 2.0 ** 95
        check(p)
