"""The way of a retained set on the GPU: a prompt's attention, what it pays to each key, the eviction,
the repair, pages, decoded tokens that add to the sums, and evictions while decoding."""
import numpy as np
import pytest
import torch

import prompt_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import decode
from paper_2608_27128_gb300 import twinkv as tk
from paper_2608_27128_gb300.pages import PageCache

pytestmark = pytest.mark.gpu

L, H, HQ = 2, 2, 8


def normal(*shape, seed=0):
    g = torch.Generator(device=device()).manual_seed(seed)
    return torch.randn(shape, generator=g, device=device()).to(torch.bfloat16)


def prompt(N, d, last):
    """A prompt's dense cache and the sums of its last tokens' attention."""
    keys, values = normal(L, H, N, d, seed=1), normal(L, H, N, d, seed=2)
    score = torch.empty((L, H, N), device=device())
    for l in range(L):
        q = normal(N, HQ, d, seed=3 + l)
        k, v = keys[l].transpose(0, 1), values[l].transpose(0, 1)
        a = tk.twinkv_prompt_attend(q, k, v, want_lse=True)
        tk.twinkv_prompt_weights(q, k, a["lse"], last=last, out={"score": score[l]})
    return keys, values, score


@pytest.mark.parametrize("d", [64, 128])
def test_the_whole_way(d):
    N, budget, steps = 500, 200, 5
    keys, values, score = prompt(N, d, 32)
    # every token and query head gives one in all, whatever the keys (weights are off by 2^-14 or so)
    np.testing.assert_allclose(score.double().sum(-1).cpu().numpy(), 32 * HQ // H, rtol=2.0 ** -12)
    policy = tk.twinkv_weight_policy(score, budget, want_score=True)
    for u in range(L * H):
        m, k, _ = R.policy(score.view(L * H, N)[u].cpu().numpy(), N, budget, 4, 64)
        np.testing.assert_array_equal(policy["mask"].view(L * H, N)[u].cpu().numpy(), m)
        np.testing.assert_array_equal(policy["score"].view(L * H, N)[u].cpu().numpy(), k)
    out = tk.twinkv_repair(keys, policy["mask"], None, 0.85)
    cache = PageCache(L, 1, H, d, n_pages=60, max_pages=8)
    assert not cache.pack(0, keys, values, out["mask"], budget).any()
    sums = torch.zeros(L, 1, H, 8 * 64, device=device())
    sums[:, 0, :, :budget] = score[out["mask"].bool()].view(L, H, budget)
    for step in range(steps):
        cache.reserve(1)
        pos = torch.full((1, 1), N + step, dtype=torch.int32, device=device())
        for l in range(L):
            q, k, v = normal(1, 1, HQ, d), normal(1, 1, H, d, seed=9), normal(1, 1, H, d, seed=10)
            cache.append(l, k, v, pos)
            before = sums[l].clone()
            a = cache.attend(l, q, want_lse=True)
            assert not cache.weigh(l, q, a["lse"], sums[l]).any()
            added = (sums[l] - before).double()
            held = budget + step + 1
            np.testing.assert_allclose(added[..., :held].sum(-1).cpu().numpy(), HQ // H,
                                       rtol=2.0 ** -10)
            assert not added[..., held:].any()
    # a second eviction: rows, positions and sums are those of the kept slots, in order
    held, less = budget + steps, 100
    rows = cache.read(0, held)
    old = sums[:, 0].contiguous()
    got = cache.evict(0, old, less)
    assert not got["status"].any() and cache.lens.eq(less).all()
    after = cache.read(0, less)
    for l in range(L):
        for h in range(H):
            m, k, _ = R.policy(old[l, h].cpu().numpy(), held, less, 4, 64)
            np.testing.assert_array_equal(got["mask"][l, h].cpu().numpy(), m)
            np.testing.assert_array_equal(got["score"][l, h].cpu().numpy(), k)
            at = torch.from_numpy(np.flatnonzero(m)).to(device())
            for name in ("keys", "values", "positions"):
                assert torch.equal(after[name][l, h], rows[name][l, h][at])
    # more than there is: everything stays
    got = cache.evict(0, got["score"], 400)
    assert not got["status"].any() and cache.lens.eq(less).all()
    for name in ("keys", "values", "positions"):
        assert torch.equal(cache.read(0, less)[name], after[name])
    assert tk.twinkv_get_last_error() == tk.OK


def test_a_prompt_in_chunks_is_the_prompt():
    """Chunks over the cache that earlier ones left: the same rows within what the roundings of two
    orders of the same sums allow, and sums that add up."""
    N, d = 700, 128
    keys, values, _ = prompt(N, d, 0)
    q = normal(N, HQ, d, seed=3)
    k, v = keys[0].transpose(0, 1), values[0].transpose(0, 1)
    whole = tk.twinkv_prompt_attend(q, k, v, want_lse=True)
    score = tk.twinkv_prompt_weights(q, k, whole["lse"])["score"]
    sums = torch.zeros(H, N, device=device())
    for begin, end in ((0, 100), (100, 357), (357, 700)):
        a = tk.twinkv_prompt_attend(q[begin:end], k[:end], v[:end], want_lse=True)
        ref = whole["out"][begin:end].double()
        # each is within 2^-7 of the rows' weighted |v| (about 1) of the exact one
        assert (a["out"].double() - ref).abs().max() <= 2 * 2.0 ** -7 * 3
        assert (a["lse"] - whole["lse"][begin:end]).abs().max() <= 2.0 ** -10
        part = sums[:, :end].contiguous()
        tk.twinkv_prompt_weights(q[begin:end], k[:end], a["lse"], score=part, out={"score": part})
        sums[:, :end] = part
    np.testing.assert_allclose(sums.cpu().numpy(), score.cpu().numpy(), rtol=2.0 ** -9)


def test_the_example_sums_weights():
    """Half the sequences' sums come from the prompt's last 32 tokens, the rest from decoded ones."""
    res = decode.demo(steps=6, N=400, say=lambda *_: None)
    held = res["cache"].lens
    for b in range(2):
        n = int(held[0, b, 0])
        assert (res["sums"][:, b, :, n:] == 0).all()
        s = res["sums"][:, b, :, :n]
        assert torch.isfinite(s).all() and (s >= 0).all() and s.any()
    # sequence 0 was not evicted: 6 tokens of 4 heads, and what the kept keys had before
    assert (res["sums"][:, 0].sum(-1) > 6 * 4 * 0.999).all()
