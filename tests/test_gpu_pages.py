"""PageCache (GPU): pages are taken, shared, copied and freed as they should be, and what a
sequence holds does not change by what happens to another; the example runs through."""
import numpy as np
import pytest
import torch

import cache_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import decode
from paper_2608_27128_gb300 import twinkv as tk
from paper_2608_27128_gb300.pages import PageCache

pytestmark = pytest.mark.gpu

L, H, D = 2, 2, 64


def rows(seed, n):
    g = torch.Generator(device=device()).manual_seed(seed)
    return (torch.randn(L, H, n, D, generator=g, device=device()).to(torch.bfloat16)
            for _ in range(2))


def held(cache, b, n):
    got = cache.read(b, n)
    return got["keys"].clone(), got["values"].clone(), got["positions"].clone()


def rounded(x):
    return torch.from_numpy(R.to_bf16(R.round_trip(x.float().cpu().numpy())))


def step(cache, seed, pos, n=1):
    """n tokens appended to both sequences in every layer; the rows, per layer."""
    g = torch.Generator(device=device()).manual_seed(seed)
    cache.reserve(n)
    got = []
    for l in range(L):
        k, v = (torch.randn(cache.B, n, H, D, generator=g, device=device()).to(torch.bfloat16)
                for _ in range(2))
        at = (pos + torch.arange(n, device=device())).int().expand(cache.B, n).contiguous()
        got.append((k, v, cache.append(l, k, v, at)))
    return got


def test_fork_append_compact_free():
    N, keep = 300, 130                                    # two full pages and two slots
    k, v = rows(1, N)
    mask = torch.zeros(L, H, N, dtype=torch.uint8, device=device())
    mask[:, :, :keep] = 1
    cache = PageCache(L, 2, H, D, n_pages=80, max_pages=5)
    assert cache.free_pages == 80
    assert cache.pack(0, k, v, mask, keep).eq(0).all()
    assert cache.free_pages == 80 - 3 * L * H
    cache.fork(0, 1)
    assert cache.free_pages == 80 - 4 * L * H             # two shared, one copied
    one = held(cache, 0, keep)
    for a, b in zip(one, held(cache, 1, keep)):
        assert torch.equal(a, b)
    np.testing.assert_array_equal(one[0].float().cpu().numpy(), rounded(k[:, :, :keep]).numpy())

    got = step(cache, 5, 1000, n=3)
    assert all(s.eq(0).all() for _, _, s in got)
    for b in range(2):
        kk, vv, pos = held(cache, b, keep + 3)
        assert torch.equal(kk[:, :, :keep], one[0]) and torch.equal(vv[:, :, :keep], one[1])
        for l in range(L):
            new = got[l][0][b].transpose(0, 1)            # [H, n, d]
            np.testing.assert_array_equal(kk[l, :, keep:].float().cpu().numpy(),
                                          rounded(new).numpy())
        assert pos[0, 0, keep:].tolist() == [1000, 1001, 1002]

    before, other = held(cache, 0, keep + 3), held(cache, 1, keep + 3)
    mask2 = torch.zeros(L, H, keep + 3, dtype=torch.uint8, device=device())
    mask2[:, :, ::2] = 1
    count = (keep + 4) // 2
    assert cache.compact(1, mask2, count).eq(0).all()
    half = held(cache, 1, count)
    for a, b in zip(half, other):
        assert torch.equal(a, b[:, :, ::2])
    for a, b in zip(held(cache, 0, keep + 3), before):
        assert torch.equal(a, b)
    assert cache.free_pages == 80 - (3 + 2) * L * H

    cache.free(0)
    assert cache.free_pages == 80 - 2 * L * H and not cache.lens[:, 0].any()
    for a, b in zip(held(cache, 1, count), half):
        assert torch.equal(a, b)
    # an empty sequence takes no tokens, and the other one does
    got = step(cache, 9, 2000)
    assert all(s[0].eq(1).all() and s[1].eq(0).all() for _, _, s in got)
    assert not cache.lens[:, 0].any() and cache.lens[:, 1].eq(count + 1).all()
    out = cache.attend(0, torch.randn(2, 1, 4, D, device=device()).to(torch.bfloat16))
    assert not out["out"][0].any() and out["out"][1].any()
    cache.free(1)
    assert cache.free_pages == 80


def test_page_boundaries_and_exhaustion():
    N = 128
    k, v = rows(2, N)
    mask = torch.ones(L, H, N, dtype=torch.uint8, device=device())
    cache = PageCache(L, 2, H, D, n_pages=3 * L * H, max_pages=3)
    cache.pack(0, k, v, mask, N)
    cache.fork(0, 1)                                      # full pages alone: nothing is copied
    assert cache.free_pages == L * H
    with pytest.raises(MemoryError):
        cache.reserve(1)                                  # both would need a page of their own
    cache.free(1)
    step(cache, 3, 500)
    assert cache.free_pages == 0 and cache.lens[:, 0].eq(N + 1).all()
    with pytest.raises(MemoryError):
        cache.fork(0, 1)                                  # its last page could not be copied
    assert cache.lens[:, 0].eq(N + 1).all() and not cache.lens[:, 1].any()
    with pytest.raises(ValueError):
        cache.pack(2, k, v, mask, N)
    with pytest.raises(ValueError):
        cache.pack(1, k, v, mask, 3 * 64 + 1)
    with pytest.raises(ValueError):
        cache.fork(0, 0)


def test_the_example_runs():
    said = []
    res = decode.demo(steps=6, N=400, say=said.append)
    torch.cuda.synchronize()
    assert len(said) == 3 and torch.isfinite(res["out"].float()).all() and res["out"].any()
    lens = res["cache"].lens
    assert lens[:, 0].eq(206).all() and lens[:, 1].eq(203).all()
    assert tk.twinkv_get_last_error() == tk.OK


def test_pack_that_does_not_fit_changes_nothing():
    k, v = rows(4, 200)
    mask = torch.ones(L, H, 200, dtype=torch.uint8, device=device())
    cache = PageCache(L, 2, H, D, n_pages=5 * L * H, max_pages=6)
    cache.pack(0, k, v, mask, 200)
    mask[:, :, 60:] = 0
    cache.pack(1, k, v, mask, 60)
    before = held(cache, 0, 200)
    with pytest.raises(MemoryError):
        cache.pack(0, k, v, mask, 300)                    # five pages a unit: four are its own
    for a, b in zip(held(cache, 0, 200), before):
        assert torch.equal(a, b)
    cache.pack(0, k, v, mask, 60)
    assert cache.free_pages == 3 * L * H
