"""PageCache (GPU): sequences whose lengths are not what the host counted, and heads without slots."""
import numpy as np
import pytest
import torch

import cache_reference as R
from gpu_harness import device
from paper_2608_27128_gb300.pages import PageCache
from test_gpu_cache import f64

pytestmark = pytest.mark.gpu


def test_page_cache_refuses_a_mask_of_another_size():
    L, H, D, N = 2, 2, 64, 300
    x = torch.randn(L, H, N, D, device=device()).to(torch.bfloat16)
    mask = torch.zeros(L, H, N, dtype=torch.uint8, device=device())
    mask[:, :, :130] = 1
    mask[1, 0, 40] = 0
    cache = PageCache(L, 2, H, D, n_pages=60, max_pages=5)
    assert cache.pack(0, x, x, mask, 130).tolist() == [[0, 0], [1, 0]]
    assert cache.lens[:, 0].tolist() == [[130, 130], [-1, 130]]
    with pytest.raises(RuntimeError):
        cache.fork(0, 1)
    cache.reserve(1)
    k = torch.randn(2, 1, H, D, device=device()).to(torch.bfloat16)
    pos = torch.full((2, 1), N, dtype=torch.int32, device=device())
    before = cache.pool[cache.table[1, 0, 0][:3].long()].clone()
    got = [cache.append(l, k, k, pos)[0].tolist() for l in range(L)]
    assert got == [[0, 0], [1, 0]]
    assert torch.equal(cache.pool[cache.table[1, 0, 0][:3].long()], before)
    out = cache.attend(1, torch.randn(2, 1, 8, D, device=device()).to(torch.bfloat16))
    assert out["status"][0].tolist() == [1, 0] and not out["out"][0, 0, :4].any()
    assert out["out"][0, 0, 4:].any()
    mask[1, 0, 40] = 1
    assert cache.pack(0, x, x, mask, 130).eq(0).all()
    cache.fork(0, 1)
    cache.reserve(1)
    with pytest.raises(RuntimeError):
        cache.fork(0, 1)
    assert all(cache.append(l, k, k, pos).eq(0).all() for l in range(L))
    assert cache.lens.eq(131).all()


def test_page_cache_head_without_slots():
    L, H, D, N = 1, 2, 128, 200
    x = torch.randn(L, H, N, D, device=device()).to(torch.bfloat16)
    mask = torch.zeros(L, H, N, dtype=torch.uint8, device=device())
    mask[:, 0, :70] = 1
    cache = PageCache(L, 1, H, D, n_pages=20, max_pages=5)
    assert cache.pack(0, x, x, mask, [70, 0]).eq(0).all()
    q = torch.randn(1, 1, 4, D, device=device()).to(torch.bfloat16)
    k = torch.randn(1, 1, H, D, device=device()).to(torch.bfloat16)
    v = torch.randn(1, 1, H, D, device=device()).to(torch.bfloat16)
    cache.reserve(1)
    assert cache.append(0, k, v, torch.full((1, 1), N, dtype=torch.int32, device=device())).eq(0).all()
    assert cache.lens.tolist() == [[[71, 1]]]
    out = f64(cache.attend(0, q)["out"])[0, 0, 2:]
    want = R.round_trip(f64(v)[0, 0, 1])
    # one slot: its probability is 1, its value rounded as a product (2^-11) and as an output
    assert (np.abs(out - want) <= 2.0 ** -7 * np.abs(want)).all()
