"""Rows that the pages' rounding cannot hold (GPU): reported, and nothing else is touched."""
import numpy as np
import pytest
import torch

from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from test_gpu_cache import dirty_pool, put

pytestmark = pytest.mark.gpu

WILD = [float("nan"), float("inf"), -float("inf"), 2.0 ** 120, -2.0 ** 127]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("side", ["keys", "values"])
def test_pack_reports_rows_it_cannot_hold(d, dtype, side):
    """Status 1; the group of the value is 0, and everything else is as it would be."""
    rng = np.random.default_rng(d)
    U, N = len(WILD) + 2, 150
    good = {s: torch.from_numpy(rng.standard_normal((1, U, N, d))).to(dtype)
            for s in ("keys", "values")}
    bad = {s: x.clone() for s, x in good.items()}
    for u, value in enumerate(WILD):
        bad[side][0, u, 70 + u, 5 + u] = value
        good[side][0, u, 70 + u, :64] = 0
    for x in (good, bad):                                 # held as they are
        x[side][0, len(WILD), 3, 9], x[side][0, len(WILD), 3, 10] = 2.0 ** 119, -2.0 ** 119
    ids = put(np.arange(U * 3, dtype=np.int32).reshape(1, U, 3))
    got = []
    for x in (bad, good):
        pool = dirty_pool(U * 3, d)
        out = tk.twinkv_cache_pack(x["keys"].to(device()), x["values"].to(device()), None, pool, ids)
        assert out["lens"].eq(N).all()
        got.append((out["status"], pool))
    assert got[0][0].tolist() == [[1] * len(WILD) + [0, 0]] and got[1][0].eq(0).all()
    assert torch.equal(got[0][1], got[1][1])
    q = torch.randn(1, 1, 4 * U, d, device=device()).to(torch.bfloat16)
    lens = torch.full((1, U), N, dtype=torch.int32, device=device())
    o = tk.twinkv_cache_attend(q, got[0][1], ids, lens)["out"]
    assert torch.isfinite(o.float()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pack_does_not_look_at_rows_that_the_mask_leaves_out(dtype):
    rng = np.random.default_rng(2)
    N, d = 200, 64
    x = torch.from_numpy(rng.standard_normal((1, 2, N, d))).to(dtype).to(device())
    mask = torch.ones(1, 2, N, dtype=torch.uint8, device=device())
    mask[:, :, 100:] = 0
    x[:, :, 100:] = float("nan")
    ids = put(np.arange(4, dtype=np.int32).reshape(1, 2, 2))
    out = tk.twinkv_cache_pack(x, x, mask, dirty_pool(4, d), ids)
    assert out["status"].eq(0).all() and out["lens"].eq(100).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("side", ["k", "v"])
def test_append_reports_rows_it_cannot_hold(d, dtype, side):
    rng = np.random.default_rng(d + 1)
    H, n = len(WILD) + 1, 9
    good = {s: torch.from_numpy(rng.standard_normal((1, n, H, d))).to(dtype) for s in "kv"}
    bad = {s: x.clone() for s, x in good.items()}
    for h, value in enumerate(WILD):
        bad[side][0, h + 2, h, d - 1 - h] = value
        good[side][0, h + 2, h, d - 64:] = 0
    ids = put(np.arange(2 * H, dtype=np.int32).reshape(1, H, 2))
    pos = torch.arange(n, dtype=torch.int32, device=device()).view(1, n)
    got = []
    for x in (bad, good):
        pool = dirty_pool(2 * H, d)
        lens = torch.full((1, H), 60, dtype=torch.int32, device=device())
        out = tk.twinkv_cache_append(x["k"].to(device()), x["v"].to(device()), pos, pool, ids, lens)
        assert out["lens"].eq(60 + n).all()
        got.append((out["status"], pool))
    assert got[0][0].tolist() == [[1] * len(WILD) + [0]] and got[1][0].eq(0).all()
    assert torch.equal(got[0][1], got[1][1])
