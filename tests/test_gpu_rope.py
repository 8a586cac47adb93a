"""Norms with rotation on the GPU against the formula in 64 bits.

Bounds.  The sum of at most 128 squares in float32, the reciprocal root (2 ulp) and the products come to
less than 16 roundings of 2^-24 on each of the two terms of an output: 2^-20 (|a| + |b|).  bf16
outputs are rounded once more: 2^-8 relative (8 significant bits)."""
import numpy as np
import pytest
import torch

import cache_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk

pytestmark = pytest.mark.gpu
EPS = 1e-6


def table(rows, d):
    theta = 1e6 ** (-2.0 * np.arange(d // 2) / d)
    a = np.arange(rows)[:, None] * theta
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1)).float().to(device())


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def check(got, x, w, cs, pos):
    want, size = R.norm_rope(f64(x), None if w is None else f64(w), f64(cs), pos, EPS)
    bound = 2.0 ** -20 * size
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    assert (np.abs(f64(got) - want) <= bound + 1e-37).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,Hq,H,norm", [(1, 32, 8, True), (1, 1, 1, False), (7, 5, 1, True),
                                         (130, 12, 4, False), (2000, 9, 3, True)])
def test_rope(dtype, d, T, Hq, H, norm):
    g = torch.Generator(device=device()).manual_seed(T + d)
    qkv = torch.randn(T, Hq + 2 * H, d, generator=g, device=device()).to(dtype)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + H]
    q[0, 0] = 0
    w = [(torch.randn(d, generator=g, device=device()) + 1).to(dtype) if norm else None
         for _ in range(2)]
    cs = table(3001, d)
    pos = torch.randint(0, 3001, (T,), generator=g, device=device(), dtype=torch.int32)
    out = tk.twinkv_qk_norm_rope(q, k, *w, cs, pos, eps=EPS)
    p = pos.cpu().numpy()
    check(out["q"], q, w[0], cs, p)
    check(out["k"], k, w[1], cs, p)
    assert out["status"].eq(0).all()


def test_in_place_one_side_and_into_a_dense_cache():
    d, T, N = 128, 50, 300
    x = torch.randn(T, 6, d, device=device()).to(torch.bfloat16)
    keys = torch.zeros(6, N, d, dtype=torch.bfloat16, device=device())   # [H, N, d] of a cache
    cs, pos = table(N, d), torch.arange(20, 20 + T, dtype=torch.int32, device=device())
    ref = tk.twinkv_qk_norm_rope(x, None, None, None, cs, pos)
    assert "k" not in ref
    view = keys[:, 20:20 + T].transpose(0, 1)
    got = tk.twinkv_qk_norm_rope(None, x, None, None, cs, pos, out={"k": view})
    assert got["k"].data_ptr() == view.data_ptr() and torch.equal(view, ref["q"])
    assert not keys[:, :20].any() and not keys[:, 20 + T:].any()
    y = x.clone()
    tk.twinkv_qk_norm_rope(y, None, None, None, cs, pos, out={"q": y})
    assert torch.equal(y, ref["q"])


def test_positions_outside_the_table():
    d = 64
    x = torch.randn(5, 2, d, device=device())
    cs = table(10, d)
    pos = torch.tensor([0, 10, -1, 9, 2 ** 31 - 1], dtype=torch.int32, device=device())
    out = tk.twinkv_qk_norm_rope(x, x, None, None, cs, pos)
    assert out["status"].tolist() == [0, 1, 1, 0, 1]
    assert not out["q"][[1, 2, 4]].any() and not out["k"][[1, 2, 4]].any()
    ok = [0, 3]
    check(out["q"][ok], x[ok], None, cs, pos.cpu().numpy()[ok])
