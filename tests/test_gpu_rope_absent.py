"""Norms with rotation of tokens whose position is outside the table (GPU)."""
import pytest
import torch

from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_a_position_outside_the_table_gives_zeros_with_norms(dtype, d, eps):
    """Whatever the weights and the table hold."""
    x = torch.randn(5, 3, d, device=device()).to(dtype)
    w = torch.full((d,), 2.0, device=device(), dtype=dtype)
    w[0], w[d - 1] = float("inf"), float("nan")
    cs = torch.randn(10, d, device=device())
    cs[0] = float("nan")
    pos = torch.tensor([3, 10, -1, 9, 2 ** 31 - 1], dtype=torch.int32, device=device())
    out = tk.twinkv_qk_norm_rope(x, x, w, w, cs, pos, eps=eps)
    assert out["status"].tolist() == [0, 1, 1, 0, 1]
    for name in ("q", "k"):
        assert out[name][[1, 2, 4]].eq(0).all()
        assert torch.isfinite(out[name][[0, 3]][..., 1:d // 2 - 1]).all()
