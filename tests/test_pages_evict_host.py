"""PageCache.evict's bookkeeping on the host, without a GPU (the model of test_pages_host)."""
import pytest
import torch

from paper_2608_27128_gb300 import twinkv as tk
from test_pages_host import D, H, L, Model


@pytest.fixture
def model(monkeypatch):
    m = Model(monkeypatch)
    compact = m.compact if hasattr(m, "compact") else None

    def policy(score, budget, *, lens=None, n_sink=None, n_recent=None, want_score=False, **kw):
        assert lens.shape == budget.shape == score.shape[:-1] and want_score
        order = score.argsort(dim=-1, descending=True, stable=True)
        rank = order.argsort(dim=-1)
        mask = (rank < budget[..., None]).to(torch.uint8)
        m.asked = budget.clone()
        return {"mask": mask, "status": torch.zeros_like(budget),
                "score": torch.zeros_like(score)}

    monkeypatch.setattr(tk, "twinkv_weight_policy", policy)
    assert compact is not None
    return m


def test_evict_keeps_the_budget_or_all(model):
    c = model.make(L, 2, H, D, n_pages=60, max_pages=4)
    N = 150
    k = torch.zeros(L, H, N, D)
    mask = torch.ones(L, H, N, dtype=torch.uint8)
    c.pack(0, k, k, mask, N)
    free = c.free_pages
    score = torch.arange(256).float().flip(0).expand(L, H, 256).contiguous()
    before = model.held(0)
    got = c.evict(0, score, 70)
    assert model.asked.eq(70).all() and not got["status"].any()
    assert c.lens[:, 0].eq(70).all()
    assert all(x == before[u][:70] for u, x in model.held(0).items())
    assert c.free_pages == free + L * H               # three pages a unit before, two now
    c.evict(0, score, 200)                            # more than there is
    assert model.asked.eq(70).all() and c.lens[:, 0].eq(70).all()
    c.evict(0, score, [10, 20, 30, 200])
    assert model.asked.flatten().tolist() == [10, 20, 30, 70]
    with pytest.raises(ValueError):
        c.evict(0, score, 5000)
    with pytest.raises(ValueError):
        c.evict(7, score, 10)
