"""PageCache.evict where the scores do not fit the cache, or the policy reports an error (host only, the
model of test_pages_host)."""
import pytest
import torch

from paper_2608_27128_gb300 import twinkv as tk
from test_pages_evict_host import model  # noqa: F401
from test_pages_host import D, H, L, same, state


def falling(N):
    """Scores that fall from slot to slot (the model's policy does not look at lengths)."""
    return torch.arange(N).float().flip(0).expand(L, H, N).contiguous()


def packed(model, lengths=(150, 150, 150, 150)):  # noqa: F811
    c = model.make(L, 2, H, D, n_pages=60, max_pages=4)
    N = 200
    mask = torch.zeros(L, H, N, dtype=torch.uint8)
    for u, n in enumerate(lengths):
        mask.view(L * H, N)[u, :n] = 1
    k = torch.zeros(L, H, N, D)
    assert not c.pack(0, k, k, mask, list(lengths)).any()
    return c


@pytest.mark.parametrize("shape", [(L, H, 149), (L, H, 100), (L, H), (H, L + 1, 200), (L, H, 200, 1),
                                   (L * H, 200), (L, 1, H, 200)])
def test_scores_that_do_not_fit_are_refused(model, shape):  # noqa: F811
    """A length that is longer than N would leave the unit without slots: refused before anything
    changes, also where one unit alone is."""
    c = packed(model, (20, 150, 70, 0))
    before, rows = state(c), model.held(0)
    with pytest.raises(ValueError):
        c.evict(0, torch.zeros(shape), 10)
    assert same(before, state(c)) and model.held(0) == rows
    with pytest.raises((ValueError, TypeError)):
        c.evict(0, None, 10)
    assert same(before, state(c)) and model.held(0) == rows
    assert not c.evict(0, falling(150), 10)["status"].any()      # the longest unit's
    assert c.lens[:, 0].flatten().tolist() == [10, 10, 10, 0]


def test_the_policys_errors_are_reported(model, monkeypatch):  # noqa: F811
    """Its status where it has one, else the compaction's."""
    c = packed(model)
    plain = tk.twinkv_weight_policy

    def policy(score, budget, **kw):
        out = plain(score, budget, **kw)
        out["status"][0, 1] = tk.ERR_TOO_LARGE
        out["mask"][0, 1] = 0
        out["mask"][1, 0, 149] ^= 1                  # one more or less than the budget
        return out

    monkeypatch.setattr(tk, "twinkv_weight_policy", policy)
    got = c.evict(0, falling(256), 70)
    assert got["status"].tolist() == [[0, tk.ERR_TOO_LARGE], [tk.ERR_INVALID_ARG, 0]]
    assert c.lens[:, 0].tolist() == [[70, -1], [-1, 70]]
