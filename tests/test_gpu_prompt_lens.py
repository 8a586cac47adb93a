"""One padded sequence: `lens` without offsets, with and without `k_lens` (GPU).  Rows behind the
sequence hold NaN, and the outputs there stay as they were."""
import numpy as np
import pytest
import torch

from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from prompt_cases import Prompts
from test_gpu_cache import put
from test_gpu_prompt import compare as compare_attention
from test_gpu_weights import compare as compare_weights, log_sums

pytestmark = pytest.mark.gpu


def one(n, m):
    return torch.tensor([n], dtype=torch.int32, device=device()), \
        torch.tensor([m], dtype=torch.int32, device=device())


def attend(p, **kw):
    given = {"out": torch.full((p.T, p.Hq, p.d), 7.0, dtype=torch.bfloat16, device=device()),
             "lse": torch.full((p.T, p.Hq), 7.0, device=device())}
    got = tk.twinkv_prompt_attend(p.q, p.k, p.v, want_lse=True, out=given, **kw)
    assert tk.twinkv_get_last_error() == tk.OK
    return got


def weights(p, lse, **kw):
    got = tk.twinkv_prompt_weights(p.q, p.k, put(lse), out={
        "score": torch.full((p.H, p.Tk), 7.0, device=device())}, **kw)
    assert tk.twinkv_get_last_error() == tk.OK
    return got


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,gap", [(1, 5), (70, 1), (100, 60), (300, 200), (1900, 100)])
def test_keys_are_as_the_tokens(d, n, gap):
    """Without k_lens a padded prompt has as many keys as tokens, not every row of k."""
    p = Prompts([(n, n)], 4, 2, d, device(), gap=gap)
    lens, _ = one(n, n)
    for kw in (dict(lens=lens), dict(lens=lens, k_lens=lens)):
        got = attend(p, **kw)
        assert got["status"].eq(0).all()
        compare_attention(p, got["out"].double().cpu().numpy(), got["lse"].double().cpu().numpy())
    lse = log_sums(p, d ** -0.5)
    for kw in (dict(lens=lens), dict(lens=lens, k_lens=lens)):
        got = weights(p, lse, **kw)
        assert got["status"].eq(0).all()
        compare_weights(p, got["score"].double().cpu().numpy(), lse, d ** -0.5, 0, 0, 0,
                        np.zeros((p.H, p.Tk)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m", [(1, 50), (33, 200), (64, 2500), (40, 25), (0, 60)])
def test_k_lens_places_a_chunk(d, n, m):
    """With k_lens a padded chunk is behind the keys before it."""
    p = Prompts([(n, m)], 4, 2, d, device(), gap=3)
    lens, k_lens = one(n, m)
    got = attend(p, lens=lens, k_lens=k_lens)
    assert got["status"].eq(0).all()
    compare_attention(p, got["out"].double().cpu().numpy(), got["lse"].double().cpu().numpy())
    lse = log_sums(p, d ** -0.5)
    got = weights(p, lse, lens=lens, k_lens=k_lens)
    compare_weights(p, got["score"].double().cpu().numpy(), lse, d ** -0.5, 0, 0, 0,
                    np.zeros((p.H, p.Tk)))


@pytest.mark.parametrize("d", [64, 128])
def test_k_lens_alone_and_k_offsets(d):
    """k_lens without lens: every row of q is a token.  k_offsets without k_lens: all of their rows."""
    p = Prompts([(40, 90)], 4, 2, d, device())
    _, k_lens = one(40, 90)
    want = attend(p)
    assert torch.equal(attend(p, k_lens=k_lens)["out"], want["out"])
    more = Prompts([(40, 90)], 4, 2, d, device(), gap=4)
    lens, _ = one(40, 90)
    at = torch.tensor([0, 90], dtype=torch.int32, device=device())
    got = attend(more, lens=lens, k_offsets=at)
    compare_attention(more, got["out"].double().cpu().numpy(), got["lse"].double().cpu().numpy())


def test_lengths_beyond_the_rows():
    """More tokens than rows of k, or of q: an error of the sequence, whose outputs stay."""
    p = Prompts([(50, 30)], 4, 2, 128, device(), gap=0)
    assert attend(p)["status"].eq(0).all()                 # every row of each
    for lens in (one(50, 50)[0], one(51, 51)[0], one(-1, -1)[0]):
        got = attend(p, lens=lens)
        assert got["status"].tolist() == [tk.ERR_INVALID_ARG]
        assert got["out"].eq(7.0).all() and got["lse"].eq(7.0).all()
        score = weights(p, np.zeros((p.T, p.Hq), np.float32), lens=lens)
        assert score["status"].tolist() == [tk.ERR_INVALID_ARG] and score["score"].eq(7.0).all()
