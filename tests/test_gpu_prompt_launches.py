"""The first kernel of each of the operators that make a retained set is a plain launch, later ones are
its dependents (see test_gpu_first_launch)."""
import pytest
import torch

from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from test_gpu_first_launch import _edges

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["attend", "weights", "cache", "cache_window", "policy"])
def test_first_kernel_is_a_plain_launch(call):
    dev = device()
    T, Hq, H, d = 2000, 8, 2, 128          # items that blocks share, which a second kernel joins
    q = torch.randn(T, Hq, d, device=dev).to(torch.bfloat16)
    k, v = (torch.randn(T, H, d, device=dev).to(torch.bfloat16) for _ in range(2))
    lse = torch.zeros(T, Hq, device=dev)
    pool, table = tk.cache_pool(8, d, dev), torch.arange(8, dtype=torch.int32, device=dev).view(1, 2, 4)
    lens = torch.full((1, 2), 200, dtype=torch.int32, device=dev)
    score, budget = torch.rand(1, 2, 256, device=dev), torch.full((1, 2), 100, dtype=torch.int32,
                                                                  device=dev)
    x = torch.zeros(64, device=dev)
    one, small = q[:1].unsqueeze(0), torch.zeros(1, 1, Hq, device=dev)
    fns = {
        "attend": lambda **kw: tk.twinkv_prompt_attend(
            q, k, v, ws=tk.prompt_attend_workspace(q.shape, k.shape, 1, dev) if not kw else ws, **kw),
        "weights": lambda **kw: tk.twinkv_prompt_weights(
            q, k, lse, ws=tk.prompt_weights_workspace(q.shape, k.shape, 1, dev) if not kw else ws,
            **kw),
        "cache": lambda **kw: tk.twinkv_cache_weights(one, small, pool, table, lens, score, **kw),
        "cache_window": lambda **kw: tk.twinkv_cache_weights(
            one, small, pool, table, lens, score, window=50, ws=ws, **kw),
        "policy": lambda **kw: tk.twinkv_weight_policy(score, budget, **kw),
    }
    ws = {"attend": lambda: tk.prompt_attend_workspace(q.shape, k.shape, 1, dev),
          "weights": lambda: tk.prompt_weights_workspace(q.shape, k.shape, 1, dev),
          "cache_window": lambda: tk.cache_weights_workspace(one.shape, H, dev)}.get(call, lambda: None)()
    out = fns[call]()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def fn():
        x.add_(1.0)                               # the caller's kernel: the graph's one root
        fns[call](stream=s, out=out)

    with torch.cuda.stream(s):
        x.add_(1.0)
        torch.cuda.synchronize()
        edges, roots = _edges(s, fn)
    assert len(roots) == 1 and len(edges) >= 1
    first = [t for a, _, t in edges if a == roots[0]]
    assert first and all(t == 0 for t in first), edges
    if call in ("attend", "weights", "cache_window"):
        assert any(t == 1 for _, _, t in edges), edges


def test_operators_on_streams_of_their_own():
    """Prompts, weights, pages and policies at the same time, each with its own workspace."""
    dev = device()
    g = torch.Generator(device=dev).manual_seed(0)

    def make(seed):
        g.manual_seed(seed)
        qkv = torch.randn(900, 8 + 4, 64, generator=g, device=dev).to(torch.bfloat16)
        q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
        score = torch.rand(4, 3000, generator=g, device=dev)

        def run(stream=None):
            a = tk.twinkv_prompt_attend(q, k, v, want_lse=True, stream=stream)
            w = tk.twinkv_prompt_weights(q, k, a["lse"], stream=stream)
            p = tk.twinkv_weight_policy(score, 1000, want_score=True, stream=stream)
            return [a["out"], a["lse"], w["score"], p["mask"], p["score"]]

        return run

    runs = [make(s) for s in range(3)]
    want = [r() for r in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(4):
        got = [r(s) for r, s in zip(runs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))
