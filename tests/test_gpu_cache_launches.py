"""The operators around the pass on streams (GPU): the first kernel of a call is fully ordered after
the caller's work, calls on two streams do not disturb one another, and captured calls replay on new
contents of their buffers."""
import numpy as np
import pytest
import torch

from gpu_harness import device
from test_gpu_first_launch import _edges
from paper_2608_27128_gb300 import twinkv as tk

pytestmark = pytest.mark.gpu

U, N, D, PAGES = 4, 600, 128, 12


def state(seed):
    g = torch.Generator(device=device()).manual_seed(seed)

    def normal(*s):
        return torch.randn(s, generator=g, device=device()).to(torch.bfloat16)

    s = {"keys": normal(1, U, N, D), "values": normal(1, U, N, D), "q": normal(1, 2, 4 * U, D),
         "k": normal(1, 2, U, D), "v": normal(1, 2, U, D),
         "mask": (torch.rand(1, U, N, generator=g, device=device()) < 0.5).to(torch.uint8)}
    ids = torch.randperm(2 * U * PAGES, generator=g, device=device()).int()
    s["table"] = ids[:U * PAGES].view(1, U, PAGES)
    s["other"] = ids[U * PAGES:].view(1, U, PAGES)
    s["pool"] = tk.cache_pool(2 * U * PAGES, D, device())
    s["pos"] = torch.full((1, 2), N, dtype=torch.int32, device=device()) + torch.arange(
        2, dtype=torch.int32, device=device())
    s["cs"] = torch.randn(N + 2, D, generator=g, device=device())
    s["ws"] = tk.cache_move_workspace(U, N + 2, device())
    s["aws"] = tk.cache_attend_workspace(s["q"].shape, U, device())
    s["out"] = {}
    return s


def step(s, stream=None):
    """Every operator once, outputs kept in s["out"]."""
    o = s["out"]

    def keep(name, got):
        o[name] = got
        return got

    kw = {"stream": stream}
    lens = keep("pack", tk.twinkv_cache_pack(s["keys"], s["values"], s["mask"], s["pool"],
                                             s["table"], ws=s["ws"], out=o.get("pack"), **kw))["lens"]
    r = keep("rope", tk.twinkv_qk_norm_rope(s["q"][0], s["k"][0], None, None, s["cs"], s["pos"][0],
                                            out=o.get("rope"), **kw))
    lens = keep("append", tk.twinkv_cache_append(r["k"][None], s["v"], s["pos"], s["pool"],
                                                 s["table"], lens, out=o.get("append"), **kw))["lens"]
    keep("attend", tk.twinkv_cache_attend(r["q"][None], s["pool"], s["table"], lens, window=300,
                                          n_sink=4, ws=s["aws"], out=o.get("attend"), **kw))
    keep("read", tk.twinkv_cache_read(s["pool"], s["table"], lens, N + 2, out=o.get("read"), **kw))
    keep("compact", tk.twinkv_cache_compact(s["pool"], s["table"], lens, s["keep"], s["other"],
                                            ws=s["ws"], out=o.get("compact"), **kw))
    keep("again", tk.twinkv_cache_read(s["pool"], s["other"], o["compact"]["lens"], N,
                                       out=o.get("again"), **kw))


def prepared(seed):
    s = state(seed)
    g = torch.Generator(device=device()).manual_seed(seed + 100)
    s["keep"] = (torch.rand(1, U, N + 2, generator=g, device=device()) < 0.4).to(torch.uint8)
    return s


def flat(s):
    return {f"{a}.{b}": t.clone() for a, d in s["out"].items() for b, t in d.items()}


def test_two_streams_at_once_equal_serial_calls():
    want = []
    for seed in (1, 2):
        s = prepared(seed)
        step(s)
        torch.cuda.synchronize()
        want.append(flat(s))
    assert want[0]["compact.lens"].min() > 50
    sets = [prepared(seed) for seed in (1, 2)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, st in zip(sets, streams):
            step(s, st)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        for name, t in flat(s).items():
            assert torch.equal(t, w[name]), name
    assert tk.twinkv_get_last_error() == tk.OK


def test_captured_calls_replay_on_new_contents():
    s = prepared(3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s)
    for seed in (4, 5, 3):
        new = prepared(seed)
        step(new)
        for name in ("keys", "values", "q", "k", "v", "mask", "table", "other", "cs", "keep"):
            s[name].copy_(new[name])
        graph.replay()
        torch.cuda.synchronize()
        want = flat(new)
        for name, t in flat(s).items():
            assert torch.equal(t, want[name]), (seed, name)


@pytest.mark.parametrize("call", ["rope", "pack", "append", "attend", "window", "read", "compact"])
def test_first_kernel_is_a_plain_launch(call):
    s = prepared(6)
    step(s)
    lens = torch.full((1, U), N, dtype=torch.int32, device=device())
    fns = {
        "rope": lambda st: tk.twinkv_qk_norm_rope(s["q"][0], s["k"][0], None, None, s["cs"],
                                                  s["pos"][0], out=s["out"]["rope"], stream=st),
        "pack": lambda st: tk.twinkv_cache_pack(s["keys"], s["values"], s["mask"], s["pool"],
                                                s["table"], ws=s["ws"], out=s["out"]["pack"],
                                                stream=st),
        "append": lambda st: tk.twinkv_cache_append(s["k"], s["v"], s["pos"], s["pool"], s["table"],
                                                    lens, out=s["out"]["append"], stream=st),
        "attend": lambda st: tk.twinkv_cache_attend(s["q"], s["pool"], s["table"], lens, ws=s["aws"],
                                                    out=s["out"]["attend"], stream=st),
        "window": lambda st: tk.twinkv_cache_attend(s["q"], s["pool"], s["table"], lens, ws=s["aws"],
                                                    window=50, out=s["out"]["attend"], stream=st),
        "read": lambda st: tk.twinkv_cache_read(s["pool"], s["table"], lens, N + 2,
                                                out=s["out"]["read"], stream=st),
        "compact": lambda st: tk.twinkv_cache_compact(s["pool"], s["table"], lens, s["keep"],
                                                      s["other"], ws=s["ws"],
                                                      out=s["out"]["compact"], stream=st),
    }
    x = torch.zeros(64, device=device())
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def fn():
        x.add_(1.0)                               # the caller's kernel: the graph's one root
        fns[call](stream)

    with torch.cuda.stream(stream):
        x.add_(1.0)
        torch.cuda.synchronize()
        edges, roots = _edges(stream, fn)
    assert len(roots) == 1 and len(edges) >= 1
    first = [t for a, _, t in edges if a == roots[0]]
    assert first and all(t == 0 for t in first), edges
    if call in ("pack", "attend", "window", "compact"):
        assert any(t == 1 for _, _, t in edges), edges
