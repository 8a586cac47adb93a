"""The operators over prompts where items are cut among blocks and their parts joined: with many
sequences, in graphs whose inputs and lengths change, and on several streams at once (GPU)."""
import numpy as np
import pytest
import torch

import prompt_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from prompt_cases import Prompts
from test_gpu_cache import put
from test_gpu_prompt import compare as compare_attention
from test_gpu_weights import compare as compare_weights, log_sums

pytestmark = pytest.mark.gpu


class WithErrors(Prompts):
    """Prompts of which the sequences `wrong` get a length that their rows do not hold."""

    def __init__(self, seqs, Hq, H, d, device, wrong=(), seed=0):
        super().__init__(seqs, Hq, H, d, device, gap=1, seed=seed)
        self.wrong = set(wrong)
        for b in self.wrong:
            n, m = seqs[b]
            self.where["lens"][b] = n + 2 if b % 2 else -1
            self.token[self.t0[b]:self.t0[b] + n] = False
            self.key[self.j0[b]:self.j0[b] + m] = False

    def heads(self):
        at = 0
        for x in super().heads():
            if at // self.Hq not in self.wrong:
                yield x
            at += 1


def short_ones(rng, count):
    """Sequences of up to 9 tokens, a third of them empty, some with keys before their tokens."""
    n = rng.integers(0, 10, count) * (rng.random(count) > 0.33)
    return [(int(x), int(x + rng.choice([0, 0, 30]))) for x in n]


def with_long_ones(rng, count, places, long):
    seqs = short_ones(rng, count)
    for at in places:
        seqs[at] = long
    wrong = [b for b in rng.choice(count, count // 12, replace=False) if b not in places]
    return seqs, wrong


def run(p, last=0):
    """Both operators in one call each, against their definitions."""
    dev = device()
    given = {"out": torch.full((p.T, p.Hq, p.d), 7.0, dtype=torch.bfloat16, device=dev),
             "lse": torch.full((p.T, p.Hq), 7.0, device=dev)}
    B = len(p.seqs)
    want = [tk.ERR_INVALID_ARG if b in p.wrong else 0 for b in range(B)]
    ws = tk.prompt_attend_workspace(p.q.shape, p.k.shape, B, dev)
    assert ws.numel() > 256                                # parts: what the case is for
    ws.fill_(0xA5)
    got = tk.twinkv_prompt_attend(p.q, p.k, p.v, **p.where, want_lse=True, out=given, ws=ws)
    assert got["status"].tolist() == want
    compare_attention(p, got["out"].double().cpu().numpy(), got["lse"].double().cpu().numpy())
    lse = log_sums(p, p.d ** -0.5)
    ws = tk.prompt_weights_workspace(p.q.shape, p.k.shape, B, dev).fill_(0xA5)
    got = tk.twinkv_prompt_weights(p.q, p.k, put(lse), **p.where, last=last, ws=ws, out={
        "score": torch.full((p.H, p.Tk), 7.0, device=dev)})
    assert got["status"].tolist() == want
    compare_weights(p, got["score"].double().cpu().numpy(), lse, p.d ** -0.5, 0, 0, last,
                    np.zeros((p.H, p.Tk)))
    assert tk.twinkv_get_last_error() == tk.OK


# Eight heads a KV head: 16 tokens a tile, so that 120 tokens are eight tiles of columns for the weights
# (two more units beside them; items of up to 7 are never cut) and 2500 keys 20 tiles for the attention.
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("places", [(0,), (50,), (99,), (0, 99), (31, 32), (10, 63, 64)])
def test_long_sequences_among_many(d, places):
    """More than 32 sequences: the division sums them in groups first."""
    rng = np.random.default_rng([d, *places])
    seqs, wrong = with_long_ones(rng, 100, places, (120, 2500))
    run(WithErrors(seqs, 8, 1, d, device(), wrong, seed=len(places)))


@pytest.mark.parametrize("d", [64, 128])
def test_prompts_among_many(d):
    """Whole prompts of more than one item each, two KV heads."""
    rng = np.random.default_rng(d)
    seqs, wrong = with_long_ones(rng, 70, (3, 40, 69), (400, 1700))
    seqs[55] = (700, 700)
    run(WithErrors(seqs, 6, 2, d, device(), [b for b in wrong if b != 55]), last=300)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("place", [0, 4097, 8999])
def test_thousands_of_sequences(d, place):
    """So many that a group holds several times 32."""
    rng = np.random.default_rng([d, place])
    n = rng.integers(1, 4, 9000) * (rng.random(9000) > 0.9)
    seqs = [(int(x), int(x)) for x in n]
    seqs[place] = (120, 2500)
    run(WithErrors(seqs, 8, 1, d, device(), [100, 4096, 8191]))


# ---------------------------------------------------------------- graphs and streams

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["attend", "weights"])
def test_replays_with_other_lengths(d, what):
    """A graph whose inputs, offsets and lengths change in place: other items are cut elsewhere, and
    nothing is left of the parts before."""
    dev = device()
    a = Prompts([(260, 260), (90, 3000)], 8, 2, d, dev, seed=1, gap=1)
    b = Prompts([(90, 3000), (260, 260)], 8, 2, d, dev, seed=2, gap=1)
    c = Prompts([(1, 2900), (349, 360)], 8, 2, d, dev, seed=3, gap=1)
    assert a.T == b.T == c.T and a.Tk == b.Tk == c.Tk
    lse = {x: log_sums(x, d ** -0.5) for x in (a, b, c)}
    q, k, v, l = a.q.clone(), a.k.clone(), a.v.clone(), put(lse[a])
    where = {n: t.clone() for n, t in a.where.items()}
    if what == "attend":
        ws = tk.prompt_attend_workspace(q.shape, k.shape, 2, dev)
        out = {"out": torch.empty(a.T, 8, d, dtype=torch.bfloat16, device=dev),
               "lse": torch.empty(a.T, 8, device=dev),
               "status": torch.empty(2, dtype=torch.int32, device=dev)}
    else:
        ws = tk.prompt_weights_workspace(q.shape, k.shape, 2, dev)
        out = {"score": torch.empty(2, a.Tk, device=dev),
               "status": torch.empty(2, dtype=torch.int32, device=dev)}
    assert ws.numel() > 256

    def call():
        if what == "attend":
            tk.twinkv_prompt_attend(q, k, v, **where, want_lse=True, out=out, ws=ws)
        else:
            tk.twinkv_prompt_weights(q, k, l, **where, out=out, ws=ws)

    def clean():
        for n, t in out.items():
            t.fill_(7)

    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for x in (a, b, a, c, b):
        for t, y in ((q, x.q), (k, x.k), (v, x.v), (l, put(lse[x]))):
            t.copy_(y)
        for n in where:
            where[n].copy_(x.where[n])
        clean()
        ws.fill_(0xA5)                                # another call's remains
        g.replay()
        torch.cuda.synchronize()
        assert out["status"].eq(0).all()
        if what == "attend":
            compare_attention(x, out["out"].double().cpu().numpy(), out["lse"].double().cpu().numpy())
        else:
            compare_weights(x, out["score"].double().cpu().numpy(), lse[x], d ** -0.5, 0, 0, 0,
                            np.zeros((2, a.Tk)))
        first = {n: t.clone() for n, t in out.items()}
        clean()
        g.replay()                                    # on its own remains
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(first[n], t) for n, t in out.items())


@pytest.mark.parametrize("d", [64, 128])
def test_calls_on_streams_with_parts(d):
    """Prompts whose items are cut, at the same time, each call with its own workspace: the numbers of
    one call after another, bit for bit."""
    dev = device()
    T = 2300
    data = []
    for seed in range(3):
        g = torch.Generator(device=dev).manual_seed(seed)
        qkv = torch.randn(T + 100 * seed, 8 + 4, d, generator=g, device=dev).to(torch.bfloat16)
        data.append((qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]))
    assert all(tk.prompt_attend_workspace(q.shape, k.shape, 1, "cpu").numel() > 256
               for q, k, _ in data)

    def run(q, k, v, stream=None):
        a = tk.twinkv_prompt_attend(q, k, v, want_lse=True, stream=stream)
        w = tk.twinkv_prompt_weights(q, k, a["lse"], stream=stream)
        few = tk.twinkv_prompt_weights(q, k, a["lse"], last=300, window=900, n_sink=4, stream=stream)
        return [a["out"], a["lse"], w["score"], few["score"]]

    want = [run(*x) for x in data]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    for _ in range(4):
        got = [run(*x, s) for x, s in zip(data, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))
