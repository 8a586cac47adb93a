"""Attention over prompts on the GPU against its definition in 64 bits, within the bounds that
prompt_reference derives."""
import numpy as np
import pytest
import torch

import prompt_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from prompt_cases import Prompts

pytestmark = pytest.mark.gpu


def check(p, scale=None, **kw):
    """One call against the reference, rows that are no token's included; returns its outputs."""
    dev = device()
    out = {"out": torch.full((p.T, p.Hq, p.d), 7.0, dtype=torch.bfloat16, device=dev),
           "lse": torch.full((p.T, p.Hq), 7.0, device=dev)}
    got = tk.twinkv_prompt_attend(p.q, p.k, p.v, **p.where, scale=scale, want_lse=True, out=out,
                                  **kw)
    assert tk.twinkv_get_last_error() == tk.OK
    assert got["status"].eq(0).all()
    compare(p, got["out"].double().cpu().numpy(), got["lse"].double().cpu().numpy(), scale, **kw)
    return got


def compare(p, out, lse, scale=None, **kw):
    assert (out[~p.token] == 7.0).all() and (lse[~p.token] == 7.0).all()
    scale = p.d ** -0.5 if scale is None else scale
    for t, j, h, kv in p.heads():
        want, log, off, off_log = R.attend(p.q64[t, h], p.k64[j, kv], p.v64[j, kv], scale, **kw)
        a, b = out[t, h], lse[t, h]
        assert np.isfinite(a).all()
        assert (np.abs(a - want) <= off).all(), (t, h, np.abs(a - want).max(), off.max())
        none = np.isinf(log)
        assert (b[none] == -np.inf).all() and (a[none] == 0).all()
        assert (np.abs(b - log)[~none] <= off_log[~none]).all(), (t, h)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 600])
def test_lengths(d, n):
    check(Prompts([(n, n)], 8, 2, d, device(), seed=n))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (2, 2), (3, 1), (6, 2), (5, 1), (14, 2), (8, 1), (33, 1),
                                  (64, 1), (100, 1), (128, 1)])
def test_groups(d, Hq, H):
    check(Prompts([(150, 150)], Hq, H, d, device(), seed=Hq))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["rows", "fused", "dense"])
@pytest.mark.parametrize("gap", [0, 3])
def test_packed(d, layout, gap):
    """Sequences of all kinds in one call: empty ones, one token, chunks, more tokens than keys."""
    seqs = [(5, 5), (0, 0), (1, 1), (130, 130), (7, 300), (1, 513), (40, 25), (9, 0), (0, 12),
            (64, 200), (128, 128), (257, 257)]
    check(Prompts(seqs, 8, 2, d, device(), gap=gap, layout=layout))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (17, 0), (17, 4), (64, 130), (128, 4),
                                           (129, 0), (300, 4), (10000, 4), (200, 10000)])
def test_windows(d, window, n_sink):
    check(Prompts([(420, 420), (33, 700), (3, 3)], 6, 2, d, device(), gap=1), window=window,
          n_sink=n_sink)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m", [(1, 3000), (2, 9001), (16, 5000), (64, 4097), (100, 2500)])
def test_chunks_of_long_prompts(d, n, m):
    """Few tokens over many keys."""
    check(Prompts([(n, m)], 8, 2, d, device(), seed=m))
    check(Prompts([(n, m), (3, 40)], 8, 2, d, device(), seed=m, gap=2), window=1500, n_sink=4)


@pytest.mark.parametrize("d", [64, 128])
def test_shared_items(d):
    """Prompts whose items of all lengths are cut where the division falls, odd groups among them."""
    check(Prompts([(1700, 1700), (40, 40)], 6, 2, d, device(), seed=3))
    check(Prompts([(130, 130), (1, 1601), (1900, 1950)], 4, 1, d, device(), seed=4, gap=3), window=700,
          n_sink=130)


@pytest.mark.parametrize("d", [64, 128])
def test_many_short_sequences(d):
    rng = np.random.default_rng(d)
    seqs = [(int(n), int(n)) for n in rng.integers(0, 4, 300)] + [(200, 200)]
    check(Prompts(seqs, 4, 2, d, device(), gap=1))


@pytest.mark.parametrize("size,scale", [(1e-3, None), (30.0, None), (1.0, 1e-6), (8.0, 1.0)])
def test_sizes_of_scores(size, scale):
    """From weights that are all alike to a single one."""
    check(Prompts([(300, 300)], 4, 1, 128, device(), size=size), scale=scale)


def test_scores_that_rise_and_fall():
    """Running maxima that change with every key, by little and by much, and never again."""
    p = Prompts([(700, 700)], 2, 1, 64, device())
    for sign, step in ((1, 0.5), (1, 0.004), (-1, 0.5)):
        k = torch.zeros(p.Tk, 1, 64)
        k[:, 0, 0] = sign * step * torch.arange(p.Tk)
        q = torch.zeros(p.T, 2, 64)
        q[:, 0, 0], q[:, 1, 0] = 8.0, -8.0
        k, q = k.to(torch.bfloat16), q.to(torch.bfloat16)
        p.k, p.q, p.k64, p.q64 = k.to(device()), q.to(device()), k.double().numpy(), q.double().numpy()
        check(p)


@pytest.mark.parametrize("d", [64, 128])
def test_without_offsets_and_without_lse(d):
    """One sequence of every row, a chunk where k has more; only the outputs asked for."""
    p = Prompts([(70, 190)], 4, 2, d, device())
    want = check(p)
    got = tk.twinkv_prompt_attend(p.q, p.k, p.v)
    assert sorted(got) == ["out", "status"]
    assert torch.equal(got["out"], want["out"])
    # the tokens' offsets stand for the keys' too
    p = Prompts([(70, 70), (5, 5)], 4, 2, d, device())
    want = check(p)
    got = tk.twinkv_prompt_attend(p.q, p.k, p.v, p.where["offsets"])
    assert torch.equal(got["out"], want["out"])


def test_data_errors_leave_rows_as_they_were():
    """Offsets and lengths that lie outside the rows: that sequence only."""
    dev = device()
    p = Prompts([(20, 20)] * 4, 4, 2, 128, dev)
    bad = {"offsets": [[0, 20, 10, 60, 80], [0, 20, 40, 60, 99], [-5, 20, 40, 60, 80]],
           "k_offsets": [[0, 20, 10, 60, 80], [0, 20, 40, 60, 99], [-5, 20, 40, 60, 80]],
           "lens": [[20, 21, 20, -1]], "k_lens": [[20, 20, 2 ** 31 - 1, -2 ** 31]]}
    wrong = [[1], [3], [0], [1], [3], [0], [1, 3], [2, 3]]
    at = iter(wrong)
    for name, lists in bad.items():
        for values in lists:
            where = dict(p.where)
            where[name] = torch.tensor(values, dtype=torch.int32, device=dev)
            out = {"out": torch.full((80, 4, 128), 7.0, dtype=torch.bfloat16, device=dev),
                   "lse": torch.full((80, 4), 7.0, device=dev)}
            got = tk.twinkv_prompt_attend(p.q, p.k, p.v, **where, want_lse=True, out=out)
            status = got["status"].cpu().tolist()
            expect = next(at)
            assert [b for b in range(4) if status[b] == tk.ERR_INVALID_ARG] == expect, (name, values)
            if name != "offsets":
                for b in range(4):
                    rows = got["out"][20 * b:20 * b + 20].float()
                    assert bool((rows == 7.0).all()) == (b in expect), (name, values, b)


def test_calls_repeat_and_replay():
    """The same numbers from call to call, from a graph, and on new contents of the same buffers."""
    dev = device()
    a = Prompts([(260, 260), (3, 900)], 8, 2, 128, dev, seed=1, gap=1)
    b = Prompts([(260, 260), (3, 900)], 8, 2, 128, dev, seed=2, gap=1)
    ws = tk.prompt_attend_workspace(a.q.shape, a.k.shape, 2, dev)
    q, k, v = a.q.clone(), a.k.clone(), a.v.clone()
    out = {}
    out.update(tk.twinkv_prompt_attend(q, k, v, **a.where, want_lse=True, ws=ws))
    first = [out[x].clone() for x in ("out", "lse")]
    for x in ("out", "lse"):
        out[x].fill_(7.0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tk.twinkv_prompt_attend(q, k, v, **a.where, want_lse=True, out=out, ws=ws)
    ws.fill_(0xA5)                                    # another call's remains
    g.replay()
    torch.cuda.synchronize()
    for rows in ("token",):
        t = torch.from_numpy(a.token).to(dev)
        assert torch.equal(out["out"][t], first[0][t]) and torch.equal(out["lse"][t], first[1][t])
    for x, y in ((q, b.q), (k, b.k), (v, b.v)):
        x.copy_(y)
    g.replay()
    torch.cuda.synchronize()
    compare(b, out["out"].double().cpu().numpy(), out["lse"].double().cpu().numpy())


def test_two_streams_at_once():
    dev = device()
    p = [Prompts([(500, 500)], 8, 2, 128, dev, seed=s) for s in (1, 2)]
    want = [tk.twinkv_prompt_attend(x.q, x.k, x.v)["out"] for x in p]
    streams = [torch.cuda.Stream() for _ in p]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [tk.twinkv_prompt_attend(x.q, x.k, x.v, stream=s)["out"] for x, s in zip(p, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
