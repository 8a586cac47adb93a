"""What attention pays to each key, over prompts and over pages, and eviction by it, on the GPU
against their definitions in 64 bits, within the bounds that prompt_reference derives."""
import numpy as np
import pytest
import torch

import cache_reference as C
import prompt_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk
from prompt_cases import Prompts
from test_gpu_cache import make_cache, put

pytestmark = pytest.mark.gpu


def log_sums(p, scale, window=0, n_sink=0):
    """float32 log denominators [T, Hq], NaN where no token is."""
    lse = np.full((p.T, p.Hq), np.nan, np.float32)
    for t, j, h, kv in p.heads():
        lse[t, h] = R.attend(p.q64[t, h], p.k64[j, kv], p.v64[j, kv], scale, window, n_sink)[1]
    return lse


def check(p, window=0, n_sink=0, last=0, carry=False, scale=None):
    dev = device()
    scale_ = p.d ** -0.5 if scale is None else scale
    lse = log_sums(p, scale_, window, n_sink)
    rng = np.random.default_rng(p.Tk)
    before = rng.random((p.H, p.Tk)).astype(np.float32) * 5
    out = {"score": torch.full((p.H, p.Tk), 7.0, device=dev)}
    score = put(before) if carry else None
    got = tk.twinkv_prompt_weights(p.q, p.k, put(lse), **p.where, scale=scale, window=window,
                                   n_sink=n_sink, last=last, score=score, out=out)
    assert tk.twinkv_get_last_error() == tk.OK
    assert got["status"].eq(0).all()
    compare(p, got["score"].double().cpu().numpy(), lse, scale_, window, n_sink, last,
            before if carry else np.zeros_like(before))
    if carry:                                         # in place
        tk.twinkv_prompt_weights(p.q, p.k, put(lse), **p.where, scale=scale, window=window,
                                 n_sink=n_sink, last=last, score=score, out={"score": score})
        key = torch.from_numpy(p.key).to(dev)
        assert torch.equal(score[:, key], got["score"][:, key])
        assert torch.equal(score[:, ~key], put(before)[:, ~key])
    return got


def compare(p, got, lse, scale, window, n_sink, last, before):
    assert (got[:, ~p.key] == 7.0).all()
    want, off = before.astype(np.float64), np.abs(before) * 2.0 ** -22
    for t, j, h, kv in p.heads():
        w, e = R.weights(p.q64[t, h], p.k64[j, kv], lse[t, h].astype(np.float64), scale, window,
                         n_sink, last)
        want[kv, j] += w
        off[kv, j] += e * (1 + 2.0 ** -20) + (p.Hq // p.H) * 2.0 ** -23 * w + 1e-37
    bad = np.abs(got - want) > off + 2.0 ** -23 * want
    assert not bad[:, p.key].any(), (np.abs(got - want)[:, p.key].max(), np.argwhere(bad)[:4])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 33, 64, 127, 128, 129, 255, 257, 600])
@pytest.mark.parametrize("last", [0, 32])
def test_lengths(d, n, last):
    check(Prompts([(n, n)], 8, 2, d, device(), seed=n), last=last)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 1), (6, 2), (5, 1), (14, 2), (33, 1), (100, 1),
                                  (128, 1)])
def test_groups(d, Hq, H):
    check(Prompts([(150, 150)], Hq, H, d, device(), seed=Hq))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["rows", "fused", "dense"])
@pytest.mark.parametrize("gap,last,carry", [(0, 0, False), (3, 0, True), (1, 16, True)])
def test_packed(d, layout, gap, last, carry):
    seqs = [(5, 5), (0, 0), (1, 1), (130, 130), (7, 300), (1, 513), (40, 25), (9, 0), (0, 12),
            (64, 200), (128, 128), (257, 257)]
    check(Prompts(seqs, 8, 2, d, device(), gap=gap, layout=layout), last=last, carry=carry)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (17, 4), (64, 130), (129, 0), (300, 4),
                                           (10000, 4)])
@pytest.mark.parametrize("last", [0, 50])
def test_windows(d, window, n_sink, last):
    check(Prompts([(420, 420), (33, 700), (3, 3)], 6, 2, d, device(), gap=1), window, n_sink, last)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m", [(1, 3000), (16, 5000), (100, 2500)])
def test_chunks_of_long_prompts(d, n, m):
    check(Prompts([(n, m)], 8, 2, d, device(), seed=m), carry=True)


@pytest.mark.parametrize("d", [64, 128])
def test_many_short_sequences(d):
    rng = np.random.default_rng(d)
    seqs = [(int(n), int(n)) for n in rng.integers(0, 4, 300)] + [(200, 200)]
    check(Prompts(seqs, 4, 2, d, device(), gap=1))


@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_sizes_of_scores(size):
    check(Prompts([(300, 300)], 4, 1, 128, device(), size=size))


def test_weights_of_a_prompt_sum_to_its_tokens():
    """With the attention's own denominators, every token and query head gives one in all."""
    dev = device()
    p = Prompts([(500, 500), (30, 900)], 8, 2, 128, dev)
    a = tk.twinkv_prompt_attend(p.q, p.k, p.v, **p.where, want_lse=True)
    s = tk.twinkv_prompt_weights(p.q, p.k, a["lse"], **p.where)["score"].double()
    for (n, m), j in zip(p.seqs, p.j0):
        sums = s[:, j:j + m].sum(1).cpu().numpy()
        # each weight within 2^-15 or so of its own (score_error at these sizes)
        np.testing.assert_allclose(sums, 4 * n, rtol=2.0 ** -13)


def test_data_errors_leave_sums_as_they_were():
    dev = device()
    p = Prompts([(20, 20)] * 4, 4, 2, 128, dev)
    lse = put(log_sums(p, 128 ** -0.5))
    for name, values, wrong in (("k_offsets", [0, 20, 10, 60, 80], [1]), ("lens", [20, 21, 20, -1],
                                                                          [1, 3]),
                                ("k_lens", [20, 20, 2 ** 31 - 1, -2 ** 31], [2, 3])):
        where = dict(p.where)
        where[name] = torch.tensor(values, dtype=torch.int32, device=dev)
        out = {"score": torch.full((2, 80), 7.0, device=dev)}
        got = tk.twinkv_prompt_weights(p.q, p.k, lse, **where, out=out)
        assert got["status"].cpu().tolist() == [int(b in wrong) for b in range(4)]
        if name != "k_offsets":
            for b in range(4):
                assert bool((got["score"][:, 20 * b:20 * b + 20] == 7.0).all()) == (b in wrong)


def test_prompt_weights_replay():
    dev = device()
    a = Prompts([(260, 260), (3, 900)], 8, 2, 128, dev, seed=1, gap=1)
    b = Prompts([(260, 260), (3, 900)], 8, 2, 128, dev, seed=2, gap=1)
    q, k, lse = a.q.clone(), a.k.clone(), put(log_sums(a, 128 ** -0.5))
    ws = tk.prompt_weights_workspace(q.shape, k.shape, 2, dev)
    out = {"score": torch.full((2, a.Tk), 7.0, device=dev)}
    out.update(tk.twinkv_prompt_weights(q, k, lse, **a.where, out=out, ws=ws))
    first = out["score"].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tk.twinkv_prompt_weights(q, k, lse, **a.where, out=out, ws=ws)
    ws.fill_(0xA5)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out["score"], first)
    log_b = log_sums(b, 128 ** -0.5)
    for x, y in ((q, b.q), (k, b.k), (lse, put(log_b))):
        x.copy_(y)
    g.replay()
    torch.cuda.synchronize()
    compare(b, out["score"].double().cpu().numpy(), log_b, 128 ** -0.5, 0, 0, 0,
            np.zeros((2, b.Tk)))


# ---------------------------------------------------------------- over pages

def cache_weights(q, lse, units, H, lens, window, n_sink, scale):
    """Sums [units][len] of the newest tokens and how far they may be off: q [B, n, Hq, d]."""
    B, n, Hq, d = q.shape
    G = Hq // H
    sums, off = [], []
    for u, (k, _, pos, _) in enumerate(units):
        b, h = divmod(u, H)
        length = len(pos)
        total, size = np.zeros(length), np.zeros(length)
        for i in range(n):
            last = length - n + i
            if last < 0:
                continue
            see = np.arange(length) <= last
            if window > 0:
                see &= (pos > pos[last] - window) | (pos < n_sink)
            for g in range(G):
                x = k @ q[b, i, h * G + g] * scale
                log = lse[b, i, h * G + g]
                w = np.where(see, np.exp(np.where(see, x - log, 0.0)), 0.0)
                # a score's float32 sums run over terms of |q| s 31 at most, and |q| s 128 once a group
                steps = np.abs(q[b, i, h * G + g]).sum() * C_STEP(units[u][0])
                e = ((31 * (d + 8) + 256) * 2.0 ** -23 * scale * steps + 2.0 ** -21
                     + 2.0 ** -22 * (np.abs(x) + abs(log)))
                total += w
                size += w * e
        sums.append(total)
        off.append(size + (n * G + 2) * 2.0 ** -23 * total)
    return sums, off


def C_STEP(k):
    """The largest scale of a group among rows of round-tripped keys, or a little more."""
    if not len(k):
        return 0.0
    g = k.reshape(len(k), -1, 64)
    return float(((np.maximum(g.max(-1), 0) - np.minimum(g.min(-1), 0)) / 14.0).max())


def check_cache(B, H, Hq, lens, n, d, window=0, n_sink=0, room=None, seed=0):
    rng = np.random.default_rng([B, H, Hq, n, d, window, seed])
    dev = device()
    unit_lens = [x for x in lens for _ in range(H)]
    pool, table, units = make_cache(rng, unit_lens, d, n_new=n)
    table, ln = table.view(B, H, -1), torch.tensor(unit_lens, dtype=torch.int32, device=dev).view(B, H)
    q = torch.from_numpy(rng.standard_normal((B, n, Hq, d))).to(torch.bfloat16)
    a = tk.twinkv_cache_attend(q.to(dev), pool, table, ln, window=window, n_sink=n_sink,
                               want_lse=True)
    N = room or max(64, max(lens) + 3)
    before = rng.random((B, H, N)).astype(np.float32) * 3
    out = {"score": torch.full((B, H, N), 7.0, device=dev)}
    got = tk.twinkv_cache_weights(q.to(dev), a["lse"], pool, table, ln, put(before), window=window,
                                  n_sink=n_sink, out=out)
    assert tk.twinkv_get_last_error() == tk.OK
    assert got["status"].eq(0).all()
    sums, off = cache_weights(q.double().numpy(), a["lse"].double().cpu().numpy(), units, H,
                              unit_lens, window, n_sink, d ** -0.5)
    s = got["score"].double().cpu().numpy().reshape(B * H, N)
    for u, length in enumerate(unit_lens):
        want = before.reshape(B * H, N)[u, :length] + sums[u]
        assert (np.abs(s[u, :length] - want) <= off[u] + 2.0 ** -22 * want).all(), \
            (u, np.abs(s[u, :length] - want).max())
        assert (s[u, length:] == 7.0).all()
    score = put(before)                               # in place
    tk.twinkv_cache_weights(q.to(dev), a["lse"], pool, table, ln, score, window=window,
                            n_sink=n_sink, out={"score": score})
    held = torch.arange(N, device=dev) < ln[..., None]
    assert torch.equal(score[held], got["score"][held])
    assert torch.equal(score[~held], put(before)[~held])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 1000])
def test_cache_lengths(d, length):
    check_cache(2, 2, 8, [length, max(1, length // 2)], 1, d, seed=length)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,H,n", [(1, 1, 1), (3, 1, 1), (4, 1, 1), (10, 2, 1), (7, 1, 2), (8, 1, 1),
                                    (16, 1, 1), (17, 1, 1), (8, 2, 7), (40, 1, 3), (4, 1, 64)])
def test_cache_rows(d, Hq, H, n):
    check_cache(1, H, Hq, [300], n, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (40, 4), (200, 130), (5000, 4)])
@pytest.mark.parametrize("n", [1, 5])
def test_cache_windows(d, window, n_sink, n):
    check_cache(3, 2, 8, [500, 37, 4], n, d, window, n_sink)


def test_cache_more_tokens_than_slots_and_empty_units():
    check_cache(3, 1, 4, [3, 0, 70], 5, 128)


def test_cache_weights_data_errors():
    """Lengths beyond the pages or the sums, pages outside the pool: that unit, or those slots, only."""
    rng = np.random.default_rng(3)
    dev = device()
    lens = [200, 130, 64, 100]
    pool, table, units = make_cache(rng, lens, 128)
    q = torch.from_numpy(rng.standard_normal((4, 1, 4, 128))).to(torch.bfloat16).to(dev)
    table = table.view(4, 1, -1).clone()
    ln = torch.tensor(lens, dtype=torch.int32, device=dev).view(4, 1)
    lse = torch.zeros(4, 1, 4, device=dev)
    before = torch.rand(4, 1, 300, device=dev)
    good = tk.twinkv_cache_weights(q, lse, pool, table, ln, before,
                                   out={"score": before.clone()})["score"]
    table[1, 0, 0] = 10 ** 6
    for value, status in ((-1, 1), (4 * 64 + 1, 1)):
        ln[0, 0] = value
        score = before.clone()
        got = tk.twinkv_cache_weights(q, lse, pool, table, ln, score, out={"score": score})
        assert got["status"].view(-1).tolist() == [status, 1, 0, 0]
        assert torch.equal(score[0], before[0])
        assert torch.equal(score[1, 0, :64], before[1, 0, :64])
        assert torch.equal(score[1, 0, 64:], good[1, 0, 64:])
        assert torch.equal(score[2:], good[2:])
    ln[0, 0] = 200
    small = before[..., :150].contiguous()
    score = small.clone()
    got = tk.twinkv_cache_weights(q, lse, pool, table, ln, score, out={"score": score})
    assert got["status"].view(-1).tolist() == [tk.ERR_TOO_LARGE, 1, 0, 0]
    assert torch.equal(score[0], small[0])


# ---------------------------------------------------------------- eviction

def check_policy(score, budget, lens=None, n_sink=4, n_recent=64, shape=None):
    units, N = score.shape
    shape = shape or (units,)
    budget = np.asarray(budget, np.int32)
    got = tk.twinkv_weight_policy(
        put(score).view(*shape, N), put(budget).view(shape),
        lens=None if lens is None else put(np.asarray(lens, np.int32)).view(shape),
        n_sink=n_sink, n_recent=n_recent, want_score=True)
    assert tk.twinkv_get_last_error() == tk.OK
    mask, kept = (got[x].cpu().numpy().reshape(units, N) for x in ("mask", "score"))
    status = got["status"].cpu().numpy().reshape(units)
    for u in range(units):
        m, k, st = R.policy(score[u], N if lens is None else int(lens[u]), int(budget[u]), n_sink,
                            n_recent)
        assert status[u] == st, u
        np.testing.assert_array_equal(mask[u], m, err_msg=str(u))
        np.testing.assert_array_equal(kept[u], k, err_msg=str(u))
    only = tk.twinkv_weight_policy(
        put(score).view(*shape, N), put(budget).view(shape),
        lens=None if lens is None else put(np.asarray(lens, np.int32)).view(shape),
        n_sink=n_sink, n_recent=n_recent)
    assert sorted(only) == ["mask", "status"] and torch.equal(only["mask"], got["mask"])


def heavy(rng, *shape):
    x = np.exp(2 * rng.standard_normal(shape) - 2).astype(np.float32)
    kind = rng.random(shape)
    x[kind < 0.1] = 0.0
    x[kind > 0.8] = np.round(4 * x[kind > 0.8]) / 4
    return x


@pytest.mark.parametrize("N", [1, 2, 5, 63, 64, 68, 69, 100, 1023, 4097, 8191, 8192, 8193, 16384,
                               40000])
def test_policy_sizes(N):
    rng = np.random.default_rng(N)
    budgets = [0, 1, N // 10, N // 2, max(0, N - 1), N]
    check_policy(heavy(rng, 6, N), budgets, shape=(2, 3))
    check_policy(heavy(rng, 6, N), budgets, lens=rng.integers(0, N + 1, 6), n_sink=0, n_recent=0)


def test_policy_ties_and_odd_values():
    rng = np.random.default_rng(1)
    N = 3000
    rows = [np.zeros(N), np.full(N, 2.5), rng.integers(0, 3, N), np.where(np.arange(N) % 2, 0.0, -0.0),
            rng.choice([np.inf, -np.inf, 0.0, 1.0], N), rng.choice([np.nan, 1.0, -1.0], N),
            np.full(N, np.nan), -heavy(rng, N), rng.choice([1e-45, -1e-45, 0.0], N),
            np.arange(N) * 1e-3, 1.0 + np.arange(N) % 4 * 2.0 ** -23]
    score = np.array(rows, np.float32)
    score[6, ::3] = -np.nan
    for budget in (1, 68, 69, 700, 1500, 2999):
        check_policy(score, [budget] * len(rows))
        check_policy(score, [budget] * len(rows), n_sink=0, n_recent=0)
    check_policy(score, [700] * len(rows), n_sink=2 ** 31 - 1, n_recent=2 ** 31 - 1)
    check_policy(score, [700] * len(rows), n_sink=10, n_recent=10 ** 6)


@pytest.mark.parametrize("N", [100, 196, 197, 4100, 16385, 40000])
def test_policy_ranges(N):
    """Scores over the whole range of floats and in the smallest corner of it, one far from all others
    among them; as few between the protected positions as are compared with one another, and one more."""
    rng = np.random.default_rng(N)
    big = np.float32(3e38)
    near = 1.0 + rng.integers(0, 2000, N) * 2.0 ** -23
    rows = [rng.standard_normal(N) * big / 8, -np.abs(rng.standard_normal(N)),
            np.where(rng.random(N) < 0.2, np.nan, -np.abs(rng.standard_normal(N)) * 1e30),
            rng.choice([np.nan, -np.inf, -big], N), rng.choice([np.inf, big], N),
            near, np.where(np.arange(N) == N // 2, np.inf, near),
            np.where(np.arange(N) == N // 2, np.nan, near),
            np.where(np.arange(N) == N // 2, -np.inf, rng.integers(0, 9, N))]
    score = np.array(rows, np.float32)
    for budget in (69, 70, N // 2, N - 7, N - 1):
        check_policy(score, [min(budget, N)] * len(rows))
    check_policy(score, [N // 3] * len(rows), n_sink=0, n_recent=0)
    check_policy(score, [N // 3] * len(rows), n_sink=N // 3 - 1, n_recent=0)


def test_policy_data_errors():
    rng = np.random.default_rng(2)
    check_policy(heavy(rng, 6, 500), [-1, 501, 100, 100, 100, 100],
                 lens=[500, 500, -1, 501, 500, 90])


def test_policy_replays_and_takes_an_int():
    dev = device()
    rng = np.random.default_rng(4)
    a, b = heavy(rng, 6, 2000), heavy(rng, 6, 2000)
    score = put(a)
    out = tk.twinkv_weight_policy(score, 900, want_score=True)
    budget = torch.full((6,), 900, dtype=torch.int32, device=dev)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tk.twinkv_weight_policy(score, budget, want_score=True, out=out)
    score.copy_(put(b))
    g.replay()
    torch.cuda.synchronize()
    for u in range(6):
        m, k, _ = R.policy(b[u], 2000, 900, 4, 64)
        np.testing.assert_array_equal(out["mask"][u].cpu().numpy(), m)
        np.testing.assert_array_equal(out["score"][u].cpu().numpy(), k)
