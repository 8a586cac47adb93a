"""What the newest tokens' attention pays to the slots of a serving batch: many units, of so many pages
that every warp of the grid takes several, of different units (GPU).  The reference is in 64 bits on
the GPU, from the definition of the pages' codes."""
import functools

import numpy as np
import pytest
import torch

import cache_reference as C
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk

pytestmark = pytest.mark.gpu

PAGE = 64


def round_trip(rows):
    """What 4 bits leave of rows [..., d] in float64, and the groups' scales (cache_reference.quantize)."""
    g = rows.double().reshape(*rows.shape[:-1], rows.shape[-1] // 64, 64)
    lo, hi = g.amin(-1).clamp(max=0.0), g.amax(-1).clamp(min=0.0)
    # nearest bf16 by the bits of a double: 7 of its 52 bits stay, ties to even
    bits = ((hi - lo) / 15.0).view(torch.int64)
    bits = (bits + (1 << 44) - 1 + (bits >> 45 & 1)) >> 45 << 45
    s = bits.view(torch.float64)
    s = torch.where(s < 2.0 ** -126, 0.0, s)
    step = torch.where(s > 0, s, 1.0)
    z = torch.where(s > 0, torch.round(-lo / step).clamp(max=15), 0.0)
    c = torch.where(s[..., None] > 0,
                    (torch.round(g / step[..., None]) + z[..., None]).clamp(max=15), 0.0)
    return ((c - z[..., None]) * s[..., None]).reshape(rows.shape), s


class Batch:
    """Units of the given lengths in pages that a pack wrote, positions with gaps."""

    def __init__(self, B, H, lens, d, seed):
        dev = device()
        self.B, self.H, self.d, self.lens = B, H, d, lens
        g = torch.Generator(device=dev).manual_seed(seed)
        most = max(lens)
        rows = most + most // 4 + 1
        keys = torch.randn(B, H, rows, d, generator=g, device=dev).to(torch.bfloat16)
        keys[..., torch.randperm(d, generator=g, device=dev)[:3]] *= 6
        # every unit keeps its length's worth of rows, wherever they are, the last ones side by side
        want = torch.tensor(lens, device=dev).view(B, H, 1)
        order = torch.rand(B, H, rows, generator=g, device=dev)
        at = torch.arange(rows, device=dev)
        order = torch.where((at >= rows - 80).expand_as(order), 2.0 + at / rows, order)
        rank = order.argsort(-1, descending=True).argsort(-1)
        mask = (rank < want).to(torch.uint8)
        pages = -(-most // PAGE)
        ids = torch.randperm(B * H * pages + 3, generator=g, device=dev)[:B * H * pages]
        self.table = ids.to(torch.int32).view(B, H, pages).contiguous()
        self.pool = tk.cache_pool(B * H * pages + 3, d, dev)
        self.pool.fill_(0xFF)                                # every scale that nothing writes is a NaN
        out = tk.twinkv_cache_pack(keys, keys, mask, self.pool, self.table)
        assert out["status"].eq(0).all()
        self.ln = out["lens"]
        assert self.ln.view(-1).tolist() == list(lens)
        self.units = [(keys.view(B * H, rows, d)[u][mask.view(B * H, rows)[u].bool()],
                       mask.view(B * H, rows)[u].nonzero().view(-1)) for u in range(B * H)]
        k, s = round_trip(self.units[max(range(B * H), key=lambda u: lens[u])][0][:200])
        np.testing.assert_array_equal(
            k.cpu().numpy(), C.round_trip(self.units[max(range(B * H), key=lambda u: lens[u])][0][:200]
                                          .double().cpu().numpy()))

    def sums(self, q, window, n_sink, absent):
        """lse [B, n, Hq] float32, and per unit the sums and how far they may be off (as in
        test_gpu_weights.cache_weights).  absent: page numbers of units that are outside the pool."""
        B, n, Hq, d = q.shape
        G, dev, scale = Hq // self.H, q.device, d ** -0.5
        lse = torch.full((B, n, Hq), -float("inf"), device=dev)
        sums, off = [], []
        for u, (k, pos) in enumerate(self.units):
            b, h = divmod(u, self.H)
            length = len(pos)
            k, s = round_trip(k)
            rows = q[b, :, h * G:(h + 1) * G].double().reshape(n * G, d)
            x = k @ rows.T * scale                                           # [len, n G]
            own = length - n + torch.arange(n, device=dev)
            slot = torch.arange(length, device=dev)[:, None]
            see = slot <= own[None]
            if window > 0 and length:
                last = pos[own.clamp(min=0)]
                see &= (pos[:, None] > last[None] - window) | (pos[:, None] < n_sink)
            for j in absent.get(u, ()):
                see[PAGE * j:PAGE * j + PAGE] = False
            see = see.repeat_interleave(G, 1)
            log = torch.logsumexp(torch.where(see, x, -float("inf")), 0) if length else torch.full(
                (n * G,), -float("inf"), device=dev, dtype=torch.float64)
            lse[b, :, h * G:(h + 1) * G] = log.float().view(n, G)
            log = log.float().double()
            w = torch.where(see, torch.exp(torch.where(see, x - log, 0.0)), 0.0)
            steps = rows.abs().sum(-1) * (s.amax() if length else 0.0)
            e = ((31 * (d + 8) + 256) * 2.0 ** -23 * scale * steps[None] + 2.0 ** -21
                 + 2.0 ** -22 * (x.abs() + torch.where(see, log.abs(), 0.0)))
            total = w.sum(-1)
            sums.append(total)
            off.append((w * e).sum(-1) + (n * G + 2) * 2.0 ** -23 * total)
        return lse, sums, off


def lengths(rng, units, most):
    """Of all sizes, a tenth of them none, and what ends a page or half of one among them."""
    n = rng.integers(1, most + 1, units)
    n[rng.random(units) < 0.1] = 0
    for i, x in enumerate((1, 31, 32, 33, 63, 64, 65, most, most - 1, 64 * (most // 64))):
        n[rng.integers(units) if i else 0] = x
    return [int(x) for x in n]


@functools.lru_cache(maxsize=None)
def serving(d):
    return Batch(20, 2, lengths(np.random.default_rng(d), 40, 80000), d, d)


@functools.lru_cache(maxsize=None)
def crowd(d):
    return Batch(275, 4, lengths(np.random.default_rng(d), 1100, 700), d, d)


def check(batch, G, n, window=0, n_sink=0, absent=None):
    dev = device()
    absent = absent or {}
    B, H, d = batch.B, batch.H, batch.d
    g = torch.Generator(device=dev).manual_seed(G * n)
    q = torch.randn(B, n, H * G, d, generator=g, device=dev).to(torch.bfloat16)
    lse, sums, off = batch.sums(q, window, n_sink, absent)
    table = batch.table.clone()
    for u, pages in absent.items():
        table.view(B * H, -1)[u, list(pages)] = torch.tensor([-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1] * len(
            pages), dtype=torch.int32, device=dev)[:len(pages)]
    N = max(batch.lens) + 5
    before = torch.rand(B, H, N, generator=g, device=dev) * 3
    given = {"score": torch.full((B, H, N), 7.0, device=dev)}
    got = tk.twinkv_cache_weights(q, lse, batch.pool, table, batch.ln, before, window=window,
                                  n_sink=n_sink, out=given)
    assert tk.twinkv_get_last_error() == tk.OK
    assert got["status"].view(-1).tolist() == [int(bool(absent.get(u))) for u in range(B * H)]
    score, old = got["score"].view(B * H, N), before.view(B * H, N)
    for u, length in enumerate(batch.lens):
        want = old[u, :length].double() + sums[u]
        bad = (score[u, :length].double() - want).abs() > off[u] + 2.0 ** -22 * want
        assert not bad.any(), (u, length, bad.nonzero()[:4].tolist())
        assert score[u, length:].eq(7.0).all(), u
        for j in absent.get(u, ()):                     # as they were
            assert torch.equal(score[u, 64 * j:64 * j + 64][:max(0, length - 64 * j)],
                               old[u, 64 * j:64 * j + 64][:max(0, length - 64 * j)])
    again = before.clone()                              # in place
    tk.twinkv_cache_weights(q, lse, batch.pool, table, batch.ln, again, window=window, n_sink=n_sink,
                            out={"score": again})
    held = torch.arange(N, device=dev) < batch.ln[..., None]
    assert torch.equal(again[held], got["score"][held]) and torch.equal(again[~held], before[~held])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (3, 1), (4, 2), (7, 1), (4, 4), (4, 18)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (3000, 130)])
def test_a_serving_batch(d, G, n, window, n_sink):
    """40 units of up to 1250 pages: the warps' rings go round, and spans pass from unit to unit."""
    batch = serving(d)
    assert sum(-(-x // PAGE) for x in batch.lens) > 16000
    check(batch, G, n, window, n_sink)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 2), (4, 4)])
def test_a_serving_batch_with_pages_outside_the_pool(d, G, n):
    """Their slots keep their sums; a ring's place without keys is not taken for one with them."""
    batch = serving(d)
    rng = np.random.default_rng(d)
    absent = {}
    for u in range(0, 40, 3):
        pages = -(-batch.lens[u] // PAGE)
        if pages > 2:
            absent[u] = sorted(rng.choice(pages - 1, max(1, pages // 5), replace=False).tolist())
    check(batch, G, n, absent=absent)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(4, 1), (4, 2), (4, 4)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (200, 4)])
def test_more_units_than_a_scan_holds(d, G, n, window, n_sink):
    """1100 units: more than 32 groups of 32, whose pages are summed in several rounds."""
    check(crowd(d), G, n, window, n_sink)
