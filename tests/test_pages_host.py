"""PageCache's bookkeeping on the host, without a GPU: the calls it makes are replaced by a model of
what they do to lengths, tables and pages (which token is in which slot of which page).

The model keeps the pool's rule: a page that a call writes is in no other unit's row from the slot
written on.  Statuses and lengths are those of include/twinkv.h."""
import pytest
import torch

from paper_2608_27128_gb300 import pages
from paper_2608_27128_gb300 import twinkv as tk

L, H, D = 2, 2, 64
SLOTS = tk.PAGE_SLOTS


class Model:
    """The pages' slots as [n_pages][64] token numbers (-1: never written)."""

    def __init__(self, monkeypatch):
        self.slots = None
        self.cache = None
        self.fresh = 0
        for name in ("pack", "append", "compact", "read"):
            monkeypatch.setattr(tk, f"twinkv_cache_{name}", getattr(self, name))

    def make(self, *a, **kw):
        self.cache = pages.PageCache(*a, **kw, device="cpu")
        self.slots = torch.full((self.cache.pool.shape[0], SLOTS), -1, dtype=torch.int64)
        return self.cache

    def token(self):
        self.fresh += 1
        return self.fresh

    def whose(self, page, slot):
        """Units whose rows hold the page and whose length is past the slot, by device lengths."""
        t, n = self.cache.table, self.cache.lens
        at = (t == page).nonzero().tolist()
        return [tuple(u) for *u, j in at if n[tuple(u)] > 64 * j + slot]

    def held(self, b):
        """Tokens of sequence b, per (layer, head)."""
        c = self.cache
        out = {}
        for l in range(c.L):
            for h in range(c.H):
                n = int(c.lens[l, b, h])
                out[l, h] = [int(self.slots[c.table[l, b, h, i // 64], i % 64])
                             for i in range(max(n, 0))]
        return out

    # ------------------------------------------------------------ the calls

    def _fill(self, rows, table, lens, status, u, limit):
        """rows: token numbers of one unit into the pages of table[u]."""
        row = table[u].tolist()
        if len(rows) > limit * SLOTS:
            status[u], lens[u] = 7, 0
            return
        if any(not 0 <= p < self.slots.shape[0] for p in row[:-(-len(rows) // SLOTS)]):
            status[u], lens[u] = 1, 0
            return
        for i, x in enumerate(rows):
            self.slots[row[i // SLOTS], i % SLOTS] = x
        lens[u] = len(rows)

    def pack(self, keys, values, mask, pool, table, **kw):
        if keys.dim() != 4 or keys.shape[:2] != table.shape[:2] or keys.shape[3] != D:
            raise ValueError("keys")
        if mask is not None and (mask.shape != keys.shape[:3] or mask.dtype is not torch.uint8):
            raise ValueError("mask")
        lens = torch.zeros(table.shape[:2], dtype=torch.int32)
        status = torch.zeros_like(lens)
        for l in range(table.shape[0]):
            for h in range(table.shape[1]):
                m = mask[l, h] if mask is not None else torch.ones(keys.shape[2])
                if (m > 1).any():
                    status[l, h] = 1
                    continue
                self._fill([self.token() for _ in range(int(m.sum()))], table, lens, status, (l, h),
                           table.shape[-1])
        return {"lens": lens, "status": status}

    def append(self, k, v, positions, pool, table, lens, *, out=None, **kw):
        n, new = k.shape[1], (out or {}).get("lens", torch.empty_like(lens))
        status = torch.zeros_like(lens)
        writes = []
        for b in range(table.shape[0]):
            for h in range(table.shape[1]):
                at, row = int(lens[b, h]), table[b, h].tolist()
                if at < 0:
                    status[b, h] = 1
                elif at + n > len(row) * SLOTS:
                    status[b, h] = 7
                elif any(not 0 <= row[i // SLOTS] < self.slots.shape[0] for i in (at, at + n - 1)):
                    status[b, h] = 1
                if status[b, h]:
                    new[b, h] = at
                    continue
                writes += [(b, h, row[i // SLOTS], i % SLOTS) for i in range(at, at + n)]
        places = [w[2:] for w in writes]
        assert len(set(places)) == len(places), "two units of one launch write the same slot"
        for b, h, page, slot in writes:
            assert not self.whose(page, slot), "a slot in use is written"
            self.slots[page, slot] = self.token()
        for u in {w[:2] for w in writes}:
            new[u] = int(lens[u]) + n
        return {"lens": new, "status": status}

    def compact(self, pool, table, lens, keep, new_table, **kw):
        if keep is not None and (keep.dtype is not torch.uint8 or keep.shape[:-1] != lens.shape):
            raise ValueError("keep")
        got = torch.zeros_like(lens)
        status = torch.zeros_like(lens)
        N = keep.shape[-1] if keep is not None else table.shape[-1] * SLOTS
        for u in [tuple(x) for x in torch.cartesian_prod(*map(torch.arange, lens.shape)).view(
                -1, lens.dim()).tolist()]:
            n = int(lens[u])
            if not 0 <= n <= min(N, table.shape[-1] * SLOTS):
                status[u] = 1
                continue
            rows = [int(self.slots[table[u][i // SLOTS], i % SLOTS]) for i in range(n)
                    if keep is None or keep[u][i]]
            self._fill(rows, new_table, got, status, u, new_table.shape[-1])
        return {"lens": got, "status": status}

    def read(self, *a, **kw):
        raise AssertionError("not modelled")


@pytest.fixture
def model(monkeypatch):
    return Model(monkeypatch)


def dense(n):
    x = torch.zeros(L, H, n, D, dtype=torch.bfloat16)
    return x, x


def ones(n, total=None):
    m = torch.zeros(L, H, total or n, dtype=torch.uint8)
    m[:, :, :n] = 1
    return m


def step(cache, n=1):
    cache.reserve(n)
    k = torch.zeros(cache.B, n, H, D, dtype=torch.bfloat16)
    pos = torch.zeros(cache.B, n, dtype=torch.int32)
    return [cache.append(l, k, k, pos) for l in range(L)]


def test_the_model_follows_a_fork(model):
    cache = model.make(L, 2, H, D, 60, 5)
    cache.pack(0, *dense(200), ones(130, 200), 130)
    cache.fork(0, 1)
    before = model.held(0)
    assert model.held(1) == before and all(len(x) == 130 for x in before.values())
    for _ in range(70):
        assert all(s.eq(0).all() for s in step(cache))
    a, b = model.held(0), model.held(1)
    for u in before:
        assert a[u][:130] == b[u][:130] == before[u] and a[u][130:] != b[u][130:]


# ---------------------------------------------------------------- counts and lengths

@pytest.mark.parametrize("kept,budget", [(100, 128), (100, 130), (140, 130), (0, 64), (64, 63)])
def test_a_pack_that_misses_its_budget_is_an_error(model, kept, budget):
    """No page of such a unit is read or written any more, whatever follows."""
    cache = model.make(L, 2, H, D, 60, 5)
    status = cache.pack(0, *dense(200), ones(kept, 200), budget)
    assert status.ne(0).all() and cache.lens[:, 0].eq(-1).all()
    pages_before = model.slots.clone()
    for _ in range(3):
        assert all(s.ne(0).all() for s in step(cache))
    assert torch.equal(model.slots, pages_before) and cache.lens[:, 0].eq(-1).all()
    with pytest.raises(RuntimeError):
        cache.fork(0, 1)
    assert cache.pack(0, *dense(200), ones(70, 200), 70).eq(0).all()
    cache.fork(0, 1)
    assert cache.lens.eq(70).all()
    cache.free(0), cache.free(1)
    assert cache.free_pages == 60


def test_one_unit_that_misses_its_budget_leaves_the_others(model):
    cache = model.make(L, 2, H, D, 60, 5)
    mask = ones(100, 200)
    mask[1, 0, 50] = 0
    status = cache.pack(0, *dense(200), mask, 100)
    assert status.tolist() == [[0, 0], [1, 0]]
    assert cache.lens[:, 0].tolist() == [[100, 100], [-1, 100]]
    assert [s[0].tolist() for s in step(cache)] == [[0, 0], [1, 0]]


def test_a_mask_with_a_data_error(model):
    """The unit has no slots on the device, and its host count is not taken for its length."""
    cache = model.make(L, 2, H, D, 60, 5)
    mask = ones(130, 200)
    mask[0, 1, 3] = 2
    assert cache.pack(0, *dense(200), mask, 130).tolist() == [[0, 1], [0, 0]]
    with pytest.raises(RuntimeError):
        cache.fork(0, 1)
    assert [s[0].tolist() for s in step(cache)] == [[0, 1], [0, 0]]


def test_a_compact_that_misses_its_budget_is_an_error(model):
    cache = model.make(L, 2, H, D, 60, 5)
    cache.pack(0, *dense(200), ones(200), 200)
    keep = ones(100, 200)
    keep[0, 0, 150] = 1
    assert cache.compact(0, keep, 100).tolist() == [[1, 0], [0, 0]]
    assert cache.lens[:, 0].tolist() == [[-1, 100], [100, 100]]
    with pytest.raises(RuntimeError):
        cache.fork(0, 1)


def test_fork_in_the_middle_of_a_step(model):
    """Between reserve and the layers' appends the host counts slots that are not written yet."""
    cache = model.make(L, 2, H, D, 60, 5)
    cache.pack(0, *dense(200), ones(127, 200), 127)
    free = cache.free_pages
    cache.reserve(1)                                 # 128: two full pages by the host's count
    with pytest.raises(RuntimeError):
        cache.fork(0, 1)
    k = torch.zeros(2, 1, H, D, dtype=torch.bfloat16)
    pos = torch.zeros(2, 1, dtype=torch.int32)
    cache.append(0, k, k, pos)
    with pytest.raises(RuntimeError):
        cache.fork(0, 1)
    assert cache.free_pages == free and not cache.lens[:, 1].any()
    cache.append(1, k, k, pos)
    cache.fork(0, 1)
    assert cache.lens.eq(128).all()
    for _ in range(3):
        assert all(s.eq(0).all() for s in step(cache))


# ---------------------------------------------------------------- calls that raise

def state(cache):
    return (sorted(cache._free), list(cache._users), {u: list(x) for u, x in cache._pages.items()},
            dict(cache._used), cache.table.clone(), cache.lens.clone())


def same(a, b):
    return a[:4] == b[:4] and torch.equal(a[4], b[4]) and torch.equal(a[5], b[5])


def bad_dense(n):
    x = torch.zeros(L, H, n, D + 1, dtype=torch.bfloat16)
    return x, x


@pytest.mark.parametrize("full", [False, True])
def test_a_pack_that_raises_changes_nothing(model, full):
    """The arguments are refused by the call, after the host has chosen pages."""
    cache = model.make(L, 2, H, D, 4 * L * H if full else 60, 5)
    cache.pack(0, *dense(200), ones(200), 200)
    before, held = state(cache), model.held(0)
    for args in ((*bad_dense(200), ones(200), 200), (*dense(200), ones(200).float(), 200),
                 (*dense(200), ones(200)[:1], 100)):
        with pytest.raises(ValueError):
            cache.pack(0, *args)
    if full:
        with pytest.raises(MemoryError):
            cache.pack(0, *dense(320), ones(320), 320)
    assert same(state(cache), before) and model.held(0) == held


def test_a_compact_that_raises_loses_no_pages(model):
    cache = model.make(L, 2, H, D, 60, 5)
    cache.pack(0, *dense(200), ones(200), 200)
    before, held = state(cache), model.held(0)
    for keep in (ones(200).float(), ones(200)[:1]):
        with pytest.raises(ValueError):
            cache.compact(0, keep, 100)
    assert same(state(cache), before) and model.held(0) == held
    cache.free(0)
    assert cache.free_pages == 60


def test_fork_onto_a_sequence_uses_its_pages(model):
    """The target's own pages are free for the copy, as they are for pack."""
    cache = model.make(L, 2, H, D, 5 * L * H, 5)
    cache.pack(0, *dense(200), ones(130, 200), 130)
    cache.pack(1, *dense(200), ones(100, 200), 100)
    assert cache.free_pages == 0
    held = model.held(0)
    cache.fork(0, 1)
    assert model.held(1) == held and model.held(0) == held
    assert cache.free_pages == L * H
    cache.fork(1, 0)                                  # and back, over pages that the two share
    assert model.held(1) == held and model.held(0) == held
    cache.free(0), cache.free(1)
    assert cache.free_pages == 5 * L * H


# ---------------------------------------------------------------- units without slots

def test_a_head_that_keeps_nothing_takes_the_next_tokens(model):
    """A budget of 0 for one head of a sequence: its new tokens are stored like the others'."""
    cache = model.make(L, 2, H, D, 60, 5)
    mask = ones(70, 200)
    mask[1, 1] = 0
    assert cache.pack(0, *dense(200), mask, [70, 70, 70, 0]).eq(0).all()
    cache.fork(0, 1)
    for _ in range(66):
        assert all(s.eq(0).all() for s in step(cache))
    assert cache.lens.tolist() == [[[136, 136]] * 2, [[136, 66]] * 2]
    a, b = model.held(0), model.held(1)
    assert not set(a[1, 1]) & set(b[1, 1]) and len(set(a[1, 1])) == 66
    keep = torch.zeros(L, H, 136, dtype=torch.uint8)
    assert cache.compact(0, keep, 0).eq(0).all()
    assert all(s.eq(0).all() for s in step(cache))
    assert cache.lens[:, 0].eq(1).all() and cache.lens[1, 1].tolist() == [137, 67]


def test_a_sequence_that_starts_without_slots(model):
    cache = model.make(L, 2, H, D, 60, 5)
    assert cache.pack(0, *dense(5), ones(0, 5), 0).eq(0).all()
    assert cache.free_pages == 60
    for _ in range(2):
        assert [s.tolist() for s in step(cache)] == [[[0, 0], [1, 1]]] * L
    assert cache.lens[:, 0].eq(2).all() and not cache.lens[:, 1].any()
    cache.free(0)
    assert cache.free_pages == 60
    assert [s.tolist() for s in step(cache)] == [[[1, 1], [1, 1]]] * L
    assert cache.free_pages == 60
