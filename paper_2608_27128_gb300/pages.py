"""A cache in pages of 4-bit codes, as a serving loop keeps it between calls.

``PageCache`` holds the pool, the page tables and the lengths of L layers, B sequences and H KV
heads, and hands out pages on the host: taking, sharing, copying and freeing them.  The repair
keeps exactly its budget (Sec. 3.4), so the host knows every unit's pages without asking the
device.  A unit that does not hold its budget after all (another mask, a data error) gets length -1,
a data error for every call: none of its pages is read or written until the sequence is packed
anew or freed.  Only fork, which shares pages by the host's counts, waits for the device and
compares them.  The computation is in ``twinkv``'s calls, which the methods make on the current stream; a
page that is free again may be written by the next call on it, so a cache stays on one stream.
"""
from __future__ import annotations

from itertools import islice

import torch

from . import twinkv as tk

SLOTS = tk.PAGE_SLOTS


class PageCache:
    """Pages for L layers, B sequences, H KV heads of dimension d; at most max_pages a unit."""

    def __init__(self, L: int, B: int, H: int, d: int, n_pages: int, max_pages: int,
                 device="cuda"):
        self.L, self.B, self.H, self.d, self.max_pages = L, B, H, d, max_pages
        self.pool = tk.cache_pool(n_pages, d, device)
        # -1: no page, which no call reads or writes
        self.table = torch.full((L, B, H, max_pages), -1, dtype=torch.int32,
                                device=self.pool.device)
        self.lens = torch.zeros((L, B, H), dtype=torch.int32, device=self.pool.device)
        self._free = list(range(n_pages - 1, -1, -1))
        self._users = [0] * n_pages
        self._pages = {(l, b, h): [] for l in range(L) for b in range(B) for h in range(H)}
        self._used = dict.fromkeys(self._pages, 0)
        self._live = [False] * B             # packed or forked, and not freed since

    # ------------------------------------------------------------ pages, on the host

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def _pick(self, need, back=()) -> list:
        """Lists of so many pages each, of those that are free and those that the units `back`
        alone hold.  They are not taken before _hold is called with them."""
        own = [i for u in back for i in self._pages[u] if self._users[i] == 1]
        n, free = sum(need), len(self._free) + len(own)
        if n > free:
            raise MemoryError(f"{n} pages wanted, {free} are free")
        own = own[:n]
        ids = own + self._free[len(self._free) - (n - len(own)):]
        ids = iter(ids)
        return [list(islice(ids, n)) for n in need]

    def _hold(self, units, lists):
        """The units hold these pages from now on, instead of those they held."""
        before = [i for u in units for i in self._pages[u]]
        taken = 0
        for u, x in zip(units, lists):
            for i in x:
                taken += self._users[i] == 0
                self._users[i] += 1
            self._pages[u] = x
        del self._free[len(self._free) - taken:]     # where _pick found them
        self._drop(before)

    def _drop(self, pages):
        for i in pages:
            self._users[i] -= 1
            if self._users[i] == 0:
                self._free.append(i)

    def _sequence(self, b):
        if not 0 <= b < self.B:
            raise ValueError(f"sequence must be in [0, {self.B})")
        return [(l, b, h) for l in range(self.L) for h in range(self.H)]

    def _counts(self, count, units) -> list:
        """A number of slots per unit: from an int, or a list or tensor of L*H."""
        if isinstance(count, torch.Tensor):
            count = count.reshape(-1).tolist()
        count = [int(count)] * len(units) if isinstance(count, int) else [int(x) for x in count]
        if len(count) != len(units):
            raise ValueError(f"{len(units)} counts wanted, got {len(count)}")
        if any(not 0 <= x <= self.max_pages * SLOTS for x in count):
            raise ValueError(f"counts must be in [0, {self.max_pages * SLOTS}]")
        return count

    def _rows(self, lists) -> torch.Tensor:
        """Table rows [len(lists), max_pages] of lists of pages."""
        rows = [x + [-1] * (self.max_pages - len(x)) for x in lists]
        return torch.tensor(rows, dtype=torch.int32).to(self.pool.device)

    def _set(self, units, lists):
        self._hold(units, lists)
        at = torch.tensor([(l * self.B + b) * self.H + h for l, b, h in units],
                          device=self.pool.device)
        self.table.view(-1, self.max_pages)[at] = self._rows(lists)

    def _filled(self, b, units, counts, out):
        """Lengths and statuses of sequence b after the call that filled its pages: -1 and an error
        where the call failed or a unit has not the slots that the host counts."""
        want = torch.tensor(counts, dtype=torch.int32).view(self.L, self.H).to(self.pool.device)
        wrong = (out["lens"] != want) | (out["status"] != 0)
        self.lens[:, b] = out["lens"].masked_fill(wrong, -1)
        self._used.update(zip(units, counts))
        self._live[b] = True
        return out["status"].masked_fill(wrong & (out["status"] == 0), tk.ERR_INVALID_ARG)

    # ------------------------------------------------------------ one sequence

    def pack(self, b: int, keys, values, mask, budget):
        """Sequence b becomes the rows of keys, values [L,H,N,d] that mask [L,H,N] retains;
        budget: how many that are per unit, as the repair was given it (an int, or L*H).  Returns
        the statuses [L,H]: 1 where the mask retains another number."""
        units = self._sequence(b)
        counts = self._counts(budget, units)
        lists = self._pick([-(-n // SLOTS) for n in counts], units)
        out = tk.twinkv_cache_pack(keys, values, mask, self.pool,
                                   self._rows(lists).view(self.L, self.H, -1))
        self._set(units, lists)
        return self._filled(b, units, counts, out)

    def read(self, b: int, rows: int) -> dict:
        """The first ``rows`` slots of sequence b: keys, values [L,H,rows,d] bf16, positions."""
        return tk.twinkv_cache_read(self.pool, self.table[:, b].contiguous(),
                                    self.lens[:, b].contiguous(), rows)

    def compact(self, b: int, keep, budget):
        """Sequence b keeps the slots that keep [L,H,N] marks, ``budget`` per unit, in new pages;
        statuses as pack's."""
        units = self._sequence(b)
        counts = self._counts(budget, units)
        lists = self._pick([-(-n // SLOTS) for n in counts])
        out = tk.twinkv_cache_compact(self.pool, self.table[:, b].contiguous(),
                                      self.lens[:, b].contiguous(), keep,
                                      self._rows(lists).view(self.L, self.H, -1))
        self._set(units, lists)
        return self._filled(b, units, counts, out)

    def evict(self, b: int, score, budget, *, n_sink=None, n_recent=None) -> dict:
        """Sequence b keeps, per unit, the budget's worth of slots with the highest score
        [L,H,N] float32 (N at least the longest unit, else ValueError), sinks and recent ones first
        (twinkv_weight_policy), in new pages; a unit with fewer slots keeps all of them.  Between steps:
        not after a reserve whose appends are still to come.  Returns a dict: status [L,H], the
        policy's or, where that is 0, as pack's; mask [L,H,N], and score [L,H,N], the kept slots' in
        order."""
        units = self._sequence(b)
        counts = [min(n, self._used[u]) for n, u in zip(self._counts(budget, units), units)]
        # a unit longer than its scores would be a data error, and lose its slots
        most = max(self._used[u] for u in units)
        if (not isinstance(score, torch.Tensor) or score.dim() != 3
                or score.shape[:2] != (self.L, self.H) or score.shape[2] < most):
            raise ValueError(f"score must be [{self.L}, {self.H}, N], N at least {most}")
        want = torch.tensor(counts, dtype=torch.int32).view(self.L, self.H).to(self.pool.device)
        out = tk.twinkv_weight_policy(score, want, lens=self.lens[:, b].contiguous(), n_sink=n_sink,
                                      n_recent=n_recent, want_score=True)
        policy = out["status"]
        out["status"] = torch.where(policy != 0, policy, self.compact(b, out["mask"], counts))
        return out

    def fork(self, b: int, to: int):
        """Sequence ``to`` becomes another end of sequence b: full pages are shared, the last
        one is copied, so that either may append.  Waits for the device, and raises RuntimeError
        between a reserve and the last layer's append, or where a pack or compact failed: what the
        host takes for full pages would be written again."""
        units, others = self._sequence(b), self._sequence(to)
        if b == to:
            raise ValueError("a sequence is no fork of itself")
        if self.lens[:, b].flatten().tolist() != [self._used[u] for u in units]:
            raise RuntimeError(f"sequence {b} does not hold the slots counted for it: a step is not "
                               "over, or a call on it failed")
        part = [u for u in units if self._used[u] % SLOTS]
        own = dict(zip(part, self._pick([1] * len(part), others)))
        lists = [self._pages[u][:self._used[u] // SLOTS] + own.get(u, []) for u in units]
        self._set(others, lists)
        self.lens[:, to] = self.lens[:, b]
        self._used.update(zip(others, (self._used[u] for u in units)))
        self._live[to] = self._live[b]
        if part:
            dev = self.pool.device
            last = torch.tensor([[self._pages[u][self._used[u] // SLOTS]] for u in part],
                                dtype=torch.int32).to(dev)
            new = torch.tensor([own[u] for u in part], dtype=torch.int32).to(dev)
            held = torch.tensor([self._used[u] % SLOTS for u in part], dtype=torch.int32).to(dev)
            tk.twinkv_cache_compact(self.pool, last, held, None, new)

    def free(self, b: int):
        """Sequence b is empty; pages that no other sequence shares are free again."""
        units = self._sequence(b)
        for u in units:
            self._drop(self._pages[u])
            self._pages[u], self._used[u] = [], 0
        self._live[b] = False
        self.table[:, b] = -1
        self.lens[:, b] = 0

    # ------------------------------------------------------------ one step of every sequence

    def reserve(self, n: int = 1):
        """Pages for n more slots of every sequence that was packed or forked, and not freed since
        (of all its units, also those without slots): once per step, before its layers append."""
        if not 1 <= n <= SLOTS:
            raise ValueError(f"n must be in [1, {SLOTS}]")
        want, lists = {}, []
        for u, pages in self._pages.items():
            need = -(-(self._used[u] + n) // SLOTS) - len(pages)
            if self._live[u[1]] and need > 0:
                if len(pages) + need > self.max_pages:
                    raise MemoryError(f"unit {u} has {self.max_pages} pages already")
                want[u] = need
        for u, new in zip(want, self._pick(want.values())):
            lists.append(self._pages[u] + new)
        if want:
            self._set(list(want), lists)
        for u, used in self._used.items():
            if self._live[u[1]]:
                self._used[u] = used + n

    def append(self, layer: int, k, v, positions):
        """The rows k, v [B,n,H,d] of the step's tokens behind one layer's slots (after reserve(n));
        a sequence that is not live stays empty, with status 1."""
        lens = self.lens[layer]
        return tk.twinkv_cache_append(k, v, positions, self.pool, self.table[layer], lens,
                                      out={"lens": lens})["status"]

    def attend(self, layer: int, q, **kw) -> dict:
        """Attention of the step's queries q [B,n,Hq,d] over one layer (twinkv_cache_attend)."""
        return tk.twinkv_cache_attend(q, self.pool, self.table[layer], self.lens[layer], **kw)

    def weigh(self, layer: int, q, lse, score, **kw):
        """Adds what the attention of the step's queries pays to each slot of one layer to score
        [B,H,N] float32, in place (twinkv_cache_weights); lse as attend gave it.  Returns the
        statuses."""
        return tk.twinkv_cache_weights(q, lse, self.pool, self.table[layer], self.lens[layer], score,
                                       out={"score": score}, **kw)["status"]
