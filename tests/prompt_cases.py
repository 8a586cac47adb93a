"""Packed prompts for the tests of the operators over them."""
import numpy as np
import torch


class Prompts:
    """Sequences of (tokens, keys), with `gap` rows that are no sequence's behind each, and rows of
    NaN wherever no token or key is.  `layout`: "fused" (views of one projection), "dense" (keys and values
    [H, rows, d]), "rows" (contiguous)."""

    def __init__(self, seqs, Hq, H, d, device, gap=0, layout="rows", seed=0, size=1.0):
        rng = np.random.default_rng([seed, Hq, H, d, len(seqs), gap])
        self.seqs, self.Hq, self.H, self.d = seqs, Hq, H, d
        self.t0 = np.cumsum([0] + [n + gap for n, _ in seqs])
        self.j0 = np.cumsum([0] + [m + 2 * gap for _, m in seqs])
        T, Tk = max(1, int(self.t0[-1]) + gap), max(1, int(self.j0[-1]) + gap)
        self.T, self.Tk = T, Tk
        q = np.full((T, Hq, d), np.nan)
        k, v = np.full((Tk, H, d), np.nan), np.full((Tk, H, d), np.nan)
        for (n, m), t, j in zip(seqs, self.t0, self.j0):
            q[t:t + n] = rng.standard_normal((n, Hq, d)) * size
            k[j:j + m] = rng.standard_normal((m, H, d)) * rng.choice([1.0, 4.0], d, p=[0.95, 0.05])
            v[j:j + m] = rng.standard_normal((m, H, d))
        q, k, v = (torch.from_numpy(x).to(torch.bfloat16) for x in (q, k, v))
        self.q64, self.k64, self.v64 = (x.double().numpy() for x in (q, k, v))
        if layout == "fused":
            rows = max(T, Tk)
            qkv = torch.full((rows, Hq + 2 * H, d), float("nan"), dtype=torch.bfloat16)
            qkv[:T, :Hq], qkv[:Tk, Hq:Hq + H], qkv[:Tk, Hq + H:] = q, k, v
            qkv = qkv.to(device)
            self.q, self.k, self.v = qkv[:T, :Hq], qkv[:Tk, Hq:Hq + H], qkv[:Tk, Hq + H:]
        elif layout == "dense":
            self.q = q.transpose(0, 1).contiguous().to(device).transpose(0, 1)
            self.k, self.v = (x.transpose(0, 1).contiguous().to(device).transpose(0, 1)
                              for x in (k, v))
        else:
            self.q, self.k, self.v = q.to(device), k.to(device), v.to(device)

        def ints(x):
            return torch.tensor([int(y) for y in x], dtype=torch.int32, device=device)

        self.where = dict(offsets=ints(self.t0), k_offsets=ints(self.j0), lens=None, k_lens=None)
        if gap:
            self.where.update(lens=ints([n for n, _ in seqs]), k_lens=ints([m for _, m in seqs]))
        self.token = np.zeros(T, bool)
        self.key = np.zeros(Tk, bool)
        for (n, m), t, j in zip(seqs, self.t0, self.j0):
            self.token[t:t + n] = True
            self.key[j:j + m] = True

    def heads(self):
        """Per sequence and query head: token rows, key rows, head, KV head."""
        for (n, m), t, j in zip(self.seqs, self.t0, self.j0):
            for h in range(self.Hq):
                yield slice(t, t + n), slice(j, j + m), h, h // (self.Hq // self.H)
