"""The whole way of a cache, on synthetic tensors: ``python -m paper_2608_27128_gb300.decode``.

A prompt's queries and keys are normed and rotated, the repair corrects a retained set, what it
keeps goes into pages of 4-bit codes, tokens are decoded over them from two ends (a fork), and the
cache is read back, audited, repaired and compacted again in the middle of decoding.
"""
from __future__ import annotations

import sys

import torch

from . import twinkv as tk
from .pages import PageCache


def cos_sin(rows: int, d: int, base: float = 1.0e6, device="cuda") -> torch.Tensor:
    """Cosines and sines of each position, [rows, d] float32, for twinkv_qk_norm_rope."""
    theta = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=device) / d)
    angle = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * theta
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def demo(L=2, H=2, Hq=8, N=1000, d=128, keep=0.5, steps=70, tau=0.85, seed=0, say=print) -> dict:
    """Runs the way above; returns the last step's attention outputs and the cache."""
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)

    def retained(units_n, lens, count):
        """A policy's stand-in: sinks, recent positions, and random ones up to the count."""
        score = torch.rand((L * H, units_n), generator=g, device=dev)
        at = torch.arange(units_n, device=dev)
        score[:, :4] = 2.0
        score[(at >= lens - 64) & (at < lens).expand(L * H, -1)] = 2.0
        score[(at >= lens).expand(L * H, -1)] = -1.0
        order = score.argsort(dim=1, descending=True)[:, :count]
        mask = torch.zeros((L * H, units_n), dtype=torch.uint8, device=dev).scatter_(1, order, 1)
        return mask.view(L, H, units_n)

    table = cos_sin(N + steps, d, device=dev)
    wq, wk = ((1 + 0.1 * normal(d).float()).to(torch.bfloat16) for _ in range(2))
    budget = tk.budget_for_ratio(N, 1.0 - keep)

    # the prompt: the rotated keys go straight into the dense cache that the audit reads
    keys = torch.empty((L, H, N, d), dtype=torch.bfloat16, device=dev)
    values = normal(L, H, N, d)
    positions = torch.arange(N, dtype=torch.int32, device=dev)
    for l in range(L):
        k = normal(N, H, d)
        k[N // 2:N // 2 + 50] = k[100:150]                 # near copies, so that there are twins
        tk.twinkv_qk_norm_rope(None, k, None, wk, table, positions,
                               out={"k": keys[l].transpose(0, 1)})
    repaired = tk.twinkv_repair(keys, retained(N, N, budget), None, tau)
    cache = PageCache(L, 2, H, d, n_pages=8 * L * H * (N // 64 + 3), max_pages=N // 64 + 3)
    cache.pack(0, keys, values, repaired["mask"], budget)
    say(f"packed {budget} of {N} positions per head: {cache.pool.shape[1] / 64:.0f} bytes a slot, "
        f"{4 * d} before")
    cache.fork(0, 1)

    out = None
    for step in range(steps):
        if step == steps // 2:
            # a second eviction of sequence 1, on what its pages hold
            held = budget + step
            rows = cache.read(1, held)
            again = tk.twinkv_repair(rows["keys"], retained(held, held, budget), None, tau)
            cache.compact(1, again["mask"], budget)
            say(f"sequence 1 compacted from {held} to {budget} slots, {cache.free_pages} pages free")
        cache.reserve(1)
        pos = torch.full((2, 1), N + step, dtype=torch.int32, device=dev)
        out = []
        for l in range(L):
            qkv = normal(2, Hq + 2 * H, d)
            qk = tk.twinkv_qk_norm_rope(qkv[:, :Hq], qkv[:, Hq:Hq + H], wq, wk, table,
                                        pos.view(-1))
            cache.append(l, qk["k"].view(2, 1, H, d), qkv[:, Hq + H:].view(2, 1, H, d), pos)
            out.append(cache.attend(l, qk["q"].view(2, 1, Hq, d))["out"])
    say(f"decoded {steps} tokens of two sequences: lengths {cache.lens[0, :, 0].tolist()}")
    return {"out": torch.stack(out), "cache": cache}


if __name__ == "__main__":
    demo()
    st = tk.twinkv_get_last_error()
    sys.exit(st)
