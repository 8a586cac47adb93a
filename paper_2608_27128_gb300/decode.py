"""The whole way of a cache, on synthetic tensors: ``python -m paper_2608_27128_gb300.decode``.

A prompt's queries and keys are normed and rotated and its attention computed, what that pays to
each key decides a retained set, which the repair corrects, and what it keeps goes into pages of
4-bit codes.  Tokens are decoded over them from two ends (a fork), their attention adding to the
sums, and the cache is read back, evicted, audited, repaired and compacted again in the middle of
decoding.
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
    """Runs the way above; returns the last step's attention outputs, the cache and the sums."""
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)

    def kept(score, mask):
        """The sums at the positions that mask keeps, budget per unit."""
        return score[mask.bool()].view(L, H, budget)

    table = cos_sin(N + steps, d, device=dev)
    wq, wk = ((1 + 0.1 * normal(d).float()).to(torch.bfloat16) for _ in range(2))
    budget = tk.budget_for_ratio(N, 1.0 - keep)

    # the prompt: the rotated keys go straight into the dense cache that the audit reads; the last 32
    # tokens' attention decides what is retained
    keys = torch.empty((L, H, N, d), dtype=torch.bfloat16, device=dev)
    values = normal(L, H, N, d)
    score = torch.empty((L, H, N), dtype=torch.float32, device=dev)
    positions = torch.arange(N, dtype=torch.int32, device=dev)
    for l in range(L):
        k0 = normal(N, H, d)
        k0[N // 2:N // 2 + 50] = k0[100:150]               # near copies, so that there are twins
        k, v = keys[l].transpose(0, 1), values[l].transpose(0, 1)
        q = tk.twinkv_qk_norm_rope(normal(N, Hq, d), k0, wq, wk, table, positions,
                                   out={"k": k})["q"]
        a = tk.twinkv_prompt_attend(q, k, v, want_lse=True)
        tk.twinkv_prompt_weights(q, k, a["lse"], last=32, out={"score": score[l]})
    repaired = tk.twinkv_repair(keys, tk.twinkv_weight_policy(score, budget)["mask"], None, tau)
    cache = PageCache(L, 2, H, d, n_pages=8 * L * H * (N // 64 + 3), max_pages=N // 64 + 3)
    cache.pack(0, keys, values, repaired["mask"], budget)
    say(f"packed {budget} of {N} positions per head: {cache.pool.shape[1] / 64:.0f} bytes a slot, "
        f"{4 * d} before")
    cache.fork(0, 1)
    sums = torch.zeros((L, 2, H, cache.max_pages * 64), dtype=torch.float32, device=dev)
    sums[:, :, :, :budget] = kept(score, repaired["mask"])[:, None]

    out = None
    for step in range(steps):
        if step == steps // 2:
            # a second eviction of sequence 1, on what its pages hold
            held = budget + step
            rows = cache.read(1, held)
            old = sums[:, 1, :, :held].contiguous()
            policy = tk.twinkv_weight_policy(old, budget)
            again = tk.twinkv_repair(rows["keys"], policy["mask"], None, tau)
            cache.compact(1, again["mask"], budget)
            sums[:, 1] = 0.0
            sums[:, 1, :, :budget] = kept(old, again["mask"])
            say(f"sequence 1 compacted from {held} to {budget} slots, {cache.free_pages} pages free")
        cache.reserve(1)
        pos = torch.full((2, 1), N + step, dtype=torch.int32, device=dev)
        out = []
        for l in range(L):
            qkv = normal(2, Hq + 2 * H, d)
            qk = tk.twinkv_qk_norm_rope(qkv[:, :Hq], qkv[:, Hq:Hq + H], wq, wk, table,
                                        pos.view(-1))
            cache.append(l, qk["k"].view(2, 1, H, d), qkv[:, Hq + H:].view(2, 1, H, d), pos)
            q = qk["q"].view(2, 1, Hq, d)
            a = cache.attend(l, q, want_lse=True)
            cache.weigh(l, q, a["lse"], sums[l])
            out.append(a["out"])
    say(f"decoded {steps} tokens of two sequences: lengths {cache.lens[0, :, 0].tolist()}")
    return {"out": torch.stack(out), "cache": cache, "sums": sums}


if __name__ == "__main__":
    demo()
    st = tk.twinkv_get_last_error()
    sys.exit(st)
