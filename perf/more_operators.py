"""The operators that make a retained set: attention over a prompt, the weight that it gives each
key, and the eviction by accumulated weight, for a prompt and while decoding.

  attend   causal attention over packed sequences with grouped heads (twinkv_prompt_attend)
  weights  what the tokens' attention weights sum to at each key (twinkv_prompt_weights)
  decode   the same for the newest tokens over pages of 4-bit codes, added to the sums so far
           (twinkv_cache_weights)
  policy   the positions that a budget keeps by accumulated weight (twinkv_weight_policy)

Token i of a sequence with n tokens and m keys is at position i + m - n and sees the keys up to its
own position; with a window, of those the ones less than `window` behind it and the first n_sink.
out_i = sum_j p_ij v_j, p_ij = exp(scale q_i . k_j - lse_i), lse_i = log sum_j exp(scale q_i . k_j).

A page holds 64 slots of one unit (one sequence and KV head).  Its keys are held in groups of 64
values: a 4-bit code per value, a bf16 scale s and a 4-bit zero z per group, s (code - z):

  K codes   [slot][4 t][G][2 w] words of 8 codes: value 64 G + 16 t + 8 w + 2 p + b in nibble 4 b + p
  K groups  [slot][G] words: the bits of s, and above them those of -(128 + z) in bf16
  values    as many bytes as the keys'
  positions [slot] int32

A case's fields: op; d; H KV and Hq query heads; for attend and weights B sequences of up to N
tokens after `prior` others of the same sequence, window, n_sink; ragged: lengths differ; padded:
every sequence has room for N; last: only so many last tokens of a sequence count (0: all); carry:
sums so far are given.  For decode B, N slots, n new tokens.  For policy L layers or sequences, N
positions, keep (the retained share).
"""
import math

import numpy as np
import torch

own = False

PAGE = 64                                # slots of a page
N_SINK, N_RECENT = 4, 64                 # the paper's protected positions (Sec. 3.2)
_MOST = 1 << 28                          # scores that the plain form holds at a time


def listed():
    return [
        # One short prompt in one Qwen3-4B layer, 32 query and 8 KV heads.  Latency counts.
        dict(op="attend", B=1, N=101, prior=0, Hq=32, H=8, d=128, window=0, n_sink=0,
             ragged=False, padded=False, name="attend_short"),
        # A 16k prompt of the same layer.
        dict(op="attend", B=1, N=16384, prior=0, Hq=32, H=8, d=128, window=0, n_sink=0,
             ragged=False, padded=False, name="attend_prompt"),
        # Twelve ragged Llama-3.2-1B prompts in one call, packed.
        dict(op="attend", B=12, N=3001, prior=0, Hq=32, H=8, d=64, window=0, n_sink=0,
             ragged=True, padded=False, name="attend_packed"),
        # A chunk of a long prompt, after 65k tokens that are already there.
        dict(op="attend", B=1, N=256, prior=65280, Hq=32, H=8, d=128, window=0, n_sink=0,
             ragged=False, padded=False, name="attend_chunk"),
        # The observation window at a 16k prompt's end: the last 32 tokens of one layer.
        dict(op="weights", B=1, N=16384, prior=0, Hq=32, H=8, d=128, window=0, n_sink=0, last=32,
             carry=False, ragged=False, padded=False, name="weights_recent"),
        # Every token of an 8k prompt counts.
        dict(op="weights", B=1, N=8192, prior=0, Hq=32, H=8, d=128, window=0, n_sink=0, last=0,
             carry=False, ragged=False, padded=False, name="weights_all"),
        # Ragged Llama-3.2-1B prompts in a padded batch, in a layer with a window and sinks.
        dict(op="weights", B=6, N=3001, prior=0, Hq=32, H=8, d=64, window=1024, n_sink=4, last=0,
             carry=False, ragged=True, padded=True, name="weights_window"),
        # One decoded token of one sequence over 2048 kept keys: latency.
        dict(op="decode", B=1, H=8, Hq=32, N=2048, n=1, d=128, window=0, n_sink=0, ragged=False,
             name="decode_one_layer"),
        # A serving batch of 32 sequences of 4k to 16k kept keys.
        dict(op="decode", B=32, H=8, Hq=32, N=16384, n=1, d=128, window=0, n_sink=0, ragged=True,
             name="decode_batch"),
        # What a serving loop decides layer by layer after a 4k prompt.
        dict(op="policy", L=1, H=8, N=4096, keep=0.5, carry=False, ragged=False,
             name="policy_one_layer"),
        # A whole Qwen3-4B cache at once.
        dict(op="policy", L=36, H=8, N=16384, keep=0.5, carry=False, ragged=False,
             name="policy_qwen"),
        # A second eviction while decoding: 64 sequences of different lengths, whose sums go on.
        dict(op="policy", L=64, H=8, N=4160, keep=0.7, carry=True, ragged=True,
             name="policy_decoding"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "weights", "weights", "decode", "policy"])
    d = rng.choice([64, 128])
    while True:
        H = rng.choice([1, 2, 4, 8])
        Hq = H * rng.choice([1, 2, 3, 4, 5, 7, 8])
        ragged = rng.random() < 0.5
        if op == "policy":
            L, N = rng.randint(1, 64), _spread(rng, 65, 65536)
            if L * H * N > 36 * 8 * 16384:
                continue
            return dict(op=op, L=L, H=H, N=N, keep=rng.choice([0.1, 0.3, 0.5, 0.7, 1.0]),
                        carry=rng.random() < 0.5, ragged=ragged)
        if op == "decode":
            B, N, n = _spread(rng, 1, 64), _spread(rng, 16, 131072), rng.choice([1, 1, 1, 2, 4, 7])
            if B * H * N * d > 32 * 8 * 16384 * 128 or B * Hq * n * N > 32 * 32 * 16384:
                continue
            window = rng.choice([0, 0, _spread(rng, 1, 2 * N)])
            return dict(op=op, B=B, H=H, Hq=Hq, N=N, n=n, d=d, window=window,
                        n_sink=rng.choice([0, 4, 130]) if window else 0, ragged=ragged)
        B, N = rng.choice([1, 1, 2, 5, 16]), _spread(rng, 1, 16384)
        prior = rng.choice([0, 0, _spread(rng, 1, 65536)])
        most = 32 * 16384 * 8192 * 128 if op == "attend" else 32 * 8192 * 4096 * 128
        if B * N * (N / 2 + prior) * Hq * d > most or B * (N + prior) * (2 * H + Hq) * d > 1 << 28:
            continue
        window = rng.choice([0, 0, _spread(rng, 1, 2 * N)])
        c = dict(op=op, B=B, N=N, prior=prior, Hq=Hq, H=H, d=d, window=window,
                 n_sink=rng.choice([0, 4, 130]) if window else 0, ragged=ragged,
                 padded=ragged and rng.random() < 0.5)
        if op == "weights":
            c.update(last=rng.choice([0, 16, 32, 64]), carry=rng.random() < 0.3)
        return c


def _lengths(case):
    """Lengths of the sequences or layers: N, or from N down to about N / 4 in even steps."""
    count = case["B"] if "B" in case else case["L"]
    down = 0.75 / count if case["ragged"] else 0.0
    return [max(case.get("n", 1), int(case["N"] * (1.0 - down * i))) for i in range(count)]


def _places(case):
    """Of each sequence: first token, tokens, first key, keys; then all tokens and keys."""
    N, prior = case["N"], case["prior"]
    places, t, j = [], 0, 0
    for n in _lengths(case):
        m = n + prior
        places.append((t, n, j, m))
        t += N if case["padded"] else n
        j += N + prior if case["padded"] else m
    return places, t, j


def _budgets(case):
    """Positions that each unit keeps."""
    return [min(x, max(1, math.ceil(case["keep"] * x))) for x in _lengths(case)
            for _ in range(case["H"])]


# ---------------------------------------------------------------- the plain form

def _unseen(case, first, count, keys, device):
    """[count, keys]: what the tokens at positions first, first + 1, ... do not see."""
    at = torch.arange(first, first + count, device=device)[:, None]
    j = torch.arange(keys, device=device)
    no = j > at
    if case["window"]:
        no |= (at - j >= case["window"]) & (j >= case["n_sink"])
    return no


def _blocks(case, s, last=0):
    """Parts of the sequences' tokens that the plain form takes at a time: (first token, count,
    position of the first, first key, keys)."""
    for t, n, j, m in _places(case)[0]:
        begin = max(0, n - last) if last else 0
        step = max(1, _MOST // (case["Hq"] * m))
        for i in range(begin, n, step):
            yield t + i, min(step, n - i), m - n + i, j, m


def _scores(case, s, block):
    """scale q . k of a block, [H, count, G, keys], -inf where a token does not see a key."""
    t, count, at, j, m = block
    H, d = case["H"], case["d"]
    q = s["q"][t:t + count].float().view(count, H, -1, d).permute(1, 0, 2, 3)
    k = s["k"][j:j + m].float().permute(1, 2, 0)
    x = torch.bmm(q.reshape(H, -1, d), k).mul_(d ** -0.5).view(H, count, -1, m)
    return x.masked_fill_(_unseen(case, at, count, m, x.device)[:, None], -math.inf)


def _plain_attend(s):
    c = s["case"]
    H, d = c["H"], c["d"]
    out = torch.zeros((s["q"].shape[0], c["Hq"], d), dtype=torch.bfloat16, device=s["q"].device)
    lse = torch.zeros(out.shape[:2], dtype=torch.float32, device=out.device)
    for block in _blocks(c, s):
        t, count, _, j, m = block
        x = _scores(c, s, block)
        top = x.amax(dim=-1, keepdim=True)
        x = x.sub_(top).exp_()
        total = x.sum(dim=-1, keepdim=True)
        v = s["v"][j:j + m].float().permute(1, 0, 2)
        o = torch.bmm(x.view(H, -1, m), v).view(H, count, -1, d) / total
        out[t:t + count] = o.permute(1, 0, 2, 3).reshape(count, -1, d).to(torch.bfloat16)
        lse[t:t + count] = (top + total.log()).squeeze(-1).permute(1, 0, 2).reshape(count, -1)
    return {"out": out, "lse": lse}


def _plain_weights(s):
    c = s["case"]
    H = c["H"]
    score = torch.zeros((H, s["k"].shape[0]), dtype=torch.float64, device=s["k"].device)
    if c["carry"]:
        for _, _, j, m in _places(c)[0]:
            score[:, j:j + m] = s["score"][:, j:j + m]
    for block in _blocks(c, s, c["last"]):
        t, count, _, j, m = block
        x = _scores(c, s, block)
        lse = s["lse"][t:t + count].view(count, H, -1).permute(1, 0, 2)
        x = x.sub_(lse[..., None]).exp_()
        score[:, j:j + m] += x.view(H, -1, m).sum(dim=1)
    return score.float()


def _nibbles(b):
    return torch.stack([b & 15, b >> 4], dim=-1).flatten(-2)


def _keys_of(pages, d):
    """Keys [p, 64, d] (float32) of pages, and the slots' positions."""
    p, G = pages.shape[0], d // 64
    codes = pages[:, :PAGE * d // 2].contiguous()
    code = _nibbles(codes).view(p, 64, 4, G, 2, 2, 4).permute(0, 1, 3, 2, 4, 6, 5)
    meta = pages[:, PAGE * d // 2:PAGE * d // 2 + PAGE * G * 4].contiguous()
    meta = meta.view(torch.bfloat16).view(p, 64, G, 2).float()
    k = (code.reshape(p, 64, G, 64).float() + (meta[..., 1] + 128.0)[..., None]) * meta[..., :1]
    return k.view(p, 64, d), pages[:, -4 * PAGE:].contiguous().view(torch.int32)


def _decode_scores(s):
    """scale q . k of the units [B H, G n, slots], -inf where a token does not see a slot."""
    c = s["case"]
    B, H, n, d, G = c["B"], c["H"], c["n"], c["d"], c["Hq"] // c["H"]
    k, pos = _keys_of(s["pool"][s["table"].reshape(-1).long()], d)
    k, pos = k.view(B * H, -1, d), pos.view(B * H, -1)
    q = s["q"].float().view(B, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(B * H, G * n, d)
    x = torch.bmm(q, k.transpose(1, 2)).mul_(d ** -0.5).view(B * H, G, n, -1)
    slot = torch.arange(k.shape[1], device=k.device)
    last = s["lens"].view(-1, 1).long() - n + torch.arange(n, device=k.device)
    seen = slot <= last[..., None]
    if c["window"]:
        at = pos.gather(1, last)[..., None]
        seen &= (at - pos[:, None, :] < c["window"]) | (pos[:, None, :] < c["n_sink"])
    return x.masked_fill_(~seen[:, None], -math.inf)


def _plain_decode(s):
    c = s["case"]
    B, H, n, G = c["B"], c["H"], c["n"], c["Hq"] // c["H"]
    x = _decode_scores(s)
    lse = s["lse"].view(B, n, H, G).permute(0, 2, 3, 1).reshape(B * H, G, n, 1)
    added = x.sub_(lse).exp_().flatten(1, 2).sum(dim=1, dtype=torch.float64)
    return (s["score"].view(B * H, -1) + added).float().view(B, H, -1)


def _plain_policy(s):
    c = s["case"]
    score = s["score"].flatten(0, 1)
    units, N = score.shape
    lens, budget = s["lens"].view(-1, 1), s["budget"].view(-1, 1)
    at = torch.arange(N, device=score.device)
    rank = torch.where((at < N_SINK) | (at >= lens - N_RECENT), 0, 1)
    rank = torch.where(at < lens, rank, 2)
    # by score, then by region, each sort leaving equal items in order
    order = torch.where(rank == 1, score, torch.zeros_like(score)).sort(
        dim=1, descending=True, stable=True).indices
    order = order.gather(1, rank.gather(1, order).sort(dim=1, stable=True).indices)
    taken = (at < budget) & (at < lens)
    mask = torch.zeros_like(score, dtype=torch.uint8).scatter_(1, order, taken.to(torch.uint8))
    got = {"mask": mask.view(s["score"].shape)}
    if c["carry"]:
        index = torch.argsort(1 - mask, dim=1, stable=True)
        kept = torch.where(taken, score.gather(1, index), torch.zeros_like(score))
        got["score"] = kept.view(s["score"].shape)
    return got


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _channels(g, d):
    """Spread of a head's channels: keys have a few large ones."""
    scale = torch.ones(d, device="cuda")
    scale[torch.randperm(d, generator=g, device="cuda")[:4]] = 4.0
    return scale


def _direction(g, d):
    """A direction in which queries agree and a sequence's first key stands out, as sinks do."""
    u = _normal(g, d)
    return u / u.square().sum().sqrt()


def _prompts(case, g):
    """Queries, keys and values: views of the fused projection, or of a cache that holds the tokens
    before the chunk too."""
    Hq, H, d = case["Hq"], case["H"], case["d"]
    places, tokens, keys = _places(case)
    u = _direction(g, d)
    s = {"case": case}
    if case["prior"]:
        s["q"] = (_normal(g, tokens, Hq, d) + 5.0 * u).to(torch.bfloat16)
        kv = _normal(g, keys, 2 * H, d)
        k, v = kv[:, :H], kv[:, H:]
    else:
        qkv = _normal(g, tokens, Hq + 2 * H, d)
        qkv[:, :Hq] += 5.0 * u
        k, v = qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        kv = qkv
    k *= _channels(g, d)
    for _, _, j, _ in places:
        k[j] += 9.0 * u
    kv = kv.to(torch.bfloat16)
    if case["prior"]:
        s["k"], s["v"] = kv[:, :H], kv[:, H:]
    else:
        s["q"], s["k"], s["v"] = kv[:, :Hq], kv[:, Hq:Hq + H], kv[:, Hq + H:]

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    s["offsets"] = ints([p[0] for p in places] + [tokens])
    s["k_offsets"] = ints([p[2] for p in places] + [keys]) if case["prior"] else None
    s["lens"] = ints([p[1] for p in places]) if case["padded"] else None
    s["k_lens"] = (ints([p[3] for p in places]) if case["padded"] and case["prior"] else None)
    return s


def _log_sums(case, s):
    """What the layer's attention left: the logarithms of its softmax's denominators."""
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    for block in _blocks(case, s):
        t, count = block[:2]
        x = _scores(case, s, block)
        top = x.amax(dim=-1, keepdim=True)
        x = top + x.sub_(top).exp_().sum(dim=-1, keepdim=True).log()
        lse[t:t + count] = x.squeeze(-1).permute(1, 0, 2).reshape(count, -1)
    return lse


def _fill(units, pages, d, lens, g, n_new):
    """Pages with keys in the slots of every unit, as after a prompt and its eviction: positions
    ascend with gaps, sinks and the newest ones without."""
    G, total = d // 64, units * pages
    table = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    gap = torch.randint(0, 2, (units, pages * PAGE), generator=g, device="cuda")
    gap[:, :N_SINK] = 0
    gap *= torch.arange(pages * PAGE, device="cuda") < (lens - n_new)[:, None]
    pos = ((gap + 1).cumsum(dim=1) - 1).to(torch.int32).view(total, PAGE)
    k = _normal(g, total, PAGE, d) * _channels(g, d)
    k.view(units, -1, d)[:, 0] += 9.0 * _direction(g, d)
    x = k.to(torch.bfloat16).float().view(total, PAGE, G, 64)
    lo, hi = x.amin(dim=-1).clamp(max=0.0), x.amax(dim=-1).clamp(min=0.0)
    scale = ((hi - lo) / 15.0).to(torch.bfloat16).float()
    zero = (-lo / scale).round().clamp(max=15.0)
    code = ((x / scale[..., None]).round() + zero[..., None]).clamp(0.0, 15.0).to(torch.uint8)
    code = code.view(total, PAGE, G, 4, 2, 4, 2).permute(0, 1, 3, 2, 4, 6, 5)
    code = code.reshape(total, PAGE, 4, G, 2, 4, 2)
    code = (code[..., 0] | (code[..., 1] << 4)).reshape(total, -1)
    meta = torch.stack([scale, -128.0 - zero], dim=-1).to(torch.bfloat16)
    meta = meta.view(torch.uint8).reshape(total, -1)
    values = torch.randint(0, 256, (total, code.shape[1] + meta.shape[1]), generator=g,
                           device="cuda", dtype=torch.uint8)
    pool = torch.empty((total, 2 * values.shape[1] + 4 * PAGE), dtype=torch.uint8, device="cuda")
    pool[table.long()] = torch.cat([code, meta, values, pos.view(torch.uint8).view(total, -1)],
                                   dim=1)
    return pool, table


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    if op in ("attend", "weights"):
        s = _prompts(case, g)
        if op == "weights":
            s["lse"] = _log_sums(case, s)
            if case["carry"]:
                s["score"] = -torch.rand((case["H"], s["k"].shape[0]), generator=g,
                                         device="cuda").clamp(min=1e-6).log()
        return s
    s = {"case": case}
    if op == "decode":
        B, H, Hq, N, n, d = (case[x] for x in ("B", "H", "Hq", "N", "n", "d"))
        pages = -(-N // PAGE)
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        lens = lens.repeat_interleave(H)
        s["pool"], table = _fill(B * H, pages, d, lens, g, n)
        s["table"], s["lens"] = table.view(B, H, pages), lens.view(B, H)
        s["q"] = (_normal(g, B, n, Hq, d) + 3.0 * _direction(g, d)).to(torch.bfloat16)
        x = _decode_scores(s)
        top = x.amax(dim=-1, keepdim=True)
        lse = (top + x.sub_(top).exp_().sum(dim=-1, keepdim=True).log()).squeeze(-1)
        s["lse"] = lse.view(B, H, Hq // H, n).permute(0, 3, 1, 2).reshape(B, n, Hq).contiguous()
        score = -torch.rand((B, H, pages * PAGE), generator=g, device="cuda").clamp(min=1e-6).log()
        held = torch.arange(pages * PAGE, device="cuda") < s["lens"][..., None]
        s["score"] = torch.where(held, score, torch.zeros_like(score))
        return s
    L, H, N = case["L"], case["H"], case["N"]
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda").repeat_interleave(H)
    s["lens"] = lens.view(L, H)
    s["budget"] = torch.tensor(_budgets(case), dtype=torch.int32, device="cuda").view(L, H)
    # weights are spread over many sizes; some are 0, and some alike
    score = (2.0 * _normal(g, L, H, N) - 2.0).exp()
    kind = torch.rand((L, H, N), generator=g, device="cuda")
    score = torch.where(kind < 0.05, torch.zeros_like(score), score)
    score = torch.where(kind > 0.9, (4.0 * score).round() / 4.0, score)
    held = torch.arange(N, device="cuda") < s["lens"][..., None]
    s["score"] = torch.where(held, score, torch.zeros_like(score))
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"attend": _plain_attend, "weights": _plain_weights, "decode": _plain_decode,
                "policy": _plain_policy}[op](s)
    from paper_2608_27128_gb300 import twinkv as tk
    # the output tensors and the workspace are kept from pass to pass; rows behind the sequences'
    # ends stay as they are
    first = "out" not in s
    out = s.setdefault("out", {})
    if op in ("attend", "weights"):
        tokens, Hq, d = s["q"].shape
        keys, H = s["k"].shape[:2]
        B = s["offsets"].shape[0] - 1
        where = dict(lens=s["lens"], k_offsets=s["k_offsets"], k_lens=s["k_lens"],
                     window=c["window"], n_sink=c["n_sink"])
        if op == "attend":
            if first:
                out["out"] = torch.zeros((tokens, Hq, d), dtype=torch.bfloat16, device="cuda")
                out["lse"] = torch.zeros((tokens, Hq), dtype=torch.float32, device="cuda")
                s["ws"] = tk.prompt_attend_workspace(s["q"].shape, s["k"].shape, B, "cuda")
            out.update(tk.twinkv_prompt_attend(s["q"], s["k"], s["v"], s["offsets"],
                                               want_lse=True, out=out, ws=s["ws"], **where))
            return {"out": out["out"], "lse": out["lse"]}
        if first:
            out["score"] = torch.zeros((H, keys), dtype=torch.float32, device="cuda")
            s["ws"] = tk.prompt_weights_workspace(s["q"].shape, s["k"].shape, B, "cuda")
        out.update(tk.twinkv_prompt_weights(s["q"], s["k"], s["lse"], s["offsets"],
                                            last=c["last"], score=s.get("score"), out=out,
                                            ws=s["ws"], **where))
        return out["score"]
    if op == "decode":
        if first:
            out["score"] = torch.zeros_like(s["score"])
        out.update(tk.twinkv_cache_weights(s["q"], s["lse"], s["pool"], s["table"], s["lens"],
                                           s["score"], window=c["window"], n_sink=c["n_sink"],
                                           out=out))
        return out["score"]
    out.update(tk.twinkv_weight_policy(s["score"], s["budget"], lens=s["lens"], n_sink=N_SINK,
                                       n_recent=N_RECENT, want_score=c["carry"], out=out))
    return {x: out[x] for x in (("mask", "score") if c["carry"] else ("mask",))}


# ---------------------------------------------------------------- work and exact values

def _pairs(case):
    """Keys that the tokens which count see, in all."""
    total = 0
    for _, n, _, m in _places(case)[0]:
        count = min(n, case.get("last") or n)
        sees = np.arange(m - count, m, dtype=np.int64) + 1
        if case["window"]:
            near = np.minimum(sees, case["window"])
            sees = near + np.minimum(sees - near, case["n_sink"])
        total += int(sees.sum())
    return total


def work(case):
    """Inputs once, outputs once; of pages what the operator looks at."""
    op = case["op"]
    if op == "policy":
        held, kept = sum(_lengths(case)) * case["H"], sum(_budgets(case))
        return {"bytes": held * 5 + (kept * 4 if case["carry"] else 0), "flops": held}
    H, Hq, d = case["H"], case["Hq"], case["d"]
    if op == "decode":
        held, n = [x * H for x in _lengths(case)], case["n"]
        looked = sum(held)
        if case["window"]:      # the positions' gaps are 1.5 on average
            looked = sum(min(x, H * (case["window"] / 1.5 + n + case["n_sink"])) for x in held)
        return {"bytes": looked * (d // 2 + 4 * (d // 64)) + sum(held) * 8
                + case["B"] * n * Hq * (2 * d + 4), "flops": looked * (Hq // H) * n * 2 * d}
    places, pairs = _places(case)[0], _pairs(case)
    tokens, keys = sum(p[1] for p in places), sum(p[3] for p in places)
    if op == "attend":
        return {"bytes": tokens * Hq * (4 * d + 4) + keys * H * 4 * d, "flops": pairs * Hq * 4 * d}
    tokens = sum(min(p[1], case["last"] or p[1]) for p in places)
    return {"bytes": tokens * Hq * (2 * d + 4) + keys * H * (2 * d + (8 if case["carry"] else 4)),
            "flops": pairs * Hq * 2 * d}


def _exact_prompt(case, s):
    """Head by head, some tokens at a time, over the keys up to the last of them."""
    H, Hq, d = case["H"], case["Hq"], case["d"]
    places, tokens, keys = _places(case)
    attend = case["op"] == "attend"
    if attend:
        out = torch.zeros((tokens, Hq, d), dtype=torch.float64, device="cuda")
        logs = torch.zeros((tokens, Hq), dtype=torch.float64, device="cuda")
    else:
        sums = torch.zeros((H, keys), dtype=torch.float64, device="cuda")
    for t, n, j, m in places:
        if not attend and case["carry"]:
            sums[:, j:j + m] = s["score"][:, j:j + m].double()
        begin = 0 if attend or not case["last"] else max(0, n - case["last"])
        step = max(16, (1 << 26) // m)
        for h in range(Hq):
            k = s["k"][j:j + m, h // (Hq // H)].double()
            v = s["v"][j:j + m, h // (Hq // H)].double() if attend else None
            for i in range(begin, n, step):
                e = min(n, i + step)
                top = m - n + e                          # keys up to the last token's own
                at = torch.arange(m - n + i, top, device="cuda").unsqueeze(1)
                j_ = torch.arange(top, device="cuda").unsqueeze(0)
                see = j_ <= at
                if case["window"]:
                    see = see & ((j_ > at - case["window"]) | (j_ < case["n_sink"]))
                x = (s["q"][t + i:t + e, h].double() @ k[:top].T) / math.sqrt(d)
                if attend:
                    x = x.masked_fill(~see, -math.inf)
                    logs[t + i:t + e, h] = torch.logsumexp(x, dim=1)
                    out[t + i:t + e, h] = torch.softmax(x, dim=1) @ v[:top]
                else:
                    w = torch.exp(x - s["lse"][t + i:t + e, h].double()[:, None])
                    sums[h // (Hq // H), j:j + top] += torch.where(see, w, 0.0).sum(dim=0)
    return {"out": out, "lse": logs} if attend else sums


def _exact_keys(raw, d):
    """Keys [p, 64, d] of pages in float64, each from the place of its own bits."""
    G = d // 64
    i = torch.arange(PAGE, device=raw.device)[:, None]
    e = torch.arange(d, device=raw.device)[None, :]
    word = ((i * 4 + e % 64 // 16) * G + e // 64) * 2 + e % 16 // 8
    nibble = 4 * (e % 2) + e % 8 // 2
    at = PAGE * d // 2 + 4 * (i * G + e // 64)

    def bf16(a):
        bits = raw[:, a].int() | (raw[:, a + 1].int() << 8)
        return (bits << 16).view(torch.float32).double()

    code = (raw[:, 4 * word + nibble // 2].int() >> (4 * (nibble % 2))) & 15
    return (code.double() + bf16(at + 2) + 128.0) * bf16(at)


def _exact_decode(case, s):
    B, H, n, G, d = case["B"], case["H"], case["n"], case["Hq"] // case["H"], case["d"]
    got = s["score"].double()
    for b in range(B):
        for h in range(H):
            raw, length = s["pool"][s["table"][b, h].long()], int(s["lens"][b, h])
            k = _exact_keys(raw, d).view(-1, d)[:length]
            pos = raw[:, -4 * PAGE:].contiguous().view(torch.int32).view(-1)[:length]
            for i in range(n):
                last = length - n + i
                see = torch.arange(length, device="cuda") <= last
                if case["window"]:
                    see &= (pos > pos[last] - case["window"]) | (pos < case["n_sink"])
                q = s["q"][b, i, h * G:(h + 1) * G].double()
                x = q @ k.T / math.sqrt(d) - s["lse"][b, i, h * G:(h + 1) * G].double()[:, None]
                got[b, h, :length] += torch.where(see, x.exp(), 0.0).sum(dim=0)
    return got


def _exact_policy(case, s):
    """Only the kept sums are numbers; the mask is whole."""
    score = s["score"].flatten(0, 1).double().cpu().numpy()
    kept = np.zeros_like(score)
    for u, (length, budget) in enumerate(zip(s["lens"].view(-1).tolist(),
                                             s["budget"].view(-1).tolist())):
        at = np.arange(length)
        free = (at >= N_SINK) & (at < length - N_RECENT)
        order = np.lexsort((at, np.where(free, -score[u, :length], 0.0), free))
        chosen = np.sort(order[:budget])
        kept[u, :len(chosen)] = score[u, chosen]
    return {"mask": None, "score": torch.from_numpy(kept).view(s["score"].shape).cuda()}


def exact(case, seed):
    if case["op"] in ("attend", "weights"):
        if _pairs(case) * case["Hq"] * case["d"] * 4.0 > 4e12:
            return None
        return _exact_prompt(case, prepare(case, seed))
    if case["op"] == "policy" and not case["carry"]:
        return None
    s = prepare(case, seed)
    return _exact_decode(case, s) if case["op"] == "decode" else _exact_policy(case, s)
