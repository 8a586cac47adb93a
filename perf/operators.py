"""The operators around the repair pass: what makes the keys it audits and what keeps, moves and
reads the keys and values it retains, in pages of 4-bit codes.

  rope      norms of queries and keys per head with the position rotation (twinkv_qk_norm_rope)
  pack      the retained rows of a dense cache into pages, and the rows read back, as the next
            audit gets them (twinkv_cache_pack, twinkv_cache_read)
  append    the rows of new tokens into pages, and those rows read back (twinkv_cache_append)
  compact   the kept slots of one set of pages into another, and the rows read back
            (twinkv_cache_compact)
  attend    attention of the newest tokens over the pages (twinkv_cache_attend)

A row of 64 or 128 values is held in groups of 64: a 4-bit code per value, a bf16 scale s and a
4-bit zero z per group, standing for s (code - z).  A page holds 64 slots of one unit (one
sequence or layer, and one KV head):

  K codes   [slot][4 t][G][2 w] words of 8 codes: value 64 G + 16 t + 8 w + 2 p + b in nibble 4 b + p
  K groups  [slot][G] words: the bits of s, and above them those of -(128 + z) in bf16
  V codes   [d / 16][8 g][4 t][2 h][2 a] words of 8 codes: value 16 m + 8 h + g of slot
            32 a + 16 c + 8 k + 2 t + b in nibble 4 b + 2 c + k
  V scales  [slot][G] bf16
  V zeros   [G][4 t][4 tile][2 k][2 b] bf16, -(128 + z) of slot 16 tile + 8 k + 2 t + b
  positions [slot] int32

A case's fields: op; d; dtype of the dense inputs; for rope T tokens, Hq and H heads, norm; for
the others L layers or B sequences, H KV heads, N slots or positions, keep (the retained share);
for append and attend n new tokens; for attend Hq, window and n_sink; ragged: lengths differ.
"""
import math

import torch

own = False

PAGE = 64                                # slots of a page
N_SINK, N_RECENT = 4, 64                 # the paper's protected positions (Sec. 3.2)
EPS = 1e-6


def page_bytes(d):
    groups = d // 64
    return PAGE * d + PAGE * groups * 8 + PAGE * 4


def slot_bytes(d):
    """Codes, scales and zeros of one slot, keys and values."""
    return d + 8 * (d // 64)


def listed():
    return [
        # One decoded token of a Qwen3-4B layer: 32 query and 8 KV heads.  Latency counts.
        dict(op="rope", T=1, Hq=32, H=8, d=128, dtype="bf16", norm=True, name="rope_token"),
        # A 16k prompt of the same layer, out of the fused projection.
        dict(op="rope", T=16384, Hq=32, H=8, d=128, dtype="bf16", norm=True, name="rope_prompt"),
        # A ragged Llama-3.2-1B prompt in float32; that model has no norms, only the rotation.
        dict(op="rope", T=3001, Hq=32, H=8, d=64, dtype="f32", norm=False,
             name="rope_llama_f32"),
        # What a serving loop does layer by layer after a 4k prompt and its repair.
        dict(op="pack", L=1, H=8, N=4096, d=128, dtype="bf16", keep=0.5, ragged=False,
             name="pack_one_layer"),
        # A whole Qwen3-4B cache, budgets shrinking with depth.
        dict(op="pack", L=36, H=8, N=8192, d=128, dtype="bf16", keep=0.5, ragged=True,
             name="pack_qwen_pyramid"),
        # One decoded token of 64 sequences into one layer's pages.
        dict(op="append", B=64, H=8, N=4096, n=1, d=128, dtype="bf16", name="append_token"),
        # A second eviction, in the middle of decoding: half of what a Qwen3-4B cache holds.
        dict(op="compact", L=36, H=8, N=8192, d=128, keep=0.5, ragged=False,
             name="compact_qwen_half"),
        # The same on a ragged Llama-3.2-1B cache, 30 % kept.
        dict(op="compact", L=16, H=8, N=3001, d=64, keep=0.3, ragged=True,
             name="compact_llama_ragged"),
        # One sequence's token in one layer over 2048 kept keys: latency.
        dict(op="attend", B=1, H=8, Hq=32, N=2048, n=1, d=128, window=0, n_sink=0, ragged=False,
             name="attend_one_layer"),
        # A token at the end of a 128k context.
        dict(op="attend", B=1, H=8, Hq=32, N=131009, n=1, d=128, window=0, n_sink=0,
             ragged=False, name="attend_long"),
        # A serving batch of 32 sequences of 4k to 16k kept keys.
        dict(op="attend", B=32, H=8, Hq=32, N=16384, n=1, d=128, window=0, n_sink=0, ragged=True,
             name="attend_batch"),
        # Four speculative tokens in a layer with a sliding window and visible sinks, d = 64.
        dict(op="attend", B=16, H=8, Hq=32, N=8192, n=4, d=64, window=4096, n_sink=4,
             ragged=False, name="attend_window_spec"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "pack", "append", "compact", "attend", "attend"])
    d = rng.choice([64, 128])
    while True:
        H = rng.choice([1, 2, 4, 8])
        if op == "rope":
            Hq = H * rng.choice([1, 2, 3, 4, 5, 8])
            T = _spread(rng, 1, 16384)
            if T * (Hq + H) * d > 16384 * 40 * 128:
                continue
            return dict(op=op, T=T, Hq=Hq, H=H, d=d, dtype=rng.choice(["bf16", "bf16", "f32"]),
                        norm=rng.random() < 0.6)
        if op in ("pack", "compact"):
            L, N = rng.randint(1, 36), _spread(rng, 65, 65536)
            if L * H * N * d > 36 * 8 * 8192 * 128:
                continue
            c = dict(op=op, L=L, H=H, N=N, d=d, keep=rng.choice([0.1, 0.3, 0.5, 0.7, 1.0]),
                     ragged=rng.random() < 0.5)
            if op == "pack":
                c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
                if c["dtype"] == "f32" and L * H * N * d > 18 * 8 * 8192 * 128:
                    continue
            return c
        if op == "append":
            return dict(op=op, B=_spread(rng, 1, 64), H=H, N=_spread(rng, 16, 4096),
                        n=rng.choice([1, 1, 2, 3, 5, 8, 16]), d=d,
                        dtype=rng.choice(["bf16", "bf16", "f32"]))
        B, N, n = _spread(rng, 1, 64), _spread(rng, 16, 131072), rng.choice([1, 1, 1, 2, 4, 7])
        Hq = H * rng.choice([1, 2, 3, 4, 5, 7, 8])
        if B * H * N * d > 32 * 8 * 16384 * 128 or B * Hq * n * N > 32 * 32 * 16384:
            continue
        window = rng.choice([0, 0, _spread(rng, 1, 2 * N)])
        return dict(op=op, B=B, H=H, Hq=Hq, N=N, n=n, d=d, window=window,
                    n_sink=rng.choice([0, 4, 130]) if window else 0, ragged=rng.random() < 0.5)


# ---------------------------------------------------------------- the plain form

def _quantize(x):
    """Codes [..., d], scales and zeros [..., G] (float32) of rows of bf16 values [..., d]."""
    g = x.view(*x.shape[:-1], -1, 64)
    lo = g.amin(dim=-1, keepdim=True).clamp(max=0.0)
    hi = g.amax(dim=-1, keepdim=True).clamp(min=0.0)
    s = ((hi - lo) / 15.0).to(torch.bfloat16).float()
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    r = torch.where(s > 0, s, torch.ones_like(s))
    z = torch.where(s > 0, (-lo / r).round().clamp(max=15.0), torch.zeros_like(s))
    c = torch.where(s > 0, ((g / r).round() + z).clamp(0.0, 15.0), torch.zeros_like(g))
    return c.view(x.shape), s.squeeze(-1), z.squeeze(-1)


def _pairs(nibbles):
    """uint8 [..., 8] of codes -> [..., 4] bytes, the even one low."""
    b = nibbles.view(*nibbles.shape[:-1], 4, 2)
    return b[..., 0] | (b[..., 1] << 4)


def _bits(x):
    """The bytes of a tensor's values, over its last dimension."""
    return x.contiguous().view(torch.uint8)


def _assemble(kc, ks, kz, vc, vs, vz, pos):
    """Pages [p, bytes] of codes [p, 64, d], scales and zeros [p, 64, G], positions [p, 64]."""
    p, _, d = kc.shape
    G = d // 64
    kc = kc.to(torch.uint8).view(p, 64, G, 4, 2, 4, 2).permute(0, 1, 3, 2, 4, 6, 5)
    kc = _pairs(kc.reshape(p, 64, 4, G, 2, 8)).reshape(p, -1)
    km = torch.stack([ks, -128.0 - kz], dim=-1).to(torch.bfloat16)
    #                               a  c  k  t  b  m        h  g
    vc = vc.to(torch.uint8).view(p, 2, 2, 2, 4, 2, d // 16, 2, 8)
    vc = vc.permute(0, 6, 8, 4, 7, 1, 5, 2, 3)
    vc = _pairs(vc.reshape(p, d // 16, 8, 4, 2, 2, 8)).reshape(p, -1)
    vz = (-128.0 - vz).to(torch.bfloat16).view(p, 4, 2, 4, 2, G).permute(0, 5, 3, 1, 2, 4)
    return torch.cat([kc, _bits(km).reshape(p, -1), vc,
                      _bits(vs.to(torch.bfloat16)).reshape(p, -1), _bits(vz).reshape(p, -1),
                      _bits(pos.to(torch.int32)).reshape(p, -1)], dim=1)


def _nibbles(b):
    return torch.stack([b & 15, b >> 4], dim=-1).flatten(-2)


def _take_apart(pages, d):
    """What _assemble put together: kc, ks, kz, vc, vs, vz (codes uint8, the rest float32), pos."""
    p, G = pages.shape[0], d // 64
    sizes = [PAGE * d // 2, PAGE * G * 4, PAGE * d // 2, PAGE * G * 2, PAGE * G * 2, PAGE * 4]
    kc, km, vc, vs, vz, pos = [x.contiguous() for x in pages.split(sizes, dim=1)]
    kc = _nibbles(kc).view(p, 64, 4, G, 2, 2, 4).permute(0, 1, 3, 2, 4, 6, 5).reshape(p, 64, d)
    km = km.view(torch.bfloat16).view(p, 64, G, 2).float()
    #                           m        g  t  h  a  b  c  k
    vc = _nibbles(vc).view(p, d // 16, 8, 4, 2, 2, 2, 2, 2).permute(0, 5, 7, 8, 3, 6, 1, 4, 2)
    vz = vz.view(torch.bfloat16).view(p, G, 4, 4, 2, 2).permute(0, 3, 4, 2, 5, 1)
    return (kc, km[..., 0], -128.0 - km[..., 1], vc.reshape(p, 64, d),
            vs.view(torch.bfloat16).view(p, 64, G).float(),
            -128.0 - vz.reshape(p, 64, G).float(), pos.view(torch.int32))


def _values(c, s, z):
    """s (code - z) of codes [p, 64, d], scales and zeros [p, 64, G], in float32."""
    p, _, d = c.shape
    return ((c.view(p, 64, -1, 64).float() - z[..., None]) * s[..., None]).view(p, 64, d)


def _encode(k, v, pos):
    """Pages [p, bytes] of rows k, v [p, 64, d] (float32 of bf16 values), positions [p, 64]."""
    return _assemble(*_quantize(k), *_quantize(v), pos)


def _decode(pages, d):
    """The values k, v [p, 64, d] that pages stand for (float32), and the positions [p, 64]."""
    kc, ks, kz, vc, vs, vz, pos = _take_apart(pages, d)
    return _values(kc, ks, kz), _values(vc, vs, vz), pos


def _rows(pool, table, lens, d, rows, first=None):
    """`rows` rows of every unit's pages (from slot `first` on) in bf16, and their positions."""
    units = table.shape[0]
    slot = torch.arange(rows, device=pool.device)[None, :]
    if first is None:
        pages = table[:, :-(-rows // PAGE)]
        k, v, pos = _decode(pool[pages.reshape(-1).long()], d)
        k, v = (x.view(units, -1, d)[:, :rows] for x in (k, v))
        pos = pos.view(units, -1)[:, :rows]
    else:
        slot = first[:, None] + slot
        at = table.gather(1, slot // PAGE)
        k, v, pos = _decode(pool[at.reshape(-1).long()], d)
        inside = (slot % PAGE).reshape(-1, 1)
        k, v = (x.gather(1, inside[..., None].expand(-1, -1, d)).view(units, rows, d)
                for x in (k, v))
        pos = pos.gather(1, inside).view(units, rows)
    held = (slot < lens[:, None])
    zero = torch.zeros((), device=pool.device)
    k, v = (torch.where(held[..., None], x, zero).to(torch.bfloat16) for x in (k, v))
    return k, v, torch.where(held, pos, torch.full_like(pos, -1))


def _plain_rope(s):
    c, d = s["case"], s["case"]["d"]
    cos, sin = s["cos_sin"][s["positions"].long()][:, None, :].split(d // 2, dim=-1)

    def one(x, w):
        x = x.float()
        if w is not None:
            x = x / (x.square().mean(dim=-1, keepdim=True) + EPS).sqrt() * w.float()
        a, b = x.split(d // 2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)

    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    return {"q": one(s["q"], s["wq"]).to(dtype), "k": one(s["k"], s["wk"]).to(dtype)}


def _plain_pack(s):
    c, d = s["case"], s["case"]["d"]
    units, N, rows = c["L"] * c["H"], c["N"], s["rows"]
    mask = s["mask"].view(units, N)
    lens = mask.sum(dim=1, dtype=torch.int32)
    index = torch.argsort(1 - mask, dim=1, stable=True)[:, :rows]
    padded = s["table"].shape[-1] * PAGE
    index = torch.nn.functional.pad(index, (0, padded - rows))
    k, v = (s[n].view(units, N, d).gather(1, index[..., None].expand(-1, -1, d)).to(
        torch.bfloat16).float().view(-1, PAGE, d) for n in ("keys", "values"))
    table = s["table"].view(units, -1)
    s["pool"][table.reshape(-1).long()] = _encode(k, v, index.view(-1, PAGE))
    k, v, pos = _rows(s["pool"], table, lens, d, rows)
    return {"keys": k, "values": v, "positions": pos, "lens": lens}


def _plain_append(s):
    c, d = s["case"], s["case"]["d"]
    B, H, n = c["B"], c["H"], c["n"]
    units = B * H
    table, lens = s["table"].view(units, -1), s["lens"].view(-1)
    first = lens[:, None].long()
    # the pages that the new rows reach, taken apart, given the rows, and put back
    reach = (n + PAGE - 2) // PAGE + 1
    pages = table.gather(1, first // PAGE + torch.arange(reach, device=first.device)).long()
    slot = first % PAGE + torch.arange(n, device=first.device)
    rows = [s[x].permute(0, 2, 1, 3).reshape(units, n, d).to(torch.bfloat16).float()
            for x in ("k", "v")]
    new = [*_quantize(rows[0]), *_quantize(rows[1]),
           s["positions"][:, None, :].expand(B, H, n).reshape(units, n)]
    old = _take_apart(s["pool"][pages.view(-1)], d)
    put = []
    for x, y in zip(old, new):
        x = x.reshape(units, reach * PAGE, *x.shape[2:])
        at = slot.view(units, n, *[1] * (x.dim() - 2)).expand(units, n, *x.shape[2:])
        put.append(x.scatter(1, at, y.to(x.dtype)).view(-1, PAGE, *x.shape[2:]))
    s["pool"][pages.view(-1)] = _assemble(*put)
    k, v, pos = _rows(s["pool"], table, lens + n, d, n, first=lens.long())
    return {"keys": k, "values": v, "positions": pos, "lens": lens + n}


def _plain_compact(s):
    d, rows = s["case"]["d"], s["rows"]
    table, lens = s["table"], s["lens"]
    units = table.shape[0]
    inside = torch.arange(s["keep"].shape[1], device=lens.device) < lens[:, None]
    keep = s["keep"] * inside
    new = keep.sum(dim=1, dtype=torch.int32)
    index = torch.argsort(1 - keep, dim=1, stable=True)[:, :rows]
    padded = s["new_table"].shape[1] * PAGE
    index = torch.nn.functional.pad(index, (0, padded - rows))
    parts = []
    for x in _take_apart(s["pool"][table.reshape(-1).long()], d):
        x = x.reshape(units, -1, *x.shape[2:])
        at = index.view(units, padded, *[1] * (x.dim() - 2)).expand(units, padded, *x.shape[2:])
        parts.append(x.gather(1, at).view(-1, PAGE, *x.shape[2:]))
    s["pool"][s["new_table"].reshape(-1).long()] = _assemble(*parts)
    k, v, pos = _rows(s["pool"], s["new_table"], new, d, rows)
    return {"keys": k, "values": v, "positions": pos, "lens": new}


def _plain_attend(s):
    c = s["case"]
    B, H, n, d, G = c["B"], c["H"], c["n"], c["d"], c["Hq"] // c["H"]
    table = s["table"].view(B * H, -1)
    k, v, pos = _decode(s["pool"][table.reshape(-1).long()], d)
    k, v, pos = k.view(B * H, -1, d), v.view(B * H, -1, d), pos.view(B * H, -1)
    q = s["q"].float().view(B, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(B * H, G * n, d)
    score = torch.bmm(q, k.transpose(1, 2)).mul_(d ** -0.5).view(B * H, G, n, -1)
    slot = torch.arange(k.shape[1], device=k.device)
    last = s["lens"].view(-1, 1).long() - n + torch.arange(n, device=k.device)
    seen = slot <= last[..., None]
    if c["window"]:
        at = pos.gather(1, last)[..., None]
        seen &= (at - pos[:, None, :] < c["window"]) | (pos[:, None, :] < c["n_sink"])
    score.masked_fill_(~seen[:, None], -math.inf)
    score -= score.amax(dim=-1, keepdim=True).clamp(min=-3.0e38)
    score.exp_()
    total = score.sum(dim=-1, keepdim=True)
    # slots past a unit's length hold no row: what their bytes say is not looked at
    v = torch.where((slot < s["lens"].view(-1, 1))[..., None], v, torch.zeros_like(v[:1, :1]))
    o = torch.bmm(score.view(B * H, G * n, -1), v).view(B * H, G, n, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.view(B, H, G, n, d).permute(0, 3, 1, 2, 4).reshape(B, n, H * G, d).to(
        torch.bfloat16)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _channels(g, d):
    """Spread of a head's channels: keys have a few large ones."""
    scale = torch.ones(d, device="cuda")
    scale[torch.randperm(d, generator=g, device="cuda")[:4]] = 4.0
    return scale


def _cos_sin(rows, d):
    theta = 1.0e6 ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * theta
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def _budgets(case):
    """Retained rows of each unit: the share, or a schedule that shrinks with depth."""
    L, H, N = case["L"], case["H"], case["N"]
    mean = max(1, math.ceil(case["keep"] * N))
    spread = min(0.5, (N - mean) / mean) if case["ragged"] else 0.0
    return [min(N, max(1, int(mean * (1.0 + spread * (1.0 - 2.0 * l / max(1, L - 1))))))
            for l in range(L) for _ in range(H)]


def _mask(units, N, budgets, g, lens=None):
    """Retained sets of exactly the budgets' sizes; sinks and recent positions first."""
    score = torch.rand((units, N), generator=g, device="cuda")
    at = torch.arange(N, device="cuda")
    lens = torch.full((units,), N, device="cuda") if lens is None else lens
    score[:, :N_SINK] = 2.0
    score.masked_fill_(at >= lens[:, None] - N_RECENT, 2.0)
    score.masked_fill_(at >= lens[:, None], -1.0)
    order = torch.argsort(score, dim=1, descending=True)
    kept = at < torch.tensor(budgets, device="cuda")[:, None]
    return torch.zeros((units, N), dtype=torch.uint8, device="cuda").scatter_(
        1, order, kept.to(torch.uint8))


def _table(units, pages, g, more=0):
    """Pages of the pool in no order, and the pool's size."""
    total = units * pages + more
    return torch.randperm(total, generator=g, device="cuda").to(torch.int32), total


def _lengths(case):
    """Lengths of the units (a sequence's or a layer's heads share one): N, or from N down to
    about N / 4 in even steps."""
    H, N = case["H"], case["N"]
    count = case["B"] if "B" in case else case["L"]
    down = 0.75 / count if case["ragged"] else 0.0
    return [max(case.get("n", 1), int(N * (1.0 - down * i))) for i in range(count)
            for _ in range(H)]


def _kept(case):
    """Slots that a compaction leaves in each unit."""
    return [max(1, math.ceil(case["keep"] * n)) for n in _lengths(case)]


def _fill(units, pages, d, lens, g, n_new=1):
    """A pool with rows in the slots of every unit, as after a prompt and its eviction: the
    positions ascend with gaps, sinks and the newest ones without."""
    table, total = _table(units, pages, g)
    slots = pages * PAGE
    gap = torch.randint(0, 2, (units, slots), generator=g, device="cuda")
    gap[:, :N_SINK] = 0
    gap *= torch.arange(slots, device="cuda") < (lens - n_new)[:, None]
    pos = (gap + 1).cumsum(dim=1) - 1
    pool = torch.empty((total, page_bytes(d)), dtype=torch.uint8, device="cuda")
    scale = _channels(g, d)
    k = (_normal(g, units * pages, PAGE, d) * scale).to(torch.bfloat16).float()
    v = _normal(g, units * pages, PAGE, d).to(torch.bfloat16).float()
    pool[table.long()] = _encode(k, v, pos.view(-1, PAGE))
    return pool, table.view(units, pages)


def prepare(case, seed):
    g = _generator(seed)
    op, d, dev = case["op"], case["d"], torch.device("cuda", torch.cuda.current_device())
    s = {"case": case}
    if op == "rope":
        T, Hq, H = case["T"], case["Hq"], case["H"]
        rows = max(T, 4096)
        # the fused projection's output, of which queries and keys are views
        qkv = _normal(g, T, Hq + 2 * H, d).to(_dtype(case))
        s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + H]
        s["wq"] = s["wk"] = None
        if case["norm"]:
            s["wq"], s["wk"] = ((1.0 + 0.2 * _normal(g, d)).to(_dtype(case)) for _ in range(2))
        s["cos_sin"] = _cos_sin(rows, d)
        first = int(torch.randint(0, rows - T + 1, (1,), generator=g, device="cuda"))
        s["positions"] = torch.arange(first, first + T, dtype=torch.int32, device=dev)
    elif op == "pack":
        L, H, N = case["L"], case["H"], case["N"]
        budgets = _budgets(case)
        s["rows"] = max(budgets)
        pages = -(-s["rows"] // PAGE)
        s["keys"] = (_normal(g, L, H, N, d) * _channels(g, d)).to(_dtype(case))
        s["values"] = _normal(g, L, H, N, d).to(_dtype(case))
        s["mask"] = _mask(L * H, N, budgets, g).view(L, H, N)
        table, total = _table(L * H, pages, g)
        s["table"] = table.view(L, H, pages)
        s["pool"] = torch.zeros((total, page_bytes(d)), dtype=torch.uint8, device=dev)
    elif op == "append":
        B, H, N, n = case["B"], case["H"], case["N"], case["n"]
        pages = -(-N // PAGE) + 2
        # every sequence is at another place of its page
        per = torch.randint(max(1, N // 2), N + 1, (B,), generator=g, device="cuda")
        lens = per.int().repeat_interleave(H)
        s["pool"], table = _fill(B * H, pages, d, lens, g)
        s["table"], s["lens"] = table.view(B, H, pages), lens.view(B, H)
        qkv = _normal(g, B, n, 6 * H, d).to(_dtype(case))      # four query heads per KV head
        s["k"], s["v"] = qkv[:, :, 4 * H:5 * H], qkv[:, :, 5 * H:]
        s["positions"] = (2 * per[:, None] + torch.arange(n, device=dev)).int()
    elif op == "compact":
        L, H, N = case["L"], case["H"], case["N"]
        units, pages = L * H, -(-N // PAGE)
        s["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device=dev)
        s["pool"], s["table"] = _fill(units, pages, d, s["lens"], g)
        s["keep"] = _mask(units, N, _kept(case), g, s["lens"])
        s["rows"] = max(_kept(case))
        more = -(-s["rows"] // PAGE)
        first = s["pool"].shape[0]
        s["new_table"] = (first + torch.randperm(units * more, generator=g, device="cuda").to(
            torch.int32)).view(units, more)
        s["pool"] = torch.cat([s["pool"], torch.zeros((units * more, page_bytes(d)),
                                                      dtype=torch.uint8, device=dev)])
    else:
        B, H, Hq, N, n = case["B"], case["H"], case["Hq"], case["N"], case["n"]
        pages = -(-N // PAGE)
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device=dev)
        s["pool"], table = _fill(B * H, pages, d, lens, g, n)
        s["table"], s["lens"] = table.view(B, H, pages), lens.view(B, H)
        s["q"] = _normal(g, B, n, Hq, d).to(torch.bfloat16)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"rope": _plain_rope, "pack": _plain_pack, "append": _plain_append,
                "compact": _plain_compact, "attend": _plain_attend}[op](s)
    from paper_2608_27128_gb300 import twinkv as tk
    d = s["case"]["d"]
    # the output tensors and the workspace are kept from pass to pass
    out, ws = s.setdefault("out", {}), s.get("ws")
    if op == "rope":
        out.update(tk.twinkv_qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["cos_sin"],
                                          s["positions"], eps=EPS, out=out))
        return {"q": out["q"], "k": out["k"]}
    if op == "attend":
        c = s["case"]
        if ws is None:
            ws = s["ws"] = tk.cache_attend_workspace(s["q"].shape, c["H"], s["q"].device)
        out.update(tk.twinkv_cache_attend(s["q"], s["pool"], s["table"], s["lens"],
                                          scale=d ** -0.5, window=c["window"],
                                          n_sink=c["n_sink"], out=out, ws=ws))
        return out["out"]
    back = s.setdefault("back", {})
    if op == "append":
        n = s["case"]["n"]
        out.update(tk.twinkv_cache_append(s["k"], s["v"], s["positions"], s["pool"], s["table"],
                                          s["lens"], out=out))
        back.update(tk.twinkv_cache_read(s["pool"], s["table"], out["lens"], n, last=True,
                                         out=back))
    elif op == "pack":
        units, N = s["case"]["L"] * s["case"]["H"], s["case"]["N"]
        if ws is None:
            ws = s["ws"] = tk.cache_move_workspace(units, N, s["pool"].device)
        out.update(tk.twinkv_cache_pack(s["keys"], s["values"], s["mask"], s["pool"],
                                        s["table"], out=out, ws=ws))
        back.update(tk.twinkv_cache_read(s["pool"], s["table"], out["lens"], s["rows"],
                                         out=back))
    else:
        units, N = s["keep"].shape
        if ws is None:
            ws = s["ws"] = tk.cache_move_workspace(units, N, s["pool"].device)
        out.update(tk.twinkv_cache_compact(s["pool"], s["table"], s["lens"], s["keep"],
                                           s["new_table"], out=out, ws=ws))
        back.update(tk.twinkv_cache_read(s["pool"], s["new_table"], out["lens"], s["rows"],
                                         out=back))
    rows = back["keys"].shape[-2]
    return {"keys": back["keys"].view(-1, rows, d), "values": back["values"].view(-1, rows, d),
            "positions": back["positions"].view(-1, rows), "lens": out["lens"].view(-1)}


# ---------------------------------------------------------------- work and exact values

def work(case):
    """Inputs once, outputs once.  Of a cache's pages the slots that hold rows count, with their
    positions where those are asked for; what is read back counts as written, not as read."""
    op, d = case["op"], case["d"]
    size = 4 if case.get("dtype") == "f32" else 2
    if op == "rope":
        n = case["T"] * (case["Hq"] + case["H"]) * d
        return {"bytes": 2 * n * size + case["T"] * (4 * d + 4), "flops": 8 * n}
    slot, back = slot_bytes(d), 4 * d + 4
    if op == "pack":
        units, kept = case["L"] * case["H"], sum(_budgets(case))
        return {"bytes": units * case["N"] + kept * (2 * d * size + slot + 4 + back),
                "flops": kept * 2 * d * 8}
    if op == "append":
        rows = case["B"] * case["H"] * case["n"]
        return {"bytes": rows * (2 * d * size + slot + 4 + back) + case["B"] * case["H"] * 8,
                "flops": rows * 2 * d * 8}
    if op == "compact":
        held, kept = sum(_lengths(case)), sum(_kept(case))
        return {"bytes": held + kept * (2 * (slot + 4) + back), "flops": kept * 2 * d * 2}
    n, held = case["n"], _lengths(case)
    if case["window"]:      # the positions' gaps are 1.5 on average
        held = [min(x, case["window"] / 1.5 + n + case["n_sink"]) for x in held]
    rows = case["Hq"] // case["H"] * n
    return {"bytes": sum(held) * slot + case["B"] * case["Hq"] * n * d * 4,
            "flops": sum(held) * rows * 4 * d}


def _slot_values(raw, d, keys):
    """Values [p, 64, d] of pages in float64, each from the place of its own bits."""
    G, dev = d // 64, raw.device
    i = torch.arange(PAGE, device=dev)[:, None]
    e = torch.arange(d, device=dev)[None, :]
    group = e // 64
    if keys:
        word = ((i * 4 + e % 64 // 16) * G + group) * 2 + e % 16 // 8
        nibble = 4 * (e % 2) + e % 8 // 2
        base, s_at = 0, PAGE * d // 2 + 4 * (i * G + group)
        z_at = s_at + 2
    else:
        word = (((e // 16 * 8 + e % 8) * 4 + i % 8 // 2) * 2 + e % 16 // 8) * 2 + i // 32
        nibble = 4 * (i % 2) + 2 * (i % 32 // 16) + i % 16 // 8
        base = PAGE * d // 2 + 4 * PAGE * G
        s_at = base + PAGE * d // 2 + 2 * (i * G + group)
        z_at = (base + PAGE * d // 2 + 2 * PAGE * G
                + 2 * (((group * 4 + i % 8 // 2) * 4 + i // 16) * 4 + i % 16 // 8 * 2 + i % 2))
    code = (raw[:, base + 4 * word + nibble // 2].int() >> (4 * (nibble % 2))) & 15

    def bf16(at):
        bits = raw[:, at].int() | (raw[:, at + 1].int() << 8)
        return (bits << 16).view(torch.float32).double()

    return (code.double() + bf16(z_at) + 128.0) * bf16(s_at)


def _exact_rows(x):
    """s (c - z) of rows [..., d] of bf16 values, in float64."""
    g = x.double().view(*x.shape[:-1], -1, 64)
    lo = g.amin(dim=-1, keepdim=True).clamp(max=0.0)
    hi = g.amax(dim=-1, keepdim=True).clamp(min=0.0)
    s = ((hi - lo) / 15.0).to(torch.bfloat16).double()
    step = torch.where(s > 0, s, torch.ones_like(s))
    z = (-lo / step).round().clamp(max=15.0)
    c = ((g / step).round() + z).clamp(0.0, 15.0)
    return (s * (c - z)).view(x.shape)


def exact(case, seed):
    op, d = case["op"], case["d"]
    s = prepare(case, seed)
    if op == "rope":
        at = s["cos_sin"].double()[s["positions"].long()]
        turn = torch.complex(at[:, :d // 2], at[:, d // 2:])[:, None, :]
        got = {}
        for name, w in (("q", s["wq"]), ("k", s["wk"])):
            x = s[name].double()
            if w is not None:
                x = x * torch.rsqrt((x * x).sum(dim=-1, keepdim=True) / d + EPS) * w.double()
            y = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
            got[name] = torch.cat([y.real, y.imag], dim=-1)
        return got
    if op == "append":
        B, H, n = case["B"], case["H"], case["n"]
        k, v = (_exact_rows(s[x].permute(0, 2, 1, 3).reshape(B * H, n, d).to(torch.bfloat16))
                for x in ("k", "v"))
        return {"keys": k, "values": v, "positions": None, "lens": None}
    if op in ("pack", "compact"):
        units, rows = case["L"] * case["H"], s["rows"]
        if units * rows * d * 8 > 6e9:
            return None
        got = {"positions": None, "lens": None}
        for name in ("keys", "values"):
            out = torch.zeros((units, rows, d), dtype=torch.float64, device="cuda")
            for u in range(units):
                if op == "pack":
                    kept = s["mask"].view(units, -1)[u].nonzero()[:, 0]
                    x = _exact_rows(s[name].view(units, -1, d)[u, kept].to(torch.bfloat16))
                else:
                    kept = s["keep"][u, :int(s["lens"][u])].nonzero()[:, 0]
                    x = _slot_values(s["pool"][s["table"][u].long()], d, name == "keys")
                    x = x.view(-1, d)[kept]
                out[u, :x.shape[0]] = x
            got[name] = out
        return got
    B, H, n, G = case["B"], case["H"], case["n"], case["Hq"] // case["H"]
    if float(B) * case["Hq"] * n * case["N"] * d > 4e9:
        return None
    out = torch.zeros((B, n, H * G, d), dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(H):
            raw, length = s["pool"][s["table"][b, h].long()], int(s["lens"][b, h])
            k = _slot_values(raw, d, True).view(-1, d)[:length]
            v = _slot_values(raw, d, False).view(-1, d)[:length]
            pos = raw[:, -4 * PAGE:].contiguous().view(torch.int32).view(-1)[:length]
            for i in range(n):
                last = length - n + i
                if last < 0:
                    continue
                see = torch.arange(length, device="cuda") <= last
                if case["window"]:
                    see &= (pos > pos[last] - case["window"]) | (pos < case["n_sink"])
                q = s["q"][b, i, h * G:(h + 1) * G].double()
                p = torch.softmax((q @ k[see].T) / math.sqrt(d), dim=-1)
                out[b, i, h * G:(h + 1) * G] = p @ v[see]
    return out
