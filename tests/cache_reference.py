"""The operators around the pass in 64 bits, from their definitions: rounding to 4-bit groups,
pages, attention, norms with rotation.  Plain numpy, none of the package's code."""
import numpy as np

PAGE = 64
PAGE_BYTES = {64: 4864, 128: 9472}


def to_bf16(x):
    """Nearest bf16 (ties to even) of float64 values, as float64 (normal range)."""
    x = np.asarray(x, np.float64)
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), e - 8)


def quantize(rows):
    """Codes, scales, zeros of rows [..., d] (bf16 values)."""
    g = np.asarray(rows, np.float64).reshape(*rows.shape[:-1], -1, 64)
    lo = np.minimum(g.min(-1), 0.0)
    hi = np.maximum(g.max(-1), 0.0)
    s = to_bf16((hi - lo) / 15.0)
    s = np.where(s < 2.0 ** -126, 0.0, s)
    step = np.where(s > 0, s, 1.0)
    z = np.where(s > 0, np.minimum(15, np.rint(-lo / step)), 0)
    c = np.where(s[..., None] > 0,
                 np.minimum(15, np.rint(g / step[..., None]) + z[..., None]), 0)
    return c.reshape(rows.shape).astype(int), s, z.astype(int)


def values(c, s, z):
    g = c.reshape(*c.shape[:-1], -1, 64)
    return ((g - z[..., None]) * s[..., None]).reshape(c.shape)


def round_trip(rows):
    """What 4 bits leave of rows, in float64."""
    return values(*quantize(rows))


def bf16_bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def page_of(k, v, pos):
    """The bytes of a page with rows k, v [n <= 64, d]; the slots past them hold 0xFF."""
    n, d = k.shape
    G = d // 64
    raw = np.full(PAGE_BYTES[d], 0xFF, np.uint8)
    kc, ks, kz = quantize(k)
    vc, vs, vz = quantize(v)

    def nibble(at, which, c):
        at += which // 2
        shift = 4 * (which % 2)
        raw[at] = (raw[at] & (0xF0 >> shift)) | (c << shift)

    def half(at, x):
        bits = int(bf16_bits(x))
        raw[at], raw[at + 1] = bits & 255, bits >> 8

    vals = PAGE * d // 2 + 4 * PAGE * G
    scales = vals + PAGE * d // 2
    zeros = scales + 2 * PAGE * G
    for i in range(n):
        for e in range(d):
            word = ((i * 4 + e % 64 // 16) * G + e // 64) * 2 + e % 16 // 8
            nibble(4 * word, 4 * (e % 2) + e % 8 // 2, kc[i, e])
            word = (((e // 16 * 8 + e % 8) * 4 + i % 8 // 2) * 2 + e % 16 // 8) * 2 + i // 32
            nibble(vals + 4 * word, 4 * (i % 2) + 2 * (i % 32 // 16) + i % 16 // 8, vc[i, e])
        for x in range(G):
            half(PAGE * d // 2 + 4 * (i * G + x), ks[i, x])
            half(PAGE * d // 2 + 4 * (i * G + x) + 2, -(128 + kz[i, x]))
            half(scales + 2 * (i * G + x), vs[i, x])
            place = ((x * 4 + i % 8 // 2) * 4 + i // 16) * 4 + i % 16 // 8 * 2 + i % 2
            half(zeros + 2 * place, -(128 + vz[i, x]))
        raw[zeros + 2 * PAGE * G + 4 * i:][:4] = np.array([pos[i]], np.int32).view(np.uint8)
    return raw


def attend(q, k, v, pos, scale, window=0, n_sink=0, v_scales=None):
    """Attention of the newest tokens q [n, G, d] of one unit over its rows k, v [len, d] at
    positions pos: outputs [n, G, d], log denominators [n, G], and the sizes by which an output may
    be off: sum_j p_j |v_j| and sum_j p_j s_j (v_scales [len, groups]), both [n, G, d]."""
    n, G, d = q.shape
    length = k.shape[0]
    s = np.zeros((length, d // 64)) if v_scales is None else v_scales
    s = np.repeat(s, 64, axis=1)
    out, size, steps = (np.zeros((n, G, d)) for _ in range(3))
    lse = np.full((n, G), -np.inf)
    for i in range(n):
        last = length - n + i
        if last < 0:
            continue
        see = np.arange(length) <= last
        if window > 0:
            see &= (pos > pos[last] - window) | (pos < n_sink)
        x = (q[i].astype(np.float64) @ k[see].T) * scale
        m = x.max(-1, keepdims=True)
        p = np.exp(x - m)
        total = p.sum(-1, keepdims=True)
        p /= total
        out[i], size[i], steps[i] = p @ v[see], p @ np.abs(v[see]), p @ s[see]
        lse[i] = (m + np.log(total))[:, 0]
    return out, lse, size, steps


def attend_bound(out, size, steps, length):
    """How far the kernel's outputs may be from attend's (`length` slots).

    bf16 has 8 significant bits, so a rounding is off by 2^-8 at most.
      2^-8 size      each probability times its value scale is rounded, to 8 bits or more
      2^-8 |out|     so is the output
      2^-10 size     scores: the float32 sums run over terms of size 136 |q| s, 2^-23 each at worst;
                     for |q| about 1.2, 128 dimensions, key scales up to 1.6 and d^-0.5 that is
                     below 5e-4, and twice that in a ratio of sums
      the last       the sums over codes and over zeros (as such, or plus 128), whose difference is the output,
                     are float32 sums of up to 143 p s in len / 16 steps each, 2^-23 a step
    """
    return (2.0 ** -8 * (size + np.abs(out)) + 2.0 ** -10 * size
            + (length / 8 + 8) * 2.0 ** -23 * 143 * steps + 1e-30)


def norm_rope(x, w, cos_sin, positions, eps):
    """x [T, heads, d] -> rotated, and the size of the terms of each sum."""
    x = np.asarray(x, np.float64)
    d = x.shape[-1]
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    row = np.asarray(cos_sin, np.float64)[positions]
    cos, sin = row[:, None, :d // 2], row[:, None, d // 2:]
    a, b = x[..., :d // 2], x[..., d // 2:]
    out = np.concatenate([a * cos - b * sin, a * sin + b * cos], -1)
    size = np.concatenate([abs(a * cos) + abs(b * sin), abs(a * sin) + abs(b * cos)], -1)
    return out, size
