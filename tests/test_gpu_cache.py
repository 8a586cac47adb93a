"""The 4-bit pages on the GPU against their definition in 64 bits.

What the pages hold is a whole number per value and rounded scales: rows read back have to be equal to
the definition's, rounded to bf16, bit for bit.

Attention is compared within cache_reference.attend_bound, which derives what the kernel's roundings
come to.  Denominators: scores are off by 5e-4 at most there, and so is the sum's logarithm."""
import numpy as np
import pytest
import torch

import cache_reference as R
from gpu_harness import device
from paper_2608_27128_gb300 import twinkv as tk

pytestmark = pytest.mark.gpu


def rng_rows(rng, *shape, outliers=True):
    x = rng.standard_normal(shape)
    if outliers:
        x[..., rng.choice(shape[-1], 3, replace=False)] *= 6.0
    return torch.from_numpy(x).to(torch.bfloat16)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def table_for(rng, units, pages, total=None):
    total = units * pages + 3 if total is None else total
    ids = rng.permutation(total)[:units * pages].astype(np.int32).reshape(units, pages)
    return ids, total


def dirty_pool(n, d):
    """Memory as another program leaves it: every scale and zero a NaN."""
    return torch.full((n, R.PAGE_BYTES[d]), 0xFF, dtype=torch.uint8, device=device())


def put(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device())


def make_cache(rng, lens, d, pages=None, n_new=1):
    """Random rows of the given lengths in pages: pool, table, lens, and per unit k, v, pos."""
    pages = pages or max(1, -(-max(lens) // 64))
    ids, total = table_for(rng, len(lens), pages)
    raw = np.full((total, R.PAGE_BYTES[d]), 0xFF, np.uint8)
    units = []
    for u, n in enumerate(lens):
        k, v = f64(rng_rows(rng, n, d)), f64(rng_rows(rng, n, d, outliers=False))
        gap = rng.integers(1, 3, n)
        gap[max(0, n - n_new):] = 1
        pos = np.cumsum(gap) - 1 if n else np.zeros(0, np.int64)
        for p in range(-(-n // 64)):
            at = slice(64 * p, min(n, 64 * p + 64))
            raw[ids[u, p]] = R.page_of(k[at], v[at], pos[at])
        units.append((R.round_trip(k) if n else k, R.round_trip(v) if n else v, pos,
                      R.quantize(v)[1] if n else np.zeros((0, d // 64))))
    return put(raw), put(ids), units


# ---------------------------------------------------------------- writing and reading

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L,H,N,keep", [(1, 1, 1, 1.0), (1, 2, 63, 0.5), (2, 3, 65, 0.9),
                                        (1, 2, 1000, 0.3), (2, 2, 4097, 0.5), (1, 1, 9001, 0.02),
                                        (1, 3, 640, 0.0)])
def test_pack_and_read(d, dtype, L, H, N, keep):
    rng = np.random.default_rng([d, L, H, N])
    U = L * H
    k = torch.from_numpy(rng.standard_normal((U, N, d)) * 3).to(dtype)
    v = torch.from_numpy(rng.standard_normal((U, N, d))).to(dtype)
    k[:, N // 2] = 0                                      # a row without range
    v[:, N // 3] = v[:, N // 3].abs()                     # one without negative values
    mask = (rng.random((U, N)) < keep).astype(np.uint8)
    if keep == 1.0:
        mask[:] = 1
    lens = mask.sum(1)
    pages = max(1, -(-int(lens.max()) // 64)) + 1
    ids, total = table_for(rng, U, pages)
    pool = dirty_pool(total, d)
    shape = (L, H, N, d)
    out = tk.twinkv_cache_pack(k.view(shape).to(device()), v.view(shape).to(device()),
                               put(mask.reshape(L, H, N)), pool, put(ids.reshape(L, H, pages)))
    assert out["status"].eq(0).all()
    np.testing.assert_array_equal(out["lens"].cpu().numpy().reshape(-1), lens)
    rows = max(1, int(lens.max())) + 5
    got = tk.twinkv_cache_read(pool, put(ids.reshape(L, H, pages)), out["lens"], rows)
    assert got["status"].eq(0).all()
    kk, vv = (f64(x.to(torch.bfloat16)) for x in (k, v))
    for u in range(U):
        at = np.flatnonzero(mask[u])
        n = len(at)
        for name, x in (("keys", kk), ("values", vv)):
            r = got[name].view(U, rows, d)[u]
            want = R.to_bf16(R.round_trip(x[u, at])) if n else np.zeros((0, d))
            np.testing.assert_array_equal(f64(r[:n]), want, err_msg=f"{name} {u}")
            assert not r[n:].any()
        pos = got["positions"].view(U, rows)[u].cpu().numpy()
        np.testing.assert_array_equal(pos[:n], at)
        assert (pos[n:] == -1).all()


@pytest.mark.parametrize("d", [64, 128])
def test_page_bytes_are_the_layout(d):
    rng = np.random.default_rng(d)
    k, v = rng_rows(rng, 1, 1, 64, d), rng_rows(rng, 1, 1, 64, d)
    pool = dirty_pool(1, d)
    tk.twinkv_cache_pack(k.to(device()), v.to(device()), None, pool, put(np.zeros((1, 1, 1), np.int32)))
    want = R.page_of(f64(k)[0, 0], f64(v)[0, 0], np.arange(64))
    np.testing.assert_array_equal(pool[0].cpu().numpy(), want)


def test_ties_and_extremes_round_as_defined():
    """Groups whose values fall on halves of the scale, powers of two apart, tiny and large."""
    rng = np.random.default_rng(9)
    rows = []
    for e in (-100, -20, 0, 30, 100):
        base = rng.integers(-15, 16, (40, 64)) * 0.5
        base[:, 0], base[:, 1] = -7.0, 8.0               # scale 1 (times 2^e)
        rows.append(np.ldexp(base, e))
    for big in (2.0 ** 13, 2.0 ** 17):                    # the ends 2^13 and 2^17 apart
        base = rng.standard_normal((40, 64))
        base[:, 5] = big
        rows.append(base)
    rows.append(np.ldexp(rng.standard_normal((10, 64)), -129))
    x = torch.from_numpy(np.concatenate(rows)).to(torch.bfloat16)
    n = x.shape[0]
    pages = -(-n // 64)
    pool = dirty_pool(pages, 64)
    tab = put(np.arange(pages, dtype=np.int32).reshape(1, 1, pages))
    t = x.view(1, 1, n, 64).to(device())
    lens = tk.twinkv_cache_pack(t, t, None, pool, tab)["lens"]
    got = tk.twinkv_cache_read(pool, tab, lens, n)
    want = R.to_bf16(R.round_trip(f64(x)))
    np.testing.assert_array_equal(f64(got["keys"])[0, 0], want)
    np.testing.assert_array_equal(f64(got["values"])[0, 0], want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,H,n,lens", [(1, 1, 1, [0]), (2, 2, 1, [63, 64]), (3, 1, 5, [61, 0, 130]),
                                        (1, 3, 64, [37]), (2, 1, 16, [48, 63])])
def test_append(d, dtype, B, H, n, lens):
    rng = np.random.default_rng([d, B, H, n])
    old = np.repeat(lens, H)
    pages = -(-(max(lens) + n) // 64)
    pool, ids, units = make_cache(rng, old.tolist(), d, pages=pages)
    qkv = torch.from_numpy(rng.standard_normal((B, n, 6 * H, d))).to(dtype).to(device())
    k, v = qkv[:, :, 4 * H:5 * H], qkv[:, :, 5 * H:]      # views into a fused projection
    pos = np.array([[10000 + 7 * b + i for i in range(n)] for b in range(B)], np.int32)
    table, have = ids.view(B, H, pages), put(old.reshape(B, H).astype(np.int32))
    out = tk.twinkv_cache_append(k, v, put(pos), pool, table, have, out={"lens": have})
    assert out["lens"].data_ptr() == have.data_ptr() and out["status"].eq(0).all()
    np.testing.assert_array_equal(have.cpu().numpy().reshape(-1), old + n)
    rows = max(lens) + n
    got = tk.twinkv_cache_read(pool, table, have, rows)
    tail = tk.twinkv_cache_read(pool, table, have, n, last=True)
    for u in range(B * H):
        b, h = divmod(u, H)
        for name, x, i in (("keys", k, 0), ("values", v, 1)):
            new = R.round_trip(f64(x[b, :, h].to(torch.bfloat16)))
            want = R.to_bf16(np.concatenate([units[u][i], new]))
            np.testing.assert_array_equal(f64(got[name][b, h, :len(want)]), want)
            np.testing.assert_array_equal(f64(tail[name][b, h]), R.to_bf16(new))
        want = np.concatenate([units[u][2], pos[b]])
        np.testing.assert_array_equal(got["positions"][b, h, :len(want)].cpu().numpy(), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,keep", [([1], 1.0), ([64, 65], 0.5), ([700, 3, 0, 129], 0.3),
                                       ([2000], 0.03), ([500, 640], None)])
def test_compact(d, lens, keep):
    rng = np.random.default_rng([d, len(lens)])
    pool, ids, units = make_cache(rng, lens, d)
    U, pages = ids.shape
    N = max(lens) + 3
    mask = (rng.random((U, N)) < (keep or 0)).astype(np.uint8)
    if keep == 1.0:
        mask[:] = 1
    kept = [np.arange(n) if keep is None else np.flatnonzero(mask[u, :n])
            for u, n in enumerate(lens)]
    for u, n in enumerate(lens):
        mask[u, n:] = 7                                   # past the length: not looked at
    new_pages = max(1, -(-max(len(x) for x in kept) // 64))
    first = pool.shape[0]
    pool = torch.cat([pool, dirty_pool(U * new_pages, d)])
    new = put((first + rng.permutation(U * new_pages)).astype(np.int32).reshape(U, new_pages))
    before = pool[:first].clone()
    have = put(np.array(lens, np.int32))
    out = tk.twinkv_cache_compact(pool, ids, have, None if keep is None else put(mask), new)
    assert out["status"].eq(0).all() and torch.equal(pool[:first], before)
    np.testing.assert_array_equal(out["lens"].cpu().numpy(), [len(x) for x in kept])
    rows = max(1, max(len(x) for x in kept))
    got = tk.twinkv_cache_read(pool, new, out["lens"], rows)
    for u, at in enumerate(kept):
        for name, i in (("keys", 0), ("values", 1)):
            np.testing.assert_array_equal(f64(got[name][u, :len(at)]), R.to_bf16(units[u][i][at]))
        np.testing.assert_array_equal(got["positions"][u, :len(at)].cpu().numpy(),
                                      units[u][2][at])


def test_mask_rows_at_any_address():
    """Rows of masks start at every offset from a 16-byte boundary."""
    rng = np.random.default_rng(3)
    U, N, d = 33, 4111, 64
    mask = (rng.random((U, N)) < 0.4).astype(np.uint8)
    store = torch.zeros(U * N + 16, dtype=torch.uint8, device=device())
    ids, total = table_for(rng, U, 65)
    x = torch.zeros(1, U, N, d, dtype=torch.bfloat16, device=device())
    pool = dirty_pool(total, d)
    for off in (0, 1, 7, 15):
        m = store[off:off + U * N].view(1, U, N)
        m.copy_(put(mask.reshape(1, U, N)))
        out = tk.twinkv_cache_pack(x, x, m, pool, put(ids.reshape(1, U, 65)))
        got = tk.twinkv_cache_read(pool, put(ids.reshape(1, U, 65)), out["lens"], 1)
        np.testing.assert_array_equal(out["lens"].cpu().numpy()[0], mask.sum(1))
        np.testing.assert_array_equal(got["positions"].cpu().numpy()[0, :, 0], mask.argmax(1))


# ---------------------------------------------------------------- attention

def check_attend(rng, lens, H, G, n, d, window=0, n_sink=0, scale=None, strided=False):
    """lens per sequence; every KV head of a sequence has a length of its own (lens + h)."""
    B = len(lens)
    per = [max(0, x - 3 * h) if x > 3 * H else x for x in lens for h in range(H)]
    pool, ids, units = make_cache(rng, per, d, n_new=n)
    pages = ids.shape[1]
    q = torch.from_numpy(rng.standard_normal((B, n, H * G, d)) * 1.5).to(torch.bfloat16)
    t = q.to(device())
    if strided:
        wide = torch.zeros(B, n, H * G + 3, d, dtype=torch.bfloat16, device=device())
        wide[:, :, 2:-1] = t
        t = wide[:, :, 2:-1]
    out = tk.twinkv_cache_attend(t, pool, ids.view(B, H, pages),
                                 put(np.array(per, np.int32).reshape(B, H)), scale=scale,
                                 window=window, n_sink=n_sink, want_lse=True)
    torch.cuda.synchronize()
    assert out["status"].eq(0).all()
    got, lse = f64(out["out"]), f64(out["lse"])
    scale = d ** -0.5 if scale is None else scale
    for u in range(B * H):
        b, h = divmod(u, H)
        k, v, pos, vs = units[u]
        qq = f64(q)[b, :, h * G:(h + 1) * G]
        want, wl, *sizes = R.attend(qq, k, v, pos, scale, window, n_sink, vs)
        err = np.abs(got[b, :, h * G:(h + 1) * G] - want)
        bound = R.attend_bound(want, *sizes, len(k))
        assert (err <= bound).all(), (u, (err / bound).max())
        gl = lse[b, :, h * G:(h + 1) * G]
        assert np.array_equal(np.isneginf(gl), np.isneginf(wl))
        fine = np.isfinite(wl)
        assert (np.abs(gl[fine] - wl[fine]) <= 5e-4 * max(1.0, scale * d ** 0.5)).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (8, 1), (3, 2), (4, 4), (7, 5), (16, 1), (40, 1)])
def test_attend_rows(d, G, n):
    check_attend(np.random.default_rng([d, G, n]), [200, 65 + n], 2, G, n, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[0], [1], [2], [63], [64], [65], [0, 1, 128, 0, 300],
                                  [1000, 7], [5000], [64] * 33])
def test_attend_lengths(d, lens):
    check_attend(np.random.default_rng([d, len(lens)]), lens, 2, 4, 1, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[0, 1, 2, 3], [3, 4, 66], [130, 1]])
def test_attend_rows_that_see_nothing(d, lens):
    """Units shorter than the number of new tokens: their first tokens have no slot."""
    check_attend(np.random.default_rng([d, 7]), lens, 1, 2, 4, d)
    check_attend(np.random.default_rng([d, 8]), lens, 1, 5, 4, d, window=2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 4), (50, 0), (64, 1), (300, 130), (700, 64),
                                           (100000, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("n", [1, 3])
def test_attend_window(d, window, n_sink, n):
    check_attend(np.random.default_rng([d, n]), [1100, 90, 5], 2, 4, n, d, window, n_sink)


def test_attend_scale_and_strides():
    check_attend(np.random.default_rng(1), [500], 2, 4, 1, 128, scale=0.7)
    check_attend(np.random.default_rng(2), [500], 2, 4, 1, 64, scale=1e-6)
    check_attend(np.random.default_rng(3), [300, 20], 2, 4, 3, 128, strided=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sizes", [[0, 0, 1], [1, 2.0 ** 12, 2.0 ** 24], [2.0 ** 24, 2.0 ** 12, 1],
                                   [2.0 ** -100, 1, 2.0 ** 100], [2.0 ** -118, 2.0 ** -118, 0],
                                   [2.0 ** 100, 0, 2.0 ** 100]])
def test_attend_value_scales_that_change_from_page_to_page(d, sizes):
    """Values of three pages many powers of two apart, per group another order: the probabilities'
    units follow the largest.  What is small beside the largest of its group counts as little."""
    rng = np.random.default_rng(d)
    n = 64 * len(sizes)
    k, v = f64(rng_rows(rng, n, d)), f64(rng_rows(rng, n, d, outliers=False))
    factor = np.repeat(np.array(sizes, np.float64), 64)[:, None]
    v[:, :64] *= factor
    v[:, 64:] *= factor[::-1]
    pos = np.arange(n)
    raw = np.stack([R.page_of(k[i:i + 64], v[i:i + 64], pos[i:i + 64]) for i in range(0, n, 64)])
    q = rng_rows(rng, 1, 1, 4, d)
    table = put(np.arange(len(sizes), dtype=np.int32).reshape(1, 1, -1))
    out = f64(tk.twinkv_cache_attend(q.to(device()), put(raw), table,
                                     put(np.array([[n]], np.int32)))["out"])
    want, _, *sz = R.attend(f64(q)[0], R.round_trip(k), R.round_trip(v), pos, d ** -0.5,
                            v_scales=R.quantize(v)[1])
    bound = R.attend_bound(want, *sz, n)
    assert (np.abs(out[0] - want) <= bound).all(), (np.abs(out[0] - want) / bound).max()


def test_attend_many_units_of_few_slots():
    """Spans that hold many units, some of them empty; and more units than a chunk of the grid's
    first step."""
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 90, 700)
    lens[100:180] = 0
    check_attend(rng, lens.tolist(), 1, 2, 1, 64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n,units,most", [(4, 1, 500, 900), (8, 1, 500, 900), (4, 3, 400, 600),
                                            (8, 3, 250, 600), (4, 4, 3, 90000)])
def test_attend_units_that_warps_and_blocks_share(d, G, n, units, most):
    """More pages than warps in the grid, and units that begin and end anywhere in a warp's span and
    a block's; with more than 16 rows several parts of each; a few units over all blocks.  The units'
    pages are drawn from 24."""
    rng = np.random.default_rng([d, G, n])
    pool, ids, cache = make_cache(rng, [24 * 64], d)
    k, v, pos, vs = cache[0]
    lens = rng.integers(0, most, units)
    lens[units // 2:units // 2 + units // 20] = 0
    table = rng.integers(0, 24, (units, -(-most // 64)))
    q = rng_rows(rng, units, n, G, d, outliers=False)
    out = tk.twinkv_cache_attend(q.to(device()), pool, ids[0][put(table)].view(units, 1, -1),
                                 put(lens.astype(np.int32).reshape(units, 1)), want_lse=True)
    got, lse = f64(out["out"]), f64(out["lse"])
    for u in range(units):
        slots = (table[u][:, None] * 64 + np.arange(64)).reshape(-1)[:lens[u]]
        want, wl, *sizes = R.attend(f64(q)[u], k[slots], v[slots], np.arange(lens[u]), d ** -0.5,
                                    v_scales=vs[slots])
        bound = R.attend_bound(want, *sizes, len(slots))
        assert (np.abs(got[u] - want) <= bound).all(), u
        assert np.array_equal(np.isneginf(lse[u]), np.isneginf(wl))
        fine = np.isfinite(wl)
        assert (np.abs(lse[u][fine] - wl[fine]) <= 5e-4).all()


def test_attend_is_the_same_twice():
    rng = np.random.default_rng(6)
    pool, ids, _ = make_cache(rng, [3000, 700], 128)
    q = rng_rows(rng, 2, 1, 4, 128).to(device())
    lens = put(np.array([[3000], [700]], np.int32))
    a = tk.twinkv_cache_attend(q, pool, ids.view(2, 1, -1), lens)["out"]
    for _ in range(3):
        b = tk.twinkv_cache_attend(q, pool, ids.view(2, 1, -1), lens)["out"]
        assert torch.equal(a, b)


def test_pages_past_four_gigabytes():
    """Page numbers whose bytes lie beyond 2^32."""
    d = 128
    n_pages = 2 ** 32 // R.PAGE_BYTES[d] + 2000
    pool = torch.zeros((n_pages, R.PAGE_BYTES[d]), dtype=torch.uint8, device=device())
    rng = np.random.default_rng(8)
    N = 300
    k, v = rng_rows(rng, 1, 2, N, d), rng_rows(rng, 1, 2, N, d)
    ids = (n_pages - 1 - np.arange(10, dtype=np.int32)).reshape(1, 2, 5)
    ids[0, 1] = np.arange(5)
    out = tk.twinkv_cache_pack(k.to(device()), v.to(device()), None, pool, put(ids))
    new = (n_pages - 1000 + np.arange(10, dtype=np.int32)).reshape(1, 2, 5)
    moved = tk.twinkv_cache_compact(pool, put(ids), out["lens"], None, put(new))
    got = tk.twinkv_cache_read(pool, put(new), moved["lens"], N)
    np.testing.assert_array_equal(f64(got["keys"])[0], R.to_bf16(R.round_trip(f64(k)[0])))
    np.testing.assert_array_equal(f64(got["values"])[0], R.to_bf16(R.round_trip(f64(v)[0])))
    q = rng_rows(rng, 1, 1, 8, d)
    o = f64(tk.twinkv_cache_attend(q.to(device()), pool, put(new), moved["lens"])["out"])
    for h in range(2):
        vv = f64(v)[0, h]
        want, _, *sizes = R.attend(f64(q)[0, :, 4 * h:4 * h + 4], R.round_trip(f64(k)[0, h]),
                                   R.round_trip(vv), np.arange(N), d ** -0.5,
                                   v_scales=R.quantize(vv)[1])
        assert (np.abs(o[0, :, 4 * h:4 * h + 4] - want)
                <= R.attend_bound(want, *sizes, N)).all()


# ---------------------------------------------------------------- data errors

def test_pack_data_errors():
    d, N = 64, 200
    x = torch.randn(1, 5, N, d, device=device()).to(torch.bfloat16)
    mask = torch.ones(1, 5, N, dtype=torch.uint8, device=device())
    mask[0, 0, 17] = 2                                    # not a mask byte
    mask[0, 4, 100:] = 0
    ids = np.arange(20, dtype=np.int32).reshape(1, 5, 4)
    ids[0, 1, 3] = 20                                     # outside the pool, and needed
    ids[0, 2, 0] = -1
    ids[0, 4, 2] = 99                                     # outside, not needed
    pool = dirty_pool(20, d)
    out = tk.twinkv_cache_pack(x, x, mask, pool, put(ids))
    assert out["status"].tolist() == [[1, 1, 1, 0, 0]]
    assert out["lens"].tolist() == [[0, 0, 0, N, 100]]
    out = tk.twinkv_cache_pack(x, x, mask, pool, put(ids[:, :, :3]))
    assert out["status"].tolist() == [[1, 7, 7, 7, 0]]
    assert out["lens"].tolist() == [[0, 0, 0, 0, 100]]


def test_append_data_errors_write_nothing():
    d = 64
    pool = dirty_pool(4, d)
    before = pool.clone()
    k = torch.randn(1, 2, 4, d, device=device()).to(torch.bfloat16)
    pos = torch.zeros(1, 2, dtype=torch.int32, device=device())
    ids = put(np.array([[[0], [1], [9], [2]]], np.int32))
    lens = put(np.array([[63, -1, 5, 128]], np.int32))
    out = tk.twinkv_cache_append(k, k, pos, pool, ids, lens)
    assert out["status"].tolist() == [[7, 1, 1, 7]]
    assert torch.equal(out["lens"], lens) and torch.equal(pool, before)


def test_read_compact_attend_data_errors():
    d = 64
    rng = np.random.default_rng(4)
    pool, ids, units = make_cache(rng, [100, 100, 100, 100], d)
    ids[1, 1] = 1000
    lens = put(np.array([100, 100, -3, 129], np.int32))
    got = tk.twinkv_cache_read(pool, ids, lens, 100)
    assert got["status"].tolist() == [0, 1, 1, 1]
    assert not got["keys"][1, 64:].any() and not got["keys"][2:].any()
    np.testing.assert_array_equal(f64(got["keys"][1, :64]), R.to_bf16(units[1][0][:64]))
    new = put(np.arange(8, dtype=np.int32).reshape(4, 2) + pool.shape[0])
    pool = torch.cat([pool, dirty_pool(8, d)])
    assert int(ids[1, 1]) >= pool.shape[0]
    keep = torch.ones(4, 128, dtype=torch.uint8, device=device())
    out = tk.twinkv_cache_compact(pool, ids, lens, keep, new)
    assert out["status"].tolist() == [0, 1, 1, 1] and out["lens"].tolist() == [100, 0, 0, 0]
    q = rng_rows(rng, 4, 1, 2, d)
    res = tk.twinkv_cache_attend(q.to(device()), pool, ids.view(4, 1, 2), lens.view(4, 1),
                                 want_lse=True)
    assert res["status"].view(-1).tolist() == [0, 1, 1, 1]
    assert not res["out"][2:].any() and torch.isneginf(res["lse"][2:]).all()
    # the page outside the pool counts as unseen
    k, v, pos, vs = (x[:64] for x in units[1])
    want, _, *sizes = R.attend(f64(q)[1], k, v, pos, d ** -0.5, v_scales=vs)
    assert (np.abs(f64(res["out"])[1] - want) <= R.attend_bound(want, *sizes, 64)).all()


# ---------------------------------------------------------------- streams and graphs

def test_calls_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(12)
    B, H, G, d, n = 2, 2, 4, 128, 1
    pool, ids, _ = make_cache(rng, [150] * 4, d, pages=4)
    table = ids.view(B, H, 4)
    lens = put(np.full((B, H), 150, np.int32))
    qkv = rng_rows(rng, B, n, H * (G + 2), d).to(device())
    q, k, v = qkv[:, :, :H * G], qkv[:, :, H * G:H * G + H], qkv[:, :, H * G + H:]
    pos = torch.full((B, n), 400, dtype=torch.int32, device=device())
    ref_pool, ref_lens = pool.clone(), lens.clone()
    ref = []
    for i in range(3):
        tk.twinkv_cache_append(k, v, pos, ref_pool, table, ref_lens, out={"lens": ref_lens})
        ref.append(tk.twinkv_cache_attend(q, ref_pool, table, ref_lens, window=200,
                                          n_sink=4)["out"])
        pos += 1
    pos.fill_(400)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    first = tk.twinkv_cache_append(k, v, pos, pool, table, lens, out={"lens": lens},
                                   stream=stream)
    out = tk.twinkv_cache_attend(q, pool, table, lens, window=200, n_sink=4, stream=stream)
    stream.synchronize()
    assert torch.equal(out["out"], ref[0])
    out.update(first)
    ws = tk.cache_attend_workspace(q.shape, H, device())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tk.twinkv_cache_append(k, v, pos, pool, table, lens,
                               out={"lens": lens, "status": first["status"]})
        res = tk.twinkv_cache_attend(q, pool, table, lens, window=200, n_sink=4, ws=ws,
                                     out={"out": out["out"]})
    for i in (1, 2):
        pos.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res["out"], ref[i])
    assert torch.equal(lens, ref_lens) and tk.twinkv_get_last_error() == tk.OK


# ---------------------------------------------------------------- what lies beyond the arrays

def guarded(n, dtype=torch.uint8):
    """n elements inside a larger array whose other bytes are 0xA5, and a check that they still are."""
    size = n * torch.empty(0, dtype=dtype).element_size()
    store = torch.full((size + 8192,), 0xA5, dtype=torch.uint8, device=device())

    def whole():
        return bool(store[:4096].eq(0xA5).all() and store[4096 + size:].eq(0xA5).all())

    return store[4096:4096 + size].view(dtype), whole


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 5, 8, 9, 16, 33])
def test_attend_stays_inside_its_workspace(d, G):
    """Enough pages that every warp of the grid has some, for every kernel."""
    H, length = 2, 170000
    pages = -(-length // 64)
    pool = torch.zeros((100, R.PAGE_BYTES[d]), dtype=torch.uint8, device=device())
    table = torch.randint(0, 100, (1, H, pages), device=device()).int()
    lens = torch.full((1, H), length, dtype=torch.int32, device=device())
    q = torch.randn(1, 1, H * G, d, device=device()).to(torch.bfloat16)
    ws, whole = guarded(tk._attend_workspace_size(1, 1, H * G, H, d))
    out, whole_out = guarded(H * G * d, torch.bfloat16)
    res = tk.twinkv_cache_attend(q, pool, table, lens, ws=ws, window=150000, n_sink=4,
                                 out={"out": out.view(1, 1, H * G, d)})
    torch.cuda.synchronize()
    assert whole() and whole_out() and not res["out"].any()


@pytest.mark.parametrize("d", [64, 128])
def test_moves_stay_inside_their_arrays(d):
    U, N = 3, 321
    ids = np.arange(18, dtype=np.int32).reshape(1, U, 6)
    flat, whole_pool = guarded(18 * R.PAGE_BYTES[d])
    pool = flat.view(18, R.PAGE_BYTES[d])
    x = torch.randn(1, U, N, d, device=device()).to(torch.bfloat16)
    mask = torch.ones(1, U, N, dtype=torch.uint8, device=device())
    ws, whole_ws = guarded(tk._move_workspace_size(U, N))
    lens = tk.twinkv_cache_pack(x, x, mask, pool, put(ids), ws=ws)["lens"]
    mask[0, 1] = 0
    new, whole_new = guarded(18 * R.PAGE_BYTES[d])
    both = torch.cat([pool, new.view(18, -1)])
    out = tk.twinkv_cache_compact(both, put(ids), lens, mask, put(ids + 18), ws=ws)
    pool.copy_(both[18:])
    n = 7
    k, whole_k = guarded(U * n * d, torch.bfloat16)
    v, whole_v = guarded(U * n * d, torch.bfloat16)
    pos, whole_pos = guarded(U * n, torch.int32)
    tk.twinkv_cache_append(x[:, :, :n].transpose(1, 2), x[:, :, :n].transpose(1, 2),
                           torch.full((1, n), 400, dtype=torch.int32, device=device()), pool,
                           put(ids), out["lens"], out={"lens": out["lens"]})
    got = tk.twinkv_cache_read(pool, put(ids), out["lens"], n, last=True,
                               out={"keys": k.view(1, U, n, d), "values": v.view(1, U, n, d),
                                    "positions": pos.view(1, U, n)})
    assert got["positions"].eq(400).all()
    torch.cuda.synchronize()
    assert all(w() for w in (whole_pool, whole_ws, whole_new, whole_k, whole_v, whole_pos))
