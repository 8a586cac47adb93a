"""Argument errors of the operators around the pass, found on the host: no GPU is needed, and
nothing is enqueued."""
import pytest
import torch

from paper_2608_27128_gb300 import twinkv as tk

FAKE = 1 << 20                      # never dereferenced: validation fails first
OFF = FAKE + 8                      # not on a 16-byte boundary
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return tk.load()


def test_sizes(lib):
    assert {d: lib.twinkv_cache_page_bytes(d) for d in (64, 128)} == tk.PAGE_BYTES
    assert lib.twinkv_cache_page_bytes(96) == 0
    assert lib.twinkv_cache_move_workspace(3, 1000) >= 12000
    for bad in ((0, 10), (65536, 10), (1, 0), (1, (1 << 20) + 1)):
        assert lib.twinkv_cache_move_workspace(*bad) == 0
    size = lib.twinkv_cache_attend_workspace
    assert size(tk.Queries(2, 8, 32, 1, 0, 0, 0), 128) > 0
    for B, H, Hq, n, d in ((0, 8, 32, 1, 128), (2, 8, 30, 1, 128), (2, 8, 32, 0, 128),
                           (2, 8, 32, 65, 128), (2, 8, 32, 1, 96), (1, 1, 257, 1, 64),
                           (8192, 8, 32, 1, 64)):
        assert size(tk.Queries(B, H, Hq, n, 0, 0, 0), d) == 0


def heads(**kw):
    s = dict(tokens=4, heads_q=8, heads_k=2, d=128, dtype=tk.BF16, rows=100, q_token=1280,
             q_head=128, k_token=1280, k_head=128, out_q_token=1024, out_q_head=128,
             out_k_token=256, out_k_head=128)
    s.update(kw)
    return tk.Heads(**s)


def rope(lib, s=None, q=FAKE, k=FAKE, wq=FAKE, cs=FAKE, pos=FAKE, oq=FAKE, eps=1e-6):
    return lib.twinkv_qk_norm_rope(q, k, s or heads(), wq, FAKE, eps, cs, pos, oq, FAKE, None,
                                   None)


def test_rope_arguments(lib):
    for kw in (dict(q=None), dict(k=None), dict(oq=None), dict(cs=None), dict(pos=None),
               dict(q=OFF), dict(wq=OFF), dict(cs=OFF), dict(pos=FAKE + 2),
               dict(eps=float("nan")), dict(eps=-1.0), dict(s=heads(d=96)),
               dict(s=heads(dtype=7)), dict(s=heads(tokens=0)), dict(s=heads(rows=0)),
               dict(s=heads(q_token=1284)), dict(s=heads(out_k_head=4)),
               dict(s=heads(heads_q=0, heads_k=0)), dict(s=heads(heads_q=-1))):
        assert rope(lib, **kw) == tk.ERR_INVALID_ARG, kw


def pool(**kw):
    p = dict(pages=FAKE, n_pages=10, d=128)
    p.update(kw)
    return tk.Pool(**p)


BAD_POOLS = [dict(pages=None), dict(pages=OFF), dict(n_pages=0), dict(d=96)]


def test_pack_arguments(lib):
    def call(keys=FAKE, values=FAKE, s=None, mask=FAKE, p=None, table=FAKE, pages=4, lens=FAKE,
             ws=FAKE, wsb=BIG):
        return lib.twinkv_cache_pack(keys, values, s or tk.Shape(1, 2, 100, 128, tk.BF16), mask,
                                     p or pool(), table, pages, lens, None, ws, wsb, None)

    for kw in (dict(keys=None), dict(values=OFF), dict(table=None), dict(pages=0),
               dict(lens=None), dict(s=tk.Shape(1, 2, 100, 64, tk.BF16)),
               dict(s=tk.Shape(1, 2, 0, 128, tk.BF16)), dict(s=tk.Shape(1, 2, 100, 128, 9)),
               dict(s=tk.Shape(300, 300, 100, 128, tk.BF16)), dict(table=FAKE + 1),
               *[dict(p=pool(**b)) for b in BAD_POOLS]):
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(wsb=100)):
        assert call(**kw) == tk.ERR_WORKSPACE, kw


def test_append_arguments(lib):
    def call(k=FAKE, v=FAKE, n=1, dtype=tk.BF16, stride=1024, pos=FAKE, p=None, lens=FAKE,
             out=FAKE, B=2):
        return lib.twinkv_cache_append(k, v, tk.Rows(B, 2, n, dtype, stride, 128, 128, 1024, 128, 128),
                                       pos, p or pool(), FAKE, 4, lens, out, None, None)

    for kw in (dict(k=None), dict(v=OFF), dict(n=0), dict(dtype=5), dict(stride=1025),
               dict(pos=None), dict(lens=None), dict(out=None), dict(B=0), dict(B=40000),
               *[dict(p=pool(**b)) for b in BAD_POOLS]):
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    assert call(n=65) == tk.ERR_UNSUPPORTED


def test_compact_and_read_arguments(lib):
    def compact(p=None, table=FAKE, lens=FAKE, units=3, keep=FAKE, N=100, new=FAKE, out=FAKE + 64,
                ws=FAKE, wsb=BIG):
        return lib.twinkv_cache_compact(p or pool(), table, 4, lens, units, keep, N, new, 4, out,
                                        None, ws, wsb, None)

    for kw in (dict(table=None), dict(new=None), dict(lens=None), dict(out=None), dict(out=FAKE),
               dict(units=0), dict(units=65536), dict(N=0), dict(N=(1 << 20) + 1),
               *[dict(p=pool(**b)) for b in BAD_POOLS]):
        assert compact(**kw) == tk.ERR_INVALID_ARG, kw
    assert compact(ws=None) == compact(wsb=8) == tk.ERR_WORKSPACE

    def read(p=None, table=FAKE, lens=FAKE, units=3, rows=10, k=FAKE, v=FAKE):
        return lib.twinkv_cache_read(p or pool(), table, 4, lens, units, rows, 0, k, v, None,
                                     None, None)

    for kw in (dict(table=None), dict(lens=None), dict(units=0), dict(rows=0), dict(k=None),
               dict(v=OFF), *[dict(p=pool(**b)) for b in BAD_POOLS]):
        assert read(**kw) == tk.ERR_INVALID_ARG, kw


def test_attend_arguments(lib):
    def call(q=FAKE, s=None, scale=0.1, window=0, n_sink=0, p=None, table=FAKE, pages=4,
             lens=FAKE, out=FAKE, ws=FAKE, wsb=BIG):
        return lib.twinkv_cache_attend(q, s or tk.Queries(2, 2, 8, 1, 1024, 1024, 128), scale,
                                       window, n_sink, p or pool(), table, pages, lens, out,
                                       None, None, ws, wsb, None)

    for kw in (dict(q=None), dict(q=OFF), dict(out=None), dict(lens=None), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")),
               dict(window=-1), dict(n_sink=-1), dict(table=None), dict(pages=0),
               dict(pages=(1 << 14) + 1), dict(s=tk.Queries(2, 3, 8, 1, 1024, 1024, 128)),
               dict(s=tk.Queries(0, 2, 8, 1, 1024, 1024, 128)),
               dict(s=tk.Queries(2, 2, 8, 1, 1024, 1024, 129)),
               *[dict(p=pool(**b)) for b in BAD_POOLS]):
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    for s in (tk.Queries(2, 2, 8, 65, 1024, 1024, 128), tk.Queries(1, 1, 300, 1, 1024, 1024, 128),
              tk.Queries(40000, 2, 8, 1, 1024, 1024, 128)):
        assert call(s=s) == tk.ERR_UNSUPPORTED
    assert call(ws=None) == call(ws=FAKE + 128) == call(wsb=64) == tk.ERR_WORKSPACE


def test_binding_refuses():
    x = torch.zeros(1, 2, 64, 64, dtype=torch.bfloat16)
    for bad in (torch.zeros(4, 100, dtype=torch.uint8), torch.zeros(4864, dtype=torch.uint8),
                torch.zeros(4, 4864, dtype=torch.uint8), "pool"):        # the last shapes: on the CPU
        with pytest.raises((ValueError, TypeError)):
            tk.twinkv_cache_read(bad, torch.zeros(1, 1, dtype=torch.int32),
                                 torch.ones(1, dtype=torch.int32), 4)
        with pytest.raises((ValueError, TypeError)):
            tk.twinkv_cache_pack(x, x, None, bad, torch.zeros(1, 2, 1, dtype=torch.int32))
    with pytest.raises((ValueError, TypeError)):
        tk.twinkv_qk_norm_rope(x[0], x[0], None, None, None, None)
    with pytest.raises(ValueError):
        tk.cache_pool(4, 96)
    with pytest.raises(ValueError):
        tk.cache_attend_workspace((1, 65, 8, 64), 8, "cpu")
    with pytest.raises(ValueError):
        tk.cache_move_workspace(0, 10, "cpu")
