"""Argument errors of the operators that make a retained set, found on the host: no GPU is needed,
and nothing is enqueued."""
import pytest
import torch

from paper_2608_27128_gb300 import twinkv as tk
from test_cache_binding import on_device

FAKE = 1 << 20                      # never dereferenced: validation fails first
OFF = FAKE + 8
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return tk.load()


def prompt(**kw):
    s = dict(B=2, H=2, Hq=8, d=128, tokens=100, keys=100, q_token=1024, q_head=128, k_token=256,
             k_head=128, v_token=256, v_head=128)
    s.update(kw)
    return tk.Prompt(*[s[n] for n, _ in tk.Prompt._fields_])


def seqs(offsets=FAKE, lens=None, k_offsets=None, k_lens=None):
    return tk.Sequences(offsets, lens, k_offsets, k_lens)


BAD_SIZES = [dict(B=0), dict(H=0), dict(Hq=0), dict(Hq=7), dict(d=96), dict(tokens=0), dict(keys=0)]
BEYOND = [dict(tokens=(1 << 24) + 1), dict(keys=(1 << 24) + 1), dict(B=65536), dict(H=1, Hq=129)]
BAD_STRIDES = [dict(q_token=1028), dict(q_head=4), dict(k_token=252), dict(k_head=132),
               dict(q_head=0), dict(k_token=0), dict(k_head=-128), dict(q_token=-1024)]


def test_sizes(lib):
    for size in (lib.twinkv_prompt_attend_workspace, lib.twinkv_prompt_weights_workspace):
        assert size(prompt()) > 0 and size(prompt()) % 256 == 0
        for kw in BAD_SIZES + BEYOND:
            assert size(prompt(**kw)) == 0, kw
    size = lib.twinkv_cache_weights_workspace
    assert size(tk.Queries(2, 8, 32, 1, 0, 0, 0), 128) >= 2 * 8 * 2 * 4
    for B, H, Hq, n, d in ((0, 8, 32, 1, 128), (2, 8, 30, 1, 128), (2, 8, 32, 65, 128),
                           (2, 8, 32, 1, 96)):
        assert size(tk.Queries(B, H, Hq, n, 0, 0, 0), d) == 0


COMMON = ([dict(q=None), dict(k=None), dict(q=OFF), dict(k=OFF), dict(status=FAKE + 2),
           dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(window=-1),
           dict(n_sink=-1), dict(at=seqs(offsets=None)), dict(at=seqs(offsets=FAKE + 1)),
           dict(at=seqs(lens=FAKE + 2)), dict(at=seqs(k_offsets=FAKE + 1)),
           dict(at=seqs(k_lens=FAKE + 1))]
          + [dict(s=prompt(**kw)) for kw in BAD_SIZES + BAD_STRIDES])


def test_attend_arguments(lib):
    def call(q=FAKE, k=FAKE, v=FAKE, s=None, at=None, scale=0.1, window=0, n_sink=0,
             out=2 * FAKE, lse=FAKE, status=FAKE, ws=FAKE, wsb=BIG):
        return lib.twinkv_prompt_attend(q, k, v, s or prompt(), at or seqs(), scale, window, n_sink,
                                        out, lse, status, ws, wsb, None)

    assert call(out=FAKE) == tk.ERR_INVALID_ARG            # what it reads
    for kw in COMMON + [dict(v=None), dict(v=OFF), dict(out=None), dict(out=OFF),
                        dict(lse=FAKE + 2), dict(s=prompt(v_token=4)), dict(s=prompt(v_head=0))]:
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    for kw in BEYOND:
        assert call(s=prompt(**kw)) == tk.ERR_UNSUPPORTED, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(wsb=1)):
        assert call(**kw) == tk.ERR_WORKSPACE, kw


def test_weights_arguments(lib):
    def call(q=FAKE, k=FAKE, lse=FAKE, s=None, at=None, scale=0.1, window=0, n_sink=0, last=0,
             score=FAKE, out=FAKE, status=FAKE, ws=FAKE, wsb=BIG):
        return lib.twinkv_prompt_weights(q, k, lse, s or prompt(), at or seqs(), scale, window,
                                         n_sink, last, score, out, status, ws, wsb, None)

    for kw in COMMON + [dict(lse=None), dict(lse=FAKE + 2), dict(last=-1), dict(score=FAKE + 2),
                        dict(out=None), dict(out=FAKE + 1)]:
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    for kw in BEYOND:
        assert call(s=prompt(**kw)) == tk.ERR_UNSUPPORTED, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(wsb=1)):
        assert call(**kw) == tk.ERR_WORKSPACE, kw


def test_cache_weights_arguments(lib):
    def call(q=FAKE, lse=FAKE, s=None, scale=0.1, window=0, n_sink=0, pool=None, table=FAKE, pages=4,
             lens=FAKE, score=FAKE, out=FAKE, N=256, status=None, ws=FAKE, wsb=BIG):
        return lib.twinkv_cache_weights(q, lse, s or tk.Queries(1, 2, 8, 1, 1024, 1024, 128), scale,
                                        window, n_sink, pool or tk.Pool(FAKE, 10, 128), table, pages,
                                        lens, score, out, N, status, ws, wsb, None)

    for kw in (dict(q=None), dict(q=OFF), dict(lse=None), dict(lse=FAKE + 2), dict(lens=None),
               dict(score=None), dict(out=None), dict(N=0), dict(N=(1 << 20) + 1), dict(scale=NAN),
               dict(scale=0.0), dict(window=-1), dict(n_sink=-1), dict(table=None), dict(pages=0),
               dict(pool=tk.Pool(FAKE, 10, 96)), dict(pool=tk.Pool(None, 10, 128)),
               dict(pool=tk.Pool(FAKE, 0, 128)), dict(status=FAKE + 1),
               dict(s=tk.Queries(1, 2, 7, 1, 1024, 1024, 128)),
               dict(s=tk.Queries(1, 2, 8, 0, 1024, 1024, 128)),
               dict(s=tk.Queries(1, 2, 8, 1, 1028, 1024, 128))):
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    for s in (tk.Queries(1, 2, 8, 65, 1024, 1024, 128), tk.Queries(1, 1, 257, 1, 0, 0, 128)):
        assert call(s=s) == tk.ERR_UNSUPPORTED
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(wsb=1)):
        assert call(window=5, **kw) == tk.ERR_WORKSPACE, kw


def test_policy_arguments(lib):
    def call(score=FAKE, units=4, N=100, lens=FAKE, budget=FAKE, n_sink=4, n_recent=64, mask=FAKE,
             out=OFF, status=FAKE):
        return lib.twinkv_weight_policy(score, units, N, lens, budget, n_sink, n_recent, mask, out,
                                        status, None)

    for kw in (dict(score=None), dict(budget=None), dict(mask=None), dict(score=FAKE + 2),
               dict(lens=FAKE + 1), dict(budget=FAKE + 1), dict(out=FAKE + 2), dict(status=FAKE + 2),
               dict(out=FAKE), dict(units=0), dict(units=65536), dict(N=0), dict(N=(1 << 20) + 1),
               dict(n_sink=-1), dict(n_recent=-1)):
        assert call(**kw) == tk.ERR_INVALID_ARG, kw


# ---------------------------------------------------------------- the binding

def rows(*shape, dtype=torch.bfloat16):
    return on_device(torch.zeros(shape, dtype=dtype))


@pytest.fixture
def device0(monkeypatch):
    monkeypatch.setattr(tk, "_current_device", lambda: 0)


def test_binding_refuses_prompts(device0):
    q, k = rows(10, 8, 128), rows(10, 2, 128)
    i32 = lambda *x: on_device(torch.tensor(x, dtype=torch.int32))
    for args, kw in (((q.float(), k, k), {}), ((q, k.float(), k), {}), ((q, k, rows(9, 2, 128)), {}),
                     ((rows(10, 7, 128), k, k), {}), ((rows(10, 8, 64), k, k), {}),
                     ((rows(10, 8, 128)[0], k, k), {}), ((q, k, None), {}),
                     ((q, rows(10, 2, 132)[..., :128], k), {}),
                     ((q, rows(10, 1, 128).expand(10, 2, 128), k), {}),
                     ((rows(1, 8, 128).expand(10, 8, 128), k, k), {}),
                     ((q, k, k), dict(offsets=i32(0))), ((q, k, k), dict(offsets=[0, 10])),
                     ((q, k, k), dict(offsets=i32(0, 10).long())),
                     ((q, k, k), dict(offsets=i32(0, 10), lens=i32(3, 4))),
                     ((q, k, k), dict(offsets=i32(0, 10), k_offsets=i32(0, 5, 10))),
                     ((rows(0, 8, 128), k, k), {}), ((q, rows(0, 2, 128), rows(0, 2, 128)), {})):
        with pytest.raises((ValueError, TypeError)):
            tk.twinkv_prompt_attend(*args, **kw)
    with pytest.raises((ValueError, TypeError)):
        tk.twinkv_prompt_weights(q, k, rows(10, 8))                    # lse has to be float32
    with pytest.raises((ValueError, TypeError)):
        tk.twinkv_prompt_weights(q, k, rows(8, 10, dtype=torch.float32))
    with pytest.raises((ValueError, TypeError)):
        tk.twinkv_prompt_attend(torch.zeros(10, 8, 128, dtype=torch.bfloat16), k, k)
    with pytest.raises(tk.TwinKVError) as e:
        tk.twinkv_prompt_attend(rows(3, 129, 64), rows(3, 1, 64), rows(3, 1, 64))
    assert e.value.status == tk.ERR_UNSUPPORTED


def test_binding_refuses_policies(device0):
    score = rows(2, 100, dtype=torch.float32)
    i32 = lambda *x: on_device(torch.tensor(x, dtype=torch.int32))
    for args, kw in (((score.double(), i32(1, 2)), {}), ((score, i32(1)), {}),
                     ((score, i32(1, 2).long()), {}), ((score, i32(1, 2)), dict(lens=i32(1))),
                     ((score.t(), i32(1, 2)), {}), ((score, i32(1, 2)), dict(n_sink=2 ** 32)),
                     ((torch.zeros(2, 100), i32(1, 2)), {})):
        with pytest.raises((ValueError, TypeError)):
            tk.twinkv_weight_policy(*args, **kw)


def test_workspaces_of_the_binding():
    assert tk.prompt_attend_workspace((10, 8, 128), (20, 2, 128), 3, "cpu").numel() > 0
    for q, k, B in (((10, 8, 128), (20, 2, 64), 1), ((10, 8, 128), (20, 3, 128), 1),
                    ((10, 8, 128), (20, 2, 128), 0)):
        with pytest.raises(ValueError):
            tk.prompt_weights_workspace(q, k, B, "cpu")
    with pytest.raises(ValueError):
        tk.cache_weights_workspace((1, 65, 8, 128), 2, "cpu")
