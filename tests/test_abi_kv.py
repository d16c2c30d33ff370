"""Sizes and argument errors of the key/value cache's entry points, without a GPU: every refusal
returns before any device work (the pointers are dummies)."""
import ctypes

import pytest

ARG, WORKSPACE = 1, 4
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)
NULL = ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def Q():
    import paper_2309_01885_amd.qe as Q
    Q.load()
    return Q


def test_page_bytes(Q):
    f = Q.load().qe_kv_page_bytes
    assert f(8, 128, 64, 64) == 8 * 2 * 32 * (128 + 16)
    assert f(1, 8, 32, 32) == 32 * (64 + 16)            # padded to 64 channels
    assert f(2, 80, 128, 96) == 2 * 3 * 32 * (96 + 8)
    assert f(1, 256, 32, 32) == 32 * (256 + 64)
    for bad in ((0, 128, 64, 64), (8, 0, 64, 64), (8, 12, 64, 64), (8, 264, 64, 64), (8, 128, 16, 64),
                (8, 128, 96, 64), (8, 128, 64, 0), (8, 128, 64, 48), (8, 128, 64, -32)):
        assert f(*bad) == 0, bad


def test_workspace_size(Q):
    f = Q.kv_attn_workspace_size
    assert f(0, 0, 0, 8, 8, 64) >= 256
    assert f(1, 1, 1, 32, 8, 128) >= 256
    assert f(1, 1, 1, 32, 5, 128) == 0                  # heads not a multiple of kv_heads
    assert f(1, 1, 1, 0, 1, 128) == 0
    assert f(-1, 1, 1, 8, 8, 128) == 0
    assert f(1, 1, 1, 8, 8, 100) == 0
    # many long chunks need no joining: the size stays small
    assert f(1 << 20, 64, 1 << 14, 32, 8, 128) < (1 << 30)


def _write(Q, K=P, V=P, dtype=0, tokens=4, kv=2, dim=64, slots=P, group=64, pages=P, num=2, page=64):
    return Q.load().qe_kv_write(K, V, dtype, tokens, kv, dim, 128, 64, 128, 64, slots, group, pages, num, page,
                                NULL, NULL)


def _read(Q, K=P, V=P, dtype=0, tokens=4, kv=2, dim=64, slots=P, group=64, pages=P, num=2, page=64):
    return Q.load().qe_kv_read(pages, num, page, slots, tokens, kv, dim, group, K, V, dtype, 128, 64, 128, 64,
                               NULL, NULL)


@pytest.mark.parametrize("call", [_write, _read])
def test_write_and_read_refusals(Q, call):
    for bad in (dict(K=NULL), dict(V=NULL), dict(slots=NULL), dict(pages=NULL), dict(pages=ODD), dict(dtype=3),
                dict(dtype=-1), dict(tokens=-1), dict(kv=0), dict(dim=0), dict(dim=68), dict(dim=264),
                dict(group=0), dict(group=48), dict(page=0), dict(page=40), dict(num=0), dict(num=1 << 40),
                dict(K=ctypes.c_void_p(4097)), dict(V=ctypes.c_void_p(4098)), dict(K=ctypes.c_void_p(4097), dtype=2)):
        assert call(Q, **bad) == ARG, bad
    assert call(Q, tokens=0) == 0
    assert call(Q, tokens=0, K=NULL, V=NULL, slots=NULL) == 0


def _attn(Q, q=P, dtype=2, total=4, heads=8, dim=64, start=P, batch=2, max_q=2, pages=P, num=2, page=64, kv=2,
          group=64, table=P, width=1, lengths=P, scale=0.1, causal=1, window=0, slopes=NULL, out=P, lse=NULL, ws=P,
          ws_bytes=1 << 40):
    return Q.load().qe_kv_attn(q, dtype, total, heads, dim, heads * dim, dim, start, batch, max_q, pages, num, page,
                               kv, group, table, width, lengths, scale, causal, window, slopes, out, heads * dim,
                               dim, lse, ws, ws_bytes, NULL)


def test_attn_refusals(Q):
    for bad in (dict(q=NULL), dict(pages=NULL), dict(pages=ODD), dict(table=NULL), dict(lengths=NULL), dict(out=NULL),
                dict(dtype=7), dict(total=-1), dict(total=1 << 31), dict(heads=0), dict(heads=7), dict(heads=-8),
                dict(dim=65), dict(batch=-1), dict(max_q=-1), dict(num=0), dict(page=33), dict(kv=0), dict(kv=3),
                dict(group=1), dict(width=-1), dict(scale=float("inf")), dict(scale=float("nan")), dict(window=-1),
                dict(causal=0, window=3), dict(causal=0, slopes=P), dict(start=NULL, total=5),
                dict(q=ctypes.c_void_p(4097)), dict(out=ctypes.c_void_p(4097))):
        assert _attn(Q, **bad) == ARG, bad
    for bad in (dict(ws=NULL), dict(ws_bytes=100)):
        assert _attn(Q, **bad) == WORKSPACE, bad
    for empty in (dict(total=0), dict(batch=0), dict(max_q=0)):
        assert _attn(Q, **empty) == 0
