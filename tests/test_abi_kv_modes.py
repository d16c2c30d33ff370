"""Sizes and argument errors of kv_attn_sinks and kv_attn_shared, without a GPU: every refusal returns before any device work
(the pointers are dummies)."""
import ctypes

import pytest

ARG, WORKSPACE, UNSUPPORTED = 1, 4, 6
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4098)
NULL = ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def Q():
    import paper_2309_01885_amd.qe as Q
    Q.load()
    return Q


COMMON = [dict(q=NULL), dict(pages=NULL), dict(pages=ctypes.c_void_p(4104)), dict(table=NULL), dict(lengths=NULL), dict(out=NULL),
          dict(dtype=7), dict(total=-1), dict(total=1 << 31), dict(heads=0), dict(heads=7), dict(dim=65), dict(batch=-1), dict(max_q=-1),
          dict(num=0), dict(page=33), dict(kv=0), dict(kv=3), dict(group=1), dict(width=-1), dict(scale=float("inf")),
          dict(scale=float("nan")), dict(causal=0, slopes=P), dict(start=NULL, total=5), dict(q=ctypes.c_void_p(4097)),
          dict(out=ctypes.c_void_p(4097)), dict(table=ODD), dict(lengths=ODD), dict(start=ODD), dict(slopes=ODD), dict(lse=ODD),
          dict(ws=ctypes.c_void_p(4104))]


def _sinks(Q, q=P, dtype=2, total=4, heads=8, dim=64, start=P, batch=2, max_q=2, pages=P, num=2, page=64, kv=2, group=64, table=P,
           width=1, lengths=P, scale=0.1, causal=1, window=10, sinks=3, slopes=NULL, out=P, lse=NULL, ws=P, ws_bytes=1 << 40):
    return Q.load().qe_kv_attn_sinks(q, dtype, total, heads, dim, heads * dim, dim, start, batch, max_q, pages, num, page, kv, group, table,
                                     width, lengths, scale, causal, window, sinks, slopes, out, heads * dim, dim, lse, ws, ws_bytes, NULL)


def test_sinks_refusals(Q):
    none = dict(window=0, sinks=0)
    for bad in COMMON:
        assert _sinks(Q, **{**(none if bad.get("causal") == 0 else {}), **bad}) == ARG, bad
    for bad in (dict(sinks=-1), dict(window=-1), dict(causal=0, window=0), dict(causal=0, sinks=0)):
        assert _sinks(Q, **bad) == ARG, bad
    for bad in (dict(ws=NULL), dict(ws_bytes=100)):
        assert _sinks(Q, **bad) == WORKSPACE, bad
    for empty in (dict(total=0), dict(batch=0), dict(max_q=0)):
        assert _sinks(Q, **empty) == 0
    assert _sinks(Q, batch=1 << 24, total=1 << 25, max_q=1 << 25) == UNSUPPORTED


def _shared(Q, q=P, dtype=2, total=4, heads=8, dim=64, start=P, batch=2, max_q=2, pages=P, num=2, page=64, kv=2, group=64, table=P,
            width=1, lengths=P, groups=P, shared=P, ngroups=1, scale=0.1, causal=1, slopes=NULL, out=P, lse=NULL, ws=P, ws_bytes=1 << 40):
    return Q.load().qe_kv_attn_shared(q, dtype, total, heads, dim, heads * dim, dim, start, batch, max_q, pages, num, page, kv, group, table,
                                      width, lengths, groups, shared, ngroups, scale, causal, slopes, out, heads * dim, dim, lse, ws,
                                      ws_bytes, NULL)


def test_shared_refusals(Q):
    for bad in COMMON + [dict(groups=NULL), dict(shared=NULL), dict(groups=ODD), dict(shared=ODD), dict(ngroups=-1), dict(ngroups=1 << 21)]:
        assert _shared(Q, **bad) == ARG, bad
    for bad in (dict(ws=NULL), dict(ws_bytes=100)):
        assert _shared(Q, **bad) == WORKSPACE, bad
    for empty in (dict(total=0), dict(batch=0), dict(max_q=0)):
        assert _shared(Q, **empty) == 0


def test_shared_workspace_size(Q):
    f, plain = Q.kv_attn_shared_workspace_size, Q.kv_attn_workspace_size
    # no groups, one sequence, more groups than the lists take: kv_attn's
    assert f(8, 8, 1, 32, 8, 128, 0) == f(8, 8, 1, 32, 8, 128, 5000) == plain(8, 8, 1, 32, 8, 128)
    assert f(1, 1, 1, 32, 8, 128, 1) == plain(1, 1, 1, 32, 8, 128)
    # rows of the results of 64 sequences of one token, in tiles of 32 and 16 rows, 512 entries beyond the units at least
    assert f(64, 64, 1, 32, 8, 128, 1) > 256 + (64 + 512) * 32 * 130 * 4 + (512 + 512) * 16 * 130 * 4
    # chunks whose rows fill tiles by themselves in kv_attn's many-row form are kv_attn's: no room for every row
    assert f(131072, 64, 2048, 32, 8, 128, 1) == plain(131072, 64, 2048, 32, 8, 128)
    for bad in ((1, 1, 1, 32, 5, 128, 1), (1, 1, 1, 32, 8, 100, 1), (-1, 1, 1, 32, 8, 128, 1), (1, 1, 1, 32, 8, 128, -1)):
        assert f(*bad) == 0, bad
