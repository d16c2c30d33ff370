"""Sizes and argument errors of kv_extend and kv_append, without a GPU: every refusal returns before any device work (the
pointers are dummies)."""
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


def test_extend_workspace_size(Q):
    f = Q.kv_extend_workspace_size
    assert f(0) >= 256 and f(-1) == 0 and f((1 << 20) + 1) == 0
    assert f(1000) >= 256 + 16000


def _extend(Q, counts=P, batch=3, table=P, width=4, lengths=P, keep=NULL, free=P, num=9, count=P, page=64, total=5, slots=P,
            positions=P, start=P, lacking=NULL, ws=P, ws_bytes=1 << 30):
    return Q.load().qe_kv_extend(counts, batch, table, width, lengths, keep, free, num, count, page, total, slots, positions, start,
                                 lacking, ws, ws_bytes, NULL)


def test_extend_refusals(Q):
    for bad in (dict(counts=NULL), dict(table=NULL), dict(lengths=NULL), dict(free=NULL), dict(count=NULL), dict(slots=NULL),
                dict(positions=NULL), dict(start=NULL), dict(batch=-1), dict(width=-1), dict(num=0), dict(num=1 << 31), dict(page=0),
                dict(page=48), dict(page=-32), dict(total=-1), dict(total=1 << 31), dict(width=1 << 31), dict(counts=ODD), dict(table=ODD),
                dict(lengths=ODD), dict(keep=ODD), dict(free=ODD), dict(count=ODD), dict(positions=ODD), dict(start=ODD),
                dict(lacking=ODD), dict(slots=ctypes.c_void_p(4100)), dict(ws=ctypes.c_void_p(4104))):
        assert _extend(Q, **bad) == ARG, bad
    assert _extend(Q, batch=(1 << 20) + 1) == UNSUPPORTED
    for bad in (dict(ws=NULL), dict(ws_bytes=256)):
        assert _extend(Q, **bad) == WORKSPACE, bad


def _append(Q, q=P, k=P, v=P, dtype=2, tokens=4, heads=8, kv=2, dim=64, qw=P, kw=P, eps=1e-6, positions=P, cos=P, sin=P, rows=10, rot=64,
            slots=P, group=64, pages=P, num=2, page=64, out=P, status=NULL):
    return Q.load().qe_kv_append(q, k, v, dtype, tokens, heads, kv, dim, 512, 64, 128, 64, 128, 64, qw, kw, eps, positions, cos, sin,
                                 rows, rot, 0, slots, group, pages, num, page, out, 512, 64, status, NULL)


def test_append_refusals(Q):
    for bad in (dict(q=NULL), dict(k=NULL), dict(v=NULL), dict(out=NULL), dict(slots=NULL), dict(pages=NULL), dict(positions=NULL),
                dict(cos=NULL), dict(sin=NULL), dict(rows=0), dict(rot=-2), dict(rot=3), dict(rot=66), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(dtype=3), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0),
                dict(kv=0), dict(dim=12), dict(dim=264), dict(group=16), dict(num=0), dict(page=33), dict(pages=ctypes.c_void_p(4104)),
                dict(q=ctypes.c_void_p(4097)), dict(out=ctypes.c_void_p(4097)), dict(qw=ODD), dict(kw=ODD), dict(cos=ODD), dict(sin=ODD),
                dict(positions=ODD), dict(status=ODD), dict(slots=ctypes.c_void_p(4100))):
        assert _append(Q, **bad) == ARG, bad
    assert _append(Q, tokens=0) == 0
