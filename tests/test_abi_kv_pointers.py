"""Pointers that are no multiple of what is read through them are refused before any device work: an atomic or a
wide access at such an address faults.  Without a GPU (the pointers are dummies)."""
import ctypes

import pytest

from test_abi_kv import ARG, _attn, _read, _write

AT = {n: ctypes.c_void_p(4096 + n) for n in (1, 2, 4, 8)}
P, NULL = ctypes.c_void_p(4096), ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def Q():
    import paper_2309_01885_amd.qe as Q
    Q.load()
    return Q


@pytest.mark.parametrize("call", [_write, _read])
def test_slots(Q, call):
    assert call(Q, slots=AT[4]) == ARG


@pytest.mark.parametrize("at", [1, 2])
def test_status(Q, at):
    lib = Q.load()
    assert lib.qe_kv_write(P, P, 0, 4, 2, 64, 128, 64, 128, 64, P, 64, P, 2, 64, AT[at], NULL) == ARG
    assert lib.qe_kv_read(P, 2, 64, P, 4, 2, 64, 64, P, P, 0, 128, 64, 128, 64, AT[at], NULL) == ARG


@pytest.mark.parametrize("at", [1, 2, 4, 8])
def test_workspace(Q, at):
    assert _attn(Q, ws=AT[at]) == ARG


@pytest.mark.parametrize("at", [1, 2])
@pytest.mark.parametrize("name", ["start", "table", "lengths", "slopes", "lse"])
def test_arrays(Q, name, at):
    assert _attn(Q, **{name: AT[at]}) == ARG
