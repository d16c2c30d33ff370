"""What a call makes for itself (output, workspace) is made with the call's stream as the current one:
filled before its kernels run, and not handed to other work before they end.

Shown without a GPU: the library call and torch's stream switch are replaced by records of the order
in which they happen."""
import contextlib

import pytest
import torch

import paper_2309_01885_amd.qe as Q


class Stream:
    cuda_stream = 77


@pytest.fixture
def calls(monkeypatch):
    """Where each allocation was made (None: torch's own current stream), and the streams of the library calls."""
    seen = {"made": [], "stream": []}
    state = {"now": None}

    @contextlib.contextmanager
    def switch(stream):
        before, state["now"] = state["now"], stream
        yield
        state["now"] = before

    def record(make):
        def made(*args, **kw):
            kw.pop("device", None)
            seen["made"].append(state["now"])
            return make(*args, **kw)
        return made

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_size") or name.endswith("_bytes"):
                return lambda *args: 1024
            return lambda *args: seen["stream"].append(getattr(args[-1], "value", args[-1])) or 0

    monkeypatch.setattr(torch.cuda, "stream", switch)
    for name in ("empty", "zeros", "empty_like", "full"):
        monkeypatch.setattr(torch, name, record(getattr(torch, name)))
    monkeypatch.setattr(Q, "load", lambda: Lib())
    monkeypatch.setattr(Q, "_pages", lambda pages, dim, group: (4, 64, 2, -1))
    return seen


def test_kv_calls(calls):
    s = Stream()
    q, pages = torch.ones((3, 4, 64)), torch.ones((4, 2, 2, 64), dtype=torch.uint8)
    table, lengths = torch.ones((3, 1), dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    Q.kv_attn(q, pages, table, lengths, stream=s)
    assert calls["made"] == [s, s] and calls["stream"] == [77]
    Q.kv_read(pages, torch.ones(5, dtype=torch.int64), 64, stream=s)
    assert calls["made"] == [s] * 4 and calls["stream"] == [77] * 2


def test_other_calls(calls, monkeypatch):
    """The quantizer's calls: every buffer of theirs, too."""
    s = Stream()
    monkeypatch.setattr(Q, "_ptr", lambda t, *args, **kw: Q._vp(None))
    W, S, codes = torch.ones((8, 16)), torch.ones((16, 16)), torch.ones((8, 16), dtype=torch.uint8)
    idx, nnz, row = torch.ones(3, dtype=torch.int64), torch.ones(1, dtype=torch.int64), torch.ones(8)
    Q.gram(W, stream=s, check=False)
    Q.grid_minmax(W, 4, stream=s)
    Q.cd_sweep(W, S, 4, row, row, W, codes, W, 1, stream=s, check=False)
    Q.cd_outlier_sweep(W, S, 4, row, row, W, codes, W, W, 3, 1.0, idx, nnz, 1, stream=s, check=False)
    Q.topk_abs(W, 3, stream=s, check=False)
    Q.topk_columns(W, 3, stream=s, check=False)
    Q.pack_codes(codes, 4, stream=s)
    Q.outliers_csr(W, idx, nnz, stream=s)
    Q.objective(W, W, S, stream=s, check=False)
    Q.lambda_max(S, stream=s)
    assert len(calls["made"]) == 2 + 2 + 1 + 1 + 4 + 5 + 1 + 3 + 2 + 1
    assert all(m is s for m in calls["made"]), calls["made"]
    assert calls["stream"] == [77] * 10
