"""What the calls of a serving step make for themselves is made with the call's stream as the current one (as
test_stream_buffers.py has it for the others)."""
import torch

import paper_2309_01885_amd.qe as Q
from test_stream_buffers import Stream, calls  # noqa: F401


def test_step_calls(calls, monkeypatch):  # noqa: F811
    monkeypatch.setattr(Q, "_gpu", lambda t, name: t.get_device())
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda t, *shape, **kw: torch.empty(*shape, **kw))    # (recorded)
    s = Stream()
    i32 = lambda *shape: torch.ones(shape, dtype=torch.int32)  # noqa: E731
    q, k, pages = torch.ones((3, 4, 64)), torch.ones((3, 2, 64)), torch.ones((4, 2, 2, 64), dtype=torch.uint8)
    made = 0
    for call, n in ((lambda: Q.kv_extend(i32(3), i32(3, 2), i32(3), i32(6), i32(1), 32, 4, stream=s), 4),
                    (lambda: Q.kv_append(q, k, k, torch.ones(3, dtype=torch.int64), pages, stream=s), 1),
                    (lambda: Q.kv_attn(q, pages, i32(3, 1), i32(3), window=5, sinks=2, stream=s), 2),
                    (lambda: Q.kv_attn_sinks(q, pages, i32(3, 1), i32(3), 5, 2, stream=s), 2),
                    (lambda: Q.kv_attn_shared(q, pages, i32(3, 1), i32(3), i32(2), i32(1), stream=s), 2)):
        before = len(calls["made"])
        call()
        assert calls["made"][before:].count(s) == n, call
        made += 1
        assert calls["stream"] == [77] * made


def test_calls_of_another_gpu(calls, monkeypatch):  # noqa: F811
    """Tensors on another GPU than the current one: the call is made with theirs as the current one."""
    import contextlib
    now, entered = [0], []

    @contextlib.contextmanager
    def device(dev):
        entered.append(dev)
        before, now[0] = now[0], dev
        yield
        now[0] = before

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(Q, "_elsewhere", lambda dev: dev != now[0])
    monkeypatch.setattr(Q, "_gpu", lambda t, name: t.get_device())
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda t, *shape, **kw: torch.empty(*shape, **kw))
    i32 = lambda *shape: torch.ones(shape, dtype=torch.int32)  # noqa: E731
    s, q, k, pages = Stream(), torch.ones((3, 4, 64)), torch.ones((3, 2, 64)), torch.ones((4, 2, 2, 64), dtype=torch.uint8)
    for call in (lambda: Q.kv_extend(i32(3), i32(3, 2), i32(3), i32(6), i32(1), 32, 4, stream=s),
                 lambda: Q.kv_append(q, k, k, torch.ones(3, dtype=torch.int64), pages, stream=s),
                 lambda: Q.kv_attn(q, pages, i32(3, 1), i32(3), window=5, sinks=2, stream=s),
                 lambda: Q.kv_attn_shared(q, pages, i32(3, 1), i32(3), i32(2), i32(1), stream=s)):
        assert call() is not None
    assert entered == [-1] * 4 and calls["stream"] == [77] * 4 and now == [0]
