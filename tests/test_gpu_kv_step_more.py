"""A serving step's calls where they leave or skip something: a stack that overflows, a recorded
append whose tokens change, first tokens whose page is absent."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from parity import dev, host
from test_gpu_kv import DT, bits, cache, check, draw, f64, rounded
from test_gpu_kv_step import Pool, tables

pytestmark = pytest.mark.gpu


def i32(x):
    return np.asarray(x, np.int32)


@pytest.mark.parametrize("batch", [2, 1100])
def test_extend_stack_overflow_stays_inside(qe, batch):
    """More pages come back than the stack has room for (a mistake of the program's): the entries beside the stack, the table, the lengths and
    the outputs stay as they were, the rest is the plain form's."""
    lengths = [320, 96] + [0] * (batch - 2)
    p = Pool(lengths, 32, 20, 3)
    p.free_count = p.free.size - 2

    def inside(x):
        room = torch.full((x.size + 128,), 0x5A5A5A5A, dtype=torch.int32, device="cuda")
        part = room[64:64 + x.size].view(x.shape)
        part.copy_(dev(x))
        return room, part

    rooms = []
    for name in ("table", "lengths", "free"):
        room, part = inside(getattr(p, name))
        setattr(p, "d" + name, part)
        rooms.append(room)
    p.dcount = dev(i32([p.free_count]))
    for name, n, dtype in (("slots", 1, torch.int64), ("positions", 1, torch.int32), ("q_start", batch + 1, torch.int32)):
        rooms.append(torch.full((n + 128,), 0x5A5A5A5A, dtype=dtype, device="cuda"))
        p.__dict__.setdefault("outs", {})[name] = rooms[-1][64:64 + n]
    assert p.step(qe, [-320, 1] + [0] * (batch - 2), 1, **p.outs)[5]
    assert p.free_count == p.free.size - 1                  # (what is taken lies where the stack has no room: no page)
    for room in rooms:
        assert bool((room[:64] == 0x5A5A5A5A).all()) and bool((room[-64:] == 0x5A5A5A5A).all())


@pytest.mark.parametrize("heads,dim,rot,interleaved", [(4, 64, 64, False), (7, 128, 36, True)])
@pytest.mark.parametrize("dtype", list(DT))
def test_append_replayed(qe, dtype, heads, dim, rot, interleaved):
    """A recorded append: queries, keys, values, positions and slots change between the replays, some tokens are skipped, others
    have no slot; the whole cache is compared after each."""
    tokens, kv, page = 40, 2, 32
    cos, sin = tables(100, rot)
    w = np.linspace(0.5, 2.0, dim, dtype=np.float32)
    pages = qe.kv_pages(4, kv, dim, 32, page)
    pages.fill_(0xAB)
    expect = host(pages)
    q, k, v = (torch.zeros(tokens, h, dim, dtype=DT[dtype], device="cuda") for h in (heads, kv, kv))
    slots, positions = dev(np.full(tokens, -1, np.int64)), dev(np.zeros(tokens, np.int32))
    out = torch.full((tokens, heads, dim), 7.0, dtype=DT[dtype], device="cuda")
    d = [dev(x) for x in (cos, sin, w)]

    def call():
        qe.kv_append(q, k, v, slots, pages, group=32, positions=positions, cos=d[0], sin=d[1], interleaved=interleaved, q_weight=d[2],
                     k_weight=d[2], out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert np.array_equal(host(pages), expect)              # (no slot: nothing is written)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    want_q = out.cpu().clone()
    r = np.random.default_rng(heads)
    for n in range(4):
        new = [draw((tokens, h, dim), 50 + 10 * n + y, dtype) for y, h in enumerate((heads, kv, kv))]
        at, pos = r.permutation(4 * page)[:tokens], i32(r.integers(0, 100, tokens))
        if n % 2 == 0:
            at = np.arange(tokens) + 32 * n // 2            # (whole records)
        pos[r.integers(0, tokens, 2)], at[r.integers(0, tokens, 2)] = -1, -1
        for t, x in zip((q, k, v, slots, positions), new + [torch.from_numpy(at.astype(np.int64)), torch.from_numpy(pos)]):
            t.copy_(x.cuda())
        graph.replay()
        torch.cuda.synchronize()
        there = pos >= 0
        how = (w, 1e-6, np.maximum(pos, 0), cos, sin, interleaved)
        okv.write(expect, np.where(there, at, -1), okv.norm_rotate(f64(k), *how), f64(v), 32)
        keep = torch.from_numpy(there)
        want_q[keep] = rounded(okv.norm_rotate(f64(q), *how), dtype)[keep]
        assert np.array_equal(host(pages), expect), n
        assert np.array_equal(bits(out), bits(want_q)), n


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("nq", [1, 9])
def test_sinks_without_the_first_page(qe, dtype, nq):
    """The page of the first 32 tokens is absent: a row's result is attention over the tokens that are left of what it sees, 32 to 39 and
    its window."""
    length, window, sinks = 400, 64, 40
    pages, table, [(k, v)] = cache(qe, [length], 2, 64, 64, 32, dtype, seed=5)
    table[0, 0] = 10 ** 6
    q = draw((nq, 4, 64), 9, dtype).cuda()
    lse = torch.full((nq, 4), 5.0, device="cuda")
    ws = qe.workspace(qe.kv_attn_workspace_size(nq, 1, nq, 4, 2, 64), "cuda")
    out = qe.kv_attn(q, pages, dev(table), dev(i32([length])), window=window, sinks=sinks, ws=ws, max_q=nq, lse=lse)
    assert qe.sync_status(ws) == qe.QE_ERR_ARG
    t = np.arange(length)
    for i in range(nq):
        pos = length - nq + i
        see = (t >= 32) & (t <= pos) & ((t > pos - window) | (t < sinks))
        check(out[i:i + 1], lse[i:i + 1], q[i:i + 1], [(k[see], v[see])], [1], 0.125, dtype)
