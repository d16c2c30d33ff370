"""Attention of sequences that begin with the same pages (kv_attn_shared), against fp64 arithmetic on the values held;
the bound is derived in test_gpu_kv.py's head (joining two parts of a row adds roundings of 2^-23 of its masses and sums
and, with slopes, one of the distance between the parts, all of which 2^-19 (1 + size) covers).

The lists that kv_attn_shared works by are tested at all sizes through the library's internal entry point, which takes them also
where kv_attn itself would be faster."""
import numpy as np
import pytest
import torch

from parity import dev, host
from test_gpu_kv import DT, check, draw, f64

pytestmark = pytest.mark.gpu


class Always:
    """The library with kv_attn_shared's lists at every size."""

    def __init__(self, lib):
        self.lib = lib
        for public, own in (("qe_kv_attn_shared", "qei_kv_attn_listed"),
                            ("qe_kv_attn_shared_workspace_size", "qei_kv_attn_listed_workspace_size")):
            call = getattr(lib, own)
            call.argtypes, call.restype = getattr(lib, public).argtypes, getattr(lib, public).restype
            setattr(self, public, call)

    def __getattr__(self, name):
        return getattr(self.lib, name)


@pytest.fixture
def listed(qe, monkeypatch):
    import paper_2309_01885_amd.qe as Q
    lib = Always(Q.load())
    monkeypatch.setattr(Q, "load", lambda: lib)
    return qe


def family(qe, parts, kv, dim, group, page, dtype, seed=0, kscale=1.0, spare=1):
    """parts: (shared pages, [lengths with them]) of groups, 0 pages for a sequence alone.  Random bytes elsewhere:
    (pages, table, lens, held, groups, shared)."""
    r = np.random.default_rng(seed)
    lens = [n for _, ls in parts for n in ls]
    width = max([-(-n // page) for n in lens] + [p for p, _ in parts]) + spare
    num = sum(p + len(ls) * width for p, ls in parts) + 2
    pages = qe.kv_pages(num, kv, dim, group, page)
    pages.copy_(torch.randint(0, 256, pages.shape, dtype=torch.uint8, device="cuda",
                              generator=torch.Generator(device="cuda").manual_seed(seed)))
    order = list(r.permutation(num))
    table, held, groups, shared = np.zeros((len(lens), width), np.int32), [], [0], []
    b = 0

    def write(slots, n):
        k, v = (draw((n, kv, dim), seed + 10 * b + y, dtype, kscale if y == 1 else 1.0).cuda() for y in (1, 2))
        qe.kv_write(k, v, dev(slots), pages, group=group)

    for p, ls in parts:
        first = [order.pop() for _ in range(p)]
        at = lambda row, t: row[t // page].astype(np.int64) * page + t % page  # noqa: E731
        if p:
            write(at(np.array(first), np.arange(p * page)), p * page)
        for n in ls:
            table[b, :p] = first
            table[b, p:] = [order.pop() for _ in range(width - p)]
            if n > p * page:
                write(at(table[b], np.arange(p * page, n)), n - p * page)
            held.append(tuple(f64(x) for x in qe.kv_read(pages, dev(at(table[b], np.arange(n))), dim, group=group)))
            b += 1
        groups.append(b)
        shared.append(p)
    return pages, table, lens, held, groups, shared


def i32(x):
    return dev(np.asarray(x, np.int32))


def attend(qe, parts, nqs, heads, kv, dim, group, page, dtype, seed=0, kscale=1.0, slopes=False, give_lse=True, causal=True,
           scale=None, compare=True, wide=0):
    """wide: the table's width (its other entries are no pages), which decides the forms."""
    pages, table, lens, held, groups, shared = family(qe, parts, kv, dim, group, page, dtype, seed, kscale)
    table = np.pad(table, ((0, 0), (0, max(0, wide - table.shape[1]))), constant_values=-1)
    total = sum(nqs)
    q = draw((total, heads, dim), seed + 7, dtype).cuda()
    scale = 1.0 / dim ** 0.5 if scale is None else scale
    sl = (2.0 ** (-8.0 * np.arange(1, heads + 1) / heads)).astype(np.float32) if slopes else None
    lse = torch.full((total, heads), 5.0, device="cuda") if give_lse else None
    start = i32(np.concatenate([[0], np.cumsum(nqs)]))
    out = qe.kv_attn_shared(q, pages, dev(table), i32(lens), i32(groups), i32(shared), group=group, q_start=start, max_q=max(nqs),
                            scale=scale, causal=causal, slopes=None if sl is None else dev(sl), lse=lse, check=True)
    if compare:
        check(out, lse, q, held, nqs, scale, dtype, slopes=sl, causal=causal)
    return out


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dim", [8, 64, 80, 128, 192, 256])
def test_shared_widths(listed, dim, group):
    """Every width and group; few rows of a group and many."""
    for dtype in DT:
        print(f"[shared] dim={dim} group={group} {dtype}", flush=True)
        attend(listed, [(2, [70, 133])], [1, 1], 6, 2, dim, group, 32, dtype, seed=dim)
        attend(listed, [(2, [170, 133, 129])], [9, 3, 17], 6, 3, dim, group, 64, dtype, seed=dim + 1)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (12, 4), (29, 1), (71, 1), (58, 2), (17, 1)])
def test_shared_head_layouts(listed, heads, kv, dtype):
    attend(listed, [(3, [130, 97, 100])], [1, 1, 1], heads, kv, 64, 64, 32, dtype, seed=heads)
    attend(listed, [(1, [130, 70])], [5, 6], heads, kv, 64, 32, 64, dtype, seed=heads + 1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", list(DT))
def test_shared_lengths(listed, dtype, causal):
    """Sequences that end inside the shared pages, before them, that have no queries, more queries than tokens, several
    groups, sequences alone between them, shared pages without a sequence behind them."""
    attend(listed, [(4, [128, 129, 127, 200]), (0, [50]), (2, [64, 64, 63])], [1, 2, 1, 3, 1, 1, 1, 2], 8, 2, 64, 64, 32, dtype, seed=1,
           causal=causal)
    attend(listed, [(4, [128, 0, 150]), (3, [96, 20, 97]), (2, [1, 70])], [1, 1, 2, 0, 0, 5, 1, 1], 4, 2, 128, 64, 32, dtype, seed=2,
           causal=causal)
    attend(listed, [(3, [96, 150, 100]), (1, [3, 2, 40])], [1, 60, 1, 7, 2, 40], 4, 1, 96, 32, 32, dtype, seed=3, causal=causal)
    attend(listed, [(2, [0, 0]), (1, [90])], [1, 2, 1], 4, 4, 64, 64, 32, dtype, seed=4, causal=causal)


@pytest.mark.parametrize("dtype", list(DT))
def test_shared_slopes(listed, dtype):
    attend(listed, [(4, [300, 170, 131])], [1, 1, 2], 20, 20, 80, 32, 32, dtype, seed=3, slopes=True)
    attend(listed, [(2, [200, 170]), (3, [200, 193])], [33, 12, 1, 5], 10, 2, 80, 64, 64, dtype, seed=4, slopes=True)


@pytest.mark.parametrize("dtype", list(DT))
def test_shared_splits(listed, dtype):
    """Long shared and own parts that take many entries each, of one size; both forms."""
    attend(listed, [(40, [2600, 2700, 2561, 4000])], [1, 1, 1, 1], 8, 4, 64, 64, 64, dtype, seed=1)
    attend(listed, [(40, [1290, 1400]), (20, [700, 650])], [20, 3, 1, 9], 16, 2, 128, 128, 32, dtype, seed=2, slopes=True)


@pytest.mark.parametrize("dtype", list(DT))
def test_shared_chunks(listed, dtype):
    """Chunks whose own part takes the many-row form or tiles of 32 rows."""
    attend(listed, [(4, [300, 290])], [150, 140], 3, 1, 64, 64, 64, dtype, seed=1)
    attend(listed, [(2, [300, 128 + 64])], [130, 64], 64, 64, 64, 64, 64, dtype, seed=2, give_lse=False)


@pytest.mark.parametrize("dim,group", [(64, 64), (64, 32), (96, 64), (128, 128), (128, 32), (192, 64), (256, 128), (256, 32)])
@pytest.mark.parametrize("dtype", list(DT))
def test_shared_many_rows(listed, dtype, dim, group):
    """The shared part in the many-row form, beside an own part in the few rows' and in the same; tiles that end inside a group,
    entries of less than a stage, several groups."""
    attend(listed, [(3, [100, 130, 97, 99, 96]), (2, [70, 64, 65])], [3, 1, 3, 2, 1, 3, 1, 2], 32, 1, dim, group, 32, dtype, seed=dim,
           wide=30000)
    attend(listed, [(5, [300, 290])], [70, 90], 4, 2, dim, group, 32, dtype, seed=dim + 1, slopes=True, wide=30000)


@pytest.mark.parametrize("dim,group", [(64, 32), (64, 64), (80, 32), (96, 64), (96, 128), (128, 32), (128, 64), (128, 128), (200, 64)])
@pytest.mark.parametrize("dtype", list(DT))
def test_shared_single_tokens(listed, dtype, dim, group):
    """Many sequences of a token each: shared tiles of 32 rows beside own ones of 16 in one launch, where the width has both."""
    lens = [130 + 7 * y for y in range(12)]
    attend(listed, [(4, lens), (1, [40, 33, 32, 50])], [1] * 16, 12, 2, dim, group, 32, dtype, seed=dim, slopes=group == 64)
    attend(listed, [(30, [n + 960 for n in lens])], [1, 2] * 6, 8, 1, dim, group, 32, dtype, seed=dim + 1)


def test_shared_many_sequences(listed):
    """More sequences than a thread each has, groups of all sizes."""
    r = np.random.default_rng(3)
    parts, nqs = [], []
    while len(nqs) < 1100:
        n = int(r.integers(1, 60))
        p = int(r.integers(0, 3))
        parts.append((p, [p * 32 + int(r.integers(0, 40)) for _ in range(n)]))
        nqs += [int(r.integers(0, 2)) for _ in range(n)]
    attend(listed, parts, nqs, 2, 1, 64, 64, 32, "bf16", seed=5)


def test_shared_many_groups(listed):
    """More groups and sequences than are searched in LDS."""
    attend(listed, [(1, [33, 40])] * 2100 + [(0, [5])] * 4200, [1] * 8400, 1, 1, 64, 64, 32, "f16", seed=6)


def test_shared_keys_far_apart(listed):
    """Scores near one-hot: one part has nearly all the weight."""
    attend(listed, [(4, [200, 150, 129])], [1, 2, 1], 8, 2, 64, 64, 32, "f32", seed=1, kscale=40.0)
    attend(listed, [(4, [200, 150, 129])], [1, 2, 1], 8, 2, 64, 64, 32, "bf16", seed=2, kscale=40.0)


def agree(a, b, dtype):
    """Two calls whose sums are cut differently: both lie within the bound of check, here relative to values of about 1."""
    tol = {"f32": 2.0 ** -16, "f16": 2.0 ** -9, "bf16": 2.0 ** -7}[dtype]
    assert np.all(np.abs(f64(a) - f64(b)) <= tol * (1.0 + np.abs(f64(b))))


def test_shared_without_q_start(listed):
    pages, table, lens, held, groups, shared = family(listed, [(3, [100, 120, 97])], 2, 64, 64, 32, "bf16")
    q = draw((6, 4, 64), 1, "bf16").cuda()
    out = listed.kv_attn_shared(q, pages, dev(table), i32(lens), i32(groups), i32(shared))
    check(out, None, q, held, [2, 2, 2], 64 ** -0.5, "bf16")


def test_shared_rows_of_no_sequence(listed):
    """Rows before the first and behind the last sequence stay; strided queries and outputs."""
    pages, table, lens, held, groups, shared = family(listed, [(3, [100, 120, 97])], 2, 64, 64, 32, "bf16")
    wide = draw((9, 6, 72), 1, "bf16").cuda()
    q = wide[:, 1:5, 4:68]
    room = torch.full((9, 4, 66), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((9, 4), 5.0, device="cuda")
    start = i32([2, 3, 5, 6])
    listed.kv_attn_shared(q, pages, dev(table), i32(lens), i32(groups), i32(shared), q_start=start, max_q=2, out=room[..., 1:65], lse=lse,
                          check=True)
    check(room[2:6, :, 1:65], lse[2:6], q[2:6], held, [1, 2, 1], 64 ** -0.5, "bf16")
    assert bool((room[:2] == 3).all()) and bool((room[6:] == 3).all()) and bool((lse[:2] == 5).all()) and bool((lse[6:] == 5).all())
    assert bool((room[..., 0] == 3).all()) and bool((room[..., 65] == 3).all())


@pytest.mark.parametrize("groups", [[0, 3, 2, 5], [-1, 5], [0, 6], [5, 0], [2, 2, 9]])
def test_shared_bad_groups(listed, groups):
    """Nothing is shared, and the results are kv_attn's."""
    pages, table, lens, held, _, _ = family(listed, [(3, [100, 120, 97, 110, 130])], 2, 64, 64, 32, "f32")
    q = draw((5, 4, 64), 1, "f32").cuda()
    ws = listed.workspace(listed.kv_attn_shared_workspace_size(5, 5, 1, 4, 2, 64, len(groups) - 1), "cuda")
    out = listed.kv_attn_shared(q, pages, dev(table), i32(lens), i32(groups), i32([3] * (len(groups) - 1)), ws=ws)
    assert listed.sync_status(ws) == listed.QE_ERR_ARG
    check(out, None, q, held, [1] * 5, 64 ** -0.5, "f32")


@pytest.mark.parametrize("pages_shared", [-4, 10 ** 6])
def test_shared_bad_counts(listed, pages_shared):
    """A count past the table is cut off at the table (here everything is the same); one below 0 shares nothing."""
    pages, table, lens, held, groups, _ = family(listed, [(5, [100, 120, 160])], 2, 64, 64, 32, "f32", spare=0)
    q = draw((3, 4, 64), 1, "f32").cuda()
    ws = listed.workspace(listed.kv_attn_shared_workspace_size(3, 3, 1, 4, 2, 64, 1), "cuda")
    out = listed.kv_attn_shared(q, pages, dev(table), i32(lens), i32(groups), i32([pages_shared]), ws=ws)
    assert listed.sync_status(ws) == listed.QE_ERR_ARG
    check(out, None, q, held, [1] * 3, 64 ** -0.5, "f32")


@pytest.mark.parametrize("start", [[0, 2, 1, 3], [0, 1, 2, 9], [-1, 1, 2, 3], [0, 3, 0, 3], [0, 1, 3, 2]])
def test_shared_bad_queries(listed, start):
    """Sequences whose rows do not exist are not computed, the others are."""
    pages, table, lens, held, groups, shared = family(listed, [(3, [100, 120, 97])], 2, 64, 64, 32, "f32")
    q = draw((3, 4, 64), 1, "f32").cuda()
    ws = listed.workspace(listed.kv_attn_shared_workspace_size(3, 3, 3, 4, 2, 64, 1), "cuda")
    out = torch.full((3, 4, 64), 3.0, device="cuda")
    listed.kv_attn_shared(q, pages, dev(table), i32(lens), i32(groups), i32(shared), q_start=i32(start), max_q=3, ws=ws, out=out)
    assert listed.sync_status(ws) == listed.QE_ERR_ARG
    assert bool(torch.isfinite(out).all())
    good = [b for b in range(3) if 0 <= start[b] <= start[b + 1] <= 3 and start[b + 1] > start[b]]
    if len(good) == 1:                                      # (rows that two claim are either's)
        a, e = start[good[0]], start[good[0] + 1]
        check(out[a:e], None, q[a:e], [held[good[0]]], [e - a], 64 ** -0.5, "f32")


def test_shared_claimed_rows_do_not_overflow(listed):
    """Many sequences that claim the same rows: more work than the rows of the call can be, all of it inside the workspace."""
    n = 40
    pages, table, lens, held, groups, shared = family(listed, [(3, [100] * n)], 2, 64, 64, 32, "f32")
    q = draw((64, 4, 64), 1, "f32").cuda()
    start = np.tile([0, 64], n // 2).tolist() + [64]
    need = listed.kv_attn_shared_workspace_size(64, n, 64, 4, 2, 64, 20)
    ws = torch.zeros(need + 65536, dtype=torch.uint8, device="cuda")
    ws[need:] = 0x5A
    out = torch.full((64, 4, 64), 3.0, device="cuda")
    pairs = i32(list(range(0, n + 1, 2)))
    listed.kv_attn_shared(q, pages, dev(table), i32(lens), pairs, i32([3] * 20), q_start=i32(start), max_q=64, ws=ws[:need], out=out)
    assert listed.sync_status(ws) == listed.QE_ERR_ARG
    assert bool((ws[need:] == 0x5A).all()) and bool(torch.isfinite(out).all())


def test_shared_bad_lengths_and_pages(listed):
    pages, table, lens, held, groups, shared = family(listed, [(3, [100, 120, 97])], 2, 64, 64, 32, "f32")
    q = draw((3, 4, 64), 1, "f32").cuda()
    size = listed.kv_attn_shared_workspace_size(3, 3, 1, 4, 2, 64, 1)
    for wrong in ([-5, 120, 97], [100, 10 ** 6, 97]):
        ws = listed.workspace(size, "cuda")
        out = listed.kv_attn_shared(q, pages, dev(table), i32(wrong), i32(groups), i32(shared), ws=ws)
        assert listed.sync_status(ws) == listed.QE_ERR_ARG
        check(out[2:], None, q[2:], held[2:], [1], 64 ** -0.5, "f32")
        plain = listed.kv_attn(q, pages, dev(table), i32(wrong), ws=ws)
        assert np.array_equal(np.isfinite(f64(out)), np.isfinite(f64(plain)))
    hole = table.copy()
    hole[:, 1] = -1
    ws = listed.workspace(size, "cuda")
    out = listed.kv_attn_shared(q, pages, dev(hole), i32(lens), i32(groups), i32(shared), ws=ws)
    assert listed.sync_status(ws) == listed.QE_ERR_ARG
    agree(out, listed.kv_attn(q, pages, dev(hole), i32(lens), ws=ws), "f32")


def test_shared_refusals(qe):
    pages, table, lens, _, groups, shared = family(qe, [(3, [100, 120, 97])], 2, 64, 64, 32, "f32")
    q = draw((3, 4, 64), 1, "f32").cuda()
    args = (q, pages, dev(table), i32(lens))
    for g, n in ((i32(groups).long(), i32(shared)), (i32(groups), i32(shared).cpu()), (i32([0, 1, 3]), i32(shared))):
        with pytest.raises(ValueError):
            qe.kv_attn_shared(*args, g, n)
    with pytest.raises(qe.QEError):
        qe.kv_attn_shared(*args, i32(groups), i32(shared), causal=False, slopes=torch.ones(4, device="cuda"))
    with pytest.raises(qe.QEError):
        qe.kv_attn_shared(*args, i32(groups), i32(shared), ws=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert torch.equal(qe.kv_attn_shared(*args, i32([0]), none), qe.kv_attn(*args))
    assert qe.kv_attn_shared(q[:0], pages, dev(table)[:0], i32([]), i32([0]), none).shape == (0, 4, 64)


@pytest.mark.parametrize("rows", [1, 20])
def test_shared_in_a_graph(listed, rows):
    """Replays after lengths, groups and shared pages changed, with eager calls in the same workspace between them."""
    pages, table, lens, held, groups, shared = family(listed, [(6, [260, 300, 200, 333])], 2, 64, 64, 32, "bf16")
    q = draw((4 * rows, 8, 64), 9, "bf16").cuda()
    t, n, g, p = dev(table), i32(lens), i32(groups), i32(shared)
    ws = listed.workspace(listed.kv_attn_shared_workspace_size(4 * rows, 4, rows, 8, 2, 64, 1), "cuda")
    call = lambda: listed.kv_attn_shared(q, pages, t, n, g, p, max_q=rows, ws=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for step in range(5):
        graph.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, call())
        check(got, None, q, [(k[:x], v[:x]) for (k, v), x in zip(held, host(n))], [rows] * 4, 64 ** -0.5, "bf16")
        n -= 13
        p.fill_(max(0, 6 - 2 * step))
        g.copy_(i32([step % 2, 4 - step % 3]))


def test_shared_on_two_streams(listed):
    """Two calls at once, each with its own workspace."""
    pages, table, lens, held, groups, shared = family(listed, [(6, [260, 300, 200])], 2, 64, 64, 32, "bf16")
    qs = [draw((3, 8, 64), y, "bf16").cuda() for y in (1, 2)]
    t, n, g, p = dev(table), i32(lens), i32(groups), i32(shared)
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    outs = [listed.kv_attn_shared(q, pages, t, n, g, p, stream=s) for _ in range(3) for q, s in zip(qs, streams)]
    torch.cuda.synchronize()
    for y, out in enumerate(outs):
        check(out, None, qs[y % 2], held, [1, 1, 1], 64 ** -0.5, "bf16")


def test_shared_is_the_same_each_time(listed):
    pages, table, lens, held, groups, shared = family(listed, [(20, [700, 900, 650])], 2, 128, 64, 32, "bf16")
    q = draw((3, 8, 128), 1, "bf16").cuda()
    args = (q, pages, dev(table), i32(lens), i32(groups), i32(shared))
    first = listed.kv_attn_shared(*args)
    for _ in range(3):
        assert torch.equal(listed.kv_attn_shared(*args), first)


def test_shared_where_it_gains(qe):
    """Through the public call, at a size that takes the lists by its own rule, and one that does not."""
    attend(qe, [(128, [8200 + 37 * y for y in range(24)])], [1] * 24, 8, 2, 64, 64, 64, "bf16", seed=1)
    attend(qe, [(1, [70, 90])], [1, 1], 8, 2, 64, 64, 64, "bf16", seed=2)


@pytest.mark.parametrize("dtype", list(DT))
def test_shared_what_a_row_does_not_see(listed, dtype):
    """NaN and huge values in one sequence's own part touch that sequence alone; NaN in the shared part every row of the
    key head that sees it, in every sequence."""
    pages, table, lens, held, groups, shared = family(listed, [(3, [140, 120, 97, 99])], 2, 64, 64, 32, dtype, seed=8)
    q = draw((4, 4, 64), 1, dtype).cuda()
    args = (q, pages, dev(table), i32(lens), i32(groups), i32(shared))

    def put(b, t, value):
        x = torch.full((1, 2, 64), value, dtype=DT[dtype], device="cuda")
        x[:, 0] = 0.5                                       # (the second key head alone)
        listed.kv_write(x, x, dev(np.array([int(table[b, t // 32]) * 32 + t % 32])), pages)

    def seen():
        out = []
        for b, n in enumerate(lens):
            t = np.arange(n)
            out.append(tuple(f64(x) for x in listed.kv_read(pages, dev(table[b][t // 32].astype(np.int64) * 32 + t % 32), 64)))
        return out

    put(0, 110, float("nan"))
    put(1, 119, 3.0e4 if dtype == "f16" else 1.0e30)
    out = listed.kv_attn_shared(*args, check=True)
    now = seen()
    assert bool(torch.isnan(out[0, 2:]).all()) and bool(torch.isfinite(out[0, :2]).all())
    for b in (2, 3):
        check(out[b:b + 1], None, q[b:b + 1], [now[b]], [1], 0.125, dtype)
    check(out[1:2, :2], None, q[1:2, :2], [tuple(x[:, :1] for x in now[1])], [1], 0.125, dtype)
    put(2, 50, float("nan"))                                # (one page for all)
    out = listed.kv_attn_shared(*args, check=True)
    assert bool(torch.isnan(out[:, 2:]).all()) and bool(torch.isfinite(out[:, :2]).all())
    # a sequence that ends before it does not see it, and keeps the others from sharing it
    out = listed.kv_attn_shared(q, pages, dev(table), i32([140, 120, 97, 50]), i32(groups), i32(shared), check=True)
    assert bool(torch.isnan(out[:3, 2:]).all()) and bool(torch.isfinite(out[3]).all())
