"""Attention over the 4-bit cache with first tokens that stay visible beside a window, against fp64 arithmetic on the values
held; the bound is derived in test_gpu_kv.py's head."""
import numpy as np
import pytest
import torch

from parity import dev, host
from test_gpu_kv import DT, attend, cache, check, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dim", [8, 64, 80, 128, 192, 256])
def test_sinks_widths(qe, dim, group):
    for dtype in DT:
        print(f"[sinks] dim={dim} group={group} {dtype}", flush=True)
        attend(qe, [270, 133], [1, 1], 6, 2, dim, group, 64, dtype, seed=dim, window=50, sinks=5)
        attend(qe, [245, 100], [9, 3], 6, 3, dim, group, 32, dtype, seed=dim + 1, window=33, sinks=40)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("sinks", [1, 4, 31, 32, 33, 64, 100, 256, 257, 2 ** 31 - 1])
def test_sinks_and_windows(qe, sinks, dtype):
    """Sinks before the window, up to it, inside it, beyond it and past the sequence; the records between both are
    full of other sequences' bytes and not read."""
    for window in (1, 32, 37, 200):
        attend(qe, [257, 90], [1, 1], 6, 2, 64, 64, 64, dtype, seed=window, window=window, sinks=sinks)
    attend(qe, [257, 300], [70, 41], 6, 2, 96, 32, 32, dtype, seed=3, window=60, sinks=sinks, slopes=True)


@pytest.mark.parametrize("n", [0, 1, 2, 31, 32, 33, 64, 65, 1000])
def test_sinks_lengths(qe, n):
    attend(qe, [n, 3], [1, 1], 8, 2, 128, 64, 64, "bf16", seed=n, window=20, sinks=3)
    attend(qe, [n, 1500], [1, 1], 4, 4, 64, 64, 96, "f32", seed=n, window=700, sinks=3)


def test_sinks_of_rows_that_see_nothing(qe):
    for dtype in DT:
        attend(qe, [3, 0, 20, 9], [7, 4, 0, 9], 4, 2, 64, 32, 32, dtype, seed=1, window=1, sinks=2)


@pytest.mark.parametrize("dtype", list(DT))
def test_sinks_with_splits(qe, dtype):
    """Windows long enough for splits, one that ends inside the first tokens' records, a gap inside a split, many key heads."""
    attend(qe, [9000], [1], 8, 2, 64, 64, 64, dtype, seed=1, window=3001, sinks=1000)
    attend(qe, [9000, 2500], [2, 1], 4, 2, 128, 128, 32, dtype, seed=2, window=1200, sinks=70, slopes=True)


@pytest.mark.parametrize("dtype", list(DT))
def test_sinks_of_chunks(qe, dtype):
    """Chunks that take the many-row form, whose tiles see different first window records."""
    attend(qe, [700, 650], [300, 200], 64, 64, 64, 64, 64, dtype, seed=1, window=100, sinks=33)
    attend(qe, [500], [256], 40, 40, 128, 128, 32, dtype, seed=2, window=64, sinks=3)


def test_sinks_of_a_window_that_hides_nothing(qe):
    """The same bits as without a window."""
    pages, table, _ = cache(qe, [300, 40], 2, 128, 64, 64, "bf16")
    q = draw((8, 8, 128), 1, "bf16").cuda()
    args = (q, pages, dev(table), dev(np.array([300, 40], np.int32)))
    plain = qe.kv_attn(*args, max_q=4)
    assert torch.equal(qe.kv_attn(*args, max_q=4, window=0, sinks=7), plain)
    assert torch.equal(qe.kv_attn_sinks(*args, 0, 7, max_q=4), plain)
    assert torch.equal(qe.kv_attn(*args, max_q=4, window=50, sinks=0), qe.kv_attn(*args, max_q=4, window=50))


def test_sinks_hide_bad_groups_and_pages(qe):
    """NaN groups between the first tokens and the window reach no row, nor do pages that are not there."""
    lens, window, sinks = [400, 390], 64, 10
    pages, table, held = cache(qe, lens, 2, 64, 64, 32, "bf16", seed=5)
    q = draw((2, 4, 64), 9, "bf16").cuda()
    bad = torch.full((1, 2, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    for b, n in enumerate(lens):
        for t in (sinks, sinks + 1, 31, n - window - 1):
            qe.kv_write(bad, bad, dev(np.array([int(table[b, t // 32]) * 32 + t % 32])), pages)
    table[:, 1:9] = -7                                     # (records 1 .. 8: tokens 32 .. 287)
    out = qe.kv_attn(q, pages, dev(table), dev(np.array(lens, np.int32)), window=window, sinks=sinks, check=True)
    check(out, None, q, held, [1, 1], 64 ** -0.5, "bf16", window=window, sinks=sinks)
    # one that a row does see makes the row NaN
    qe.kv_write(bad, bad, dev(np.array([int(table[0, 0]) * 32 + sinks - 1])), pages)
    out = qe.kv_attn(q, pages, dev(table), dev(np.array(lens, np.int32)), window=window, sinks=sinks, check=True)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isfinite(out[1]).all())


def test_sinks_report_an_absent_page(qe):
    pages, table, _ = cache(qe, [400], 2, 64, 64, 32, "bf16", seed=5)
    table[0, 0] = 10 ** 6
    q = draw((1, 4, 64), 9, "bf16").cuda()
    ws = qe.workspace(qe.kv_attn_workspace_size(1, 1, 1, 4, 2, 64), "cuda")
    out = qe.kv_attn(q, pages, dev(table), dev(np.array([400], np.int32)), window=64, sinks=40, ws=ws)
    assert qe.sync_status(ws) == qe.QE_ERR_ARG
    table[0, 0] = 0
    # tokens 0 .. 31 count as absent: what is left are 32 .. 39 and the window, as a call without sinks over them says
    assert bool(torch.isfinite(out).all())


def test_sinks_refusals(qe):
    pages, table, _ = cache(qe, [40], 2, 64, 64, 32, "bf16")
    args = (draw((1, 4, 64), 9, "bf16").cuda(), pages, dev(table), dev(np.array([40], np.int32)))
    for bad in (dict(window=5, sinks=-1), dict(window=5, sinks=-2 ** 40), dict(sinks=3, causal=False)):
        with pytest.raises(qe.QEError):
            qe.kv_attn(*args, **bad)
    assert torch.equal(qe.kv_attn(*args, window=5, sinks=2 ** 40), qe.kv_attn(*args))


@pytest.mark.parametrize("rows", [1, 150])
def test_sinks_in_a_graph(qe, rows):
    """Replays after the sequences grew, with other work in between."""
    lens = [600, 500]
    pages, table, held = cache(qe, [700, 700], 4, 64, 64, 32, "bf16")
    q = draw((2 * rows, 8, 64), 9, "bf16").cuda()
    t, n = dev(table), dev(np.array(lens, np.int32))
    ws = qe.workspace(qe.kv_attn_workspace_size(2 * rows, 2, rows, 8, 4, 64), "cuda")
    call = lambda: qe.kv_attn(q, pages, t, n, max_q=rows, window=90, sinks=40, ws=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for step in range(4):
        graph.replay()
        got = out.clone()
        assert torch.equal(got, call())
        check(got, None, q, [(k[:lens[b] + 9 * step], v[:lens[b] + 9 * step]) for b, (k, v) in enumerate(held)], [rows] * 2, 64 ** -0.5,
              "bf16", window=90, sinks=40)
        n += 9
        torch.cuda.synchronize()
