"""First tokens beside a window in the many-row form: chunks of enough rows and key heads that the call takes it (two workgroups
of 64 or 128 rows for a compute unit), every width, group and type, against fp64 arithmetic on the tokens that a row sees."""
import numpy as np
import pytest
import torch

from parity import dev
from test_gpu_kv import DT, cache, check, draw

pytestmark = pytest.mark.gpu

# two sequences, 32 key heads of 8 query heads each, 130 queries: 64 times 9 workgroups of 128 rows
SEQS, KV, PER, NQ = 2, 32, 8, 130


def chunk(qe, lens, dim, group, dtype, window, sinks, slopes=False, absent=None, step=29):
    heads = KV * PER
    pages, table, held = cache(qe, lens, KV, dim, group, 32, dtype, seed=dim + window)
    if absent is not None:
        table[:, absent] = 10 ** 6, -3
    q = draw((SEQS * NQ, heads, dim), 9, dtype).cuda()
    sl = (2.0 ** (-8.0 * np.arange(1, heads + 1) / heads)).astype(np.float32) if slopes else None
    lse = torch.full((SEQS * NQ, heads), 5.0, device="cuda")
    ws = qe.workspace(qe.kv_attn_workspace_size(SEQS * NQ, SEQS, NQ, heads, KV, dim), "cuda")
    out = qe.kv_attn(q, pages, dev(table), dev(np.asarray(lens, np.int32)), group=group, window=window, sinks=sinks, max_q=NQ, lse=lse,
                     slopes=None if sl is None else dev(sl), ws=ws)
    assert qe.sync_status(ws) == (qe.QE_OK if absent is None else qe.QE_ERR_ARG)
    for b, (k, v) in enumerate(held):
        t = np.arange(lens[b])
        for i in sorted({*range(0, NQ, step), NQ - 1}):
            pos, row = lens[b] - NQ + i, b * NQ + i
            see = (t <= pos) & ((t > pos - window) | (t < sinks))
            if absent is not None:
                see &= t // 32 != absent
            if not see.any():
                assert bool((out[row] == 0).all()) and bool(torch.isneginf(lse[row]).all())
                continue
            # (without slopes the tokens' places do not matter: the row stands behind those that it sees)
            if not slopes:
                check(out[row:row + 1], lse[row:row + 1], q[row:row + 1], [(k[see], v[see])], [1], dim ** -0.5, dtype)
            else:
                check(out[row:row + 1], lse[row:row + 1], q[row:row + 1], [(k[:pos + 1], v[:pos + 1])], [1], dim ** -0.5, dtype, slopes=sl,
                      window=window, sinks=sinks)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_sinks_many_rows_widths(qe, dim, group):
    for dtype in DT:
        print(f"[sinks] dim={dim} group={group} {dtype}", flush=True)
        chunk(qe, [500, 331], dim, group, dtype, 64, 40, step=43)


@pytest.mark.parametrize("window,sinks", [(1, 3), (37, 100), (200, 33), (64, 64), (100, 2 ** 31 - 1), (33, 290), (5, 1)])
@pytest.mark.parametrize("dtype", list(DT))
def test_sinks_many_rows_windows(qe, dtype, window, sinks):
    """Gaps inside a stage and beside it, none, sequences shorter than their queries, of which the first see nothing."""
    chunk(qe, [401, 97], 80, 64, dtype, window, sinks)
    chunk(qe, [1000, 300], 64, 64, dtype, window, sinks, slopes=True)


@pytest.mark.parametrize("dtype", list(DT))
def test_sinks_many_rows_without_a_page(qe, dtype):
    """The page of the first 32 tokens is absent; a page of the windows is."""
    chunk(qe, [500, 431], 64, 64, dtype, 64, 40, absent=0)
    chunk(qe, [500, 431], 128, 64, dtype, 64, 40, absent=13)
