"""Attention over the 4-bit cache where few splits along the tokens are joined by one workgroup a unit, and
what its contract says of rows and pages that are not there."""
import numpy as np
import pytest
import torch

from parity import dev
from test_gpu_kv import SPARE, attend, cache, check, draw

pytestmark = pytest.mark.gpu

DTYPES = ["f32", "f16", "bf16"]
DIMS = [(64, 64), (40, 32), (96, 32), (128, 64), (128, 128), (192, 64), (256, 128)]


def splits(lens, nqs, heads, kv, page, rows_of_a_unit, spare=0, window=0):
    """Splits of the call by the planner's rule (768 workgroups, 1536 for 385 to 767 units of 256 records and more; at least
    4 records each, none below 20 records).  2 to 8 are joined by units."""
    tiles = -(-max(nqs) * (heads // kv) // rows_of_a_unit)
    records = (max(max(-(-n // page) for n in lens), 1) + 1 + spare) * (page // 32)
    if window:
        records = min(records, (window + max(nqs)) // 32 + 2)
    units = len(lens) * kv * tiles
    return min((1536 if 384 < units < 768 and records >= 256 else 768) // units, records // 4) if records >= 20 else 1


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,group", DIMS)
def test_join_of_units_widths(qe, dim, group, dtype):
    """Sequences of 7 splits and of one, tiles of 16 rows that end inside; 29 to 33 records."""
    for lens, nqs, heads in (([900, 300, 40, 0], [1, 1, 1, 1], 4), ([900, 641, 700], [9, 3, 1], 8), ([930], [17], 2)):
        assert 2 <= splits(lens, nqs, heads, 2, 32, 16) <= 8
        attend(qe, lens, nqs, heads, 2, dim, group, 32, dtype, seed=dim + group)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_join_of_units_wide_tiles(qe, group, dtype):
    """Units of 20 rows in a tile of 32 (16-bit calls up to 128 channels; two of 16 otherwise); of 6 splits, 5, 1 and none."""
    for dim in (64, 96, 128):
        for n in (32, 16):
            assert 2 <= splits([900, 200, 700, 0], [1] * 4, 640, 32, 64, n, SPARE) <= 8
        attend(qe, [900, 200, 700, 0], [1] * 4, 640, 32, dim, group, 64, dtype, seed=dim + group, spare=SPARE)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim,group", [(64, 32), (128, 64), (256, 64)])
def test_join_of_units_many_sequences(qe, dim, group, dtype):
    """Every number of splits in use from 1 to 7; units that are more than half of the chip's, in three over long tables."""
    lens = [1000, 100, 639, 640, 800, 790, 5, 0, 960, 700]
    assert splits(lens, [1] * 10, 20, 10, 32, 16) == 7
    attend(qe, lens, [1] * 10, 20, 10, dim, group, 32, dtype, seed=dim)
    assert splits(lens, [2] * 10, 80, 40, 32, 16, 300) == 3
    attend(qe, lens, [2] * 10, 80, 40, dim, group, 32, dtype, seed=dim + 1, spare=300)


@pytest.mark.parametrize("dtype", DTYPES)
def test_join_of_units_masks(qe, dtype):
    for window in (700, 5000):
        assert 2 <= splits([1000, 900], [9, 20], 4, 2, 32, 16, window=window) <= 8
        attend(qe, [1000, 900], [9, 20], 4, 2, 64, 32, 32, dtype, seed=window, window=window, slopes=True)
    attend(qe, [1000, 300], [9, 20], 4, 2, 128, 64, 32, dtype, seed=3, causal=False)
    attend(qe, [900, 4, 0], [7, 9, 3], 20, 20, 80, 32, 32, dtype, seed=4, slopes=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kscale,vscale", [(30.0, 1e-6), (1e-3, 1e-3), (1e-6, 1e4)])
def test_join_of_units_magnitudes(qe, dtype, kscale, vscale):
    if dtype == "f16" and vscale == 1e4:
        pytest.skip("fp16 holds no such values")
    attend(qe, [900, 700], [3, 1], 8, 2, 64, 64, 32, dtype, seed=1, kscale=kscale, vscale=vscale)


def test_join_of_units_nan_groups(qe):
    """A NaN group in one split reaches the rows and channels that see it, through the join."""
    n, dim = 900, 64
    pages, table, held = cache(qe, [n], 2, dim, 32, 32, "f32", 5)
    slot = dev(np.array([table[0][500 // 32] * 32 + 500 % 32], np.int64))
    v = torch.ones((1, 2, dim), device="cuda")
    v[0, :, 40] = float("nan")
    qe.kv_write(torch.ones((1, 2, dim), device="cuda"), v, slot, pages, group=32)
    q = draw((1, 2, dim), 3).cuda()
    for at, sees in ((499, False), (500, True), (899, True)):
        out = qe.kv_attn(q, pages, dev(table), dev(np.array([at + 1], np.int32)), group=32)
        assert bool(torch.isfinite(out[:, :, :32]).all())
        assert bool(torch.isnan(out[:, :, 32:]).all()) == sees and bool(torch.isfinite(out[:, :, 32:]).all()) != sees


@pytest.mark.parametrize("heads", [2, 200])
def test_missing_pages_beside_a_first_page_of_infinities(qe, heads):
    """A page number outside of the cache counts as absent, whatever the cache's first page holds: words that are
    infinite scales there.  Both forms."""
    n, dim, page = 140, 64, 32
    pages, table, held = cache(qe, [n], heads, dim, 64, page, "f32", 7)
    num = pages.shape[0]
    keep = int(np.setdiff1d(np.arange(num), table[0])[0])      # a page that no sequence has
    # page 0 becomes the one of infinities; what it held moves to the spare page
    pages[keep].copy_(pages[0])
    table[0][table[0] == 0] = keep
    words = pages[0].view(torch.int32)
    words.fill_(0x7f800000)
    bad = table.copy()
    bad[0, 1] = -1
    q = draw((n, heads, dim), 3).cuda()
    ws = qe.workspace(qe.kv_attn_workspace_size(n, 1, n, heads, heads, dim), "cuda")
    out = qe.kv_attn(q, pages, dev(bad), dev(np.array([n], np.int32)), ws=ws)
    assert qe.sync_status(ws) == qe.QE_ERR_ARG
    k, v = held[0]
    absent = np.r_[0:32, 64:n]
    check(out[64:], None, q[64:], [(k[absent], v[absent])], [n - 64], dim ** -0.5, "f32")
    check(out[:32], None, q[:32], [(k[:32], v[:32])], [32], dim ** -0.5, "f32")


@pytest.mark.parametrize("many", [False, True])
def test_rows_of_no_sequence_are_not_written(qe, many):
    """Rows of Q before q_start[0], after its last entry and between sequences' ranges (a range past max_q is cut,
    and reported) keep what out held."""
    heads, dim = (200, 64) if many else (4, 64)
    lens = [140, 20]
    pages, table, held = cache(qe, lens, heads, dim, 64, 32, "bf16", 3)
    nq = 140 if many else 5
    q = draw((nq + 30, heads, dim), 5, "bf16").cuda()
    out = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 3.0, device="cuda")
    start = dev(np.array([2, 2 + nq, 2 + nq + 4], np.int32))
    qe.kv_attn(q, pages, dev(table), dev(np.array(lens, np.int32)), q_start=start, max_q=nq, out=out, lse=lse, check=True)
    check(out[2:nq + 6], lse[2:nq + 6], q[2:nq + 6], held, [nq, 4], dim ** -0.5, "bf16")
    for t in (out, lse):
        assert bool((t[:2] == 3.0).all()) and bool((t[nq + 6:] == 3.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [60, 80])
def test_wide_heads_in_groups_of_32_on_both_sides_of_their_rule(qe, heads, dtype):
    """128 rows a key head of 256 channels: 120 workgroups of the many-row form (few rows, split) and 160 (many)."""
    attend(qe, [700], [128], heads, heads, 256, 32, 64, dtype, seed=heads)
