"""Who holds a page after kv_extend refused some of the sequences: the state itself is looked over, beside the comparison with
the plain form."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from parity import dev, host
from test_gpu_kv_step import Pool
from test_oracle_kv_pages import owned, rows_past_total

pytestmark = pytest.mark.gpu


def i32(x):
    return np.asarray(x, np.int32)


def look(p):
    owned(host(p.dtable), host(p.dlengths), host(p.dfree), int(p.dcount), p.page, p.keep)


@pytest.mark.parametrize("pad", [0, 3000])
def test_extend_rows_past_total_by_hand(qe, pad):
    """A sequence behind one whose rows pass the total gives its page back and is shorter; undone, it has as many again."""
    p = Pool([0, 40 + pad, 64], 32, 120, spare=3)
    assert p.step(qe, [5, 10 + pad, -40], 14 + pad)[5]
    look(p)
    assert p.lengths.tolist() == [5, 40 + pad, 24]
    assert not p.step(qe, [-5, 0, 40], 40)[5]
    look(p)
    assert p.lengths.tolist() == [0, 40 + pad, 64]


@pytest.mark.parametrize("batch", [2, 40, 1025, 2500])
def test_extend_rows_past_total(qe, batch):
    """Counts of either sign and totals that cut off the rows of some, sequences a thread each and several."""
    for seed in range(4):
        lengths, counts, total = rows_past_total(batch, seed)
        p = Pool(lengths.tolist(), 32, 9, spare=3 * batch, seed=seed)
        p.step(qe, counts, total)
        look(p)
        assert np.all(p.lengths[counts <= 0] == np.maximum(lengths + counts, 0)[counts <= 0])


@pytest.mark.parametrize("spare", [0, 1, 4, 9, 40])
@pytest.mark.parametrize("batch", [5, 1100])
def test_extend_taken_back_after_a_refusal(qe, batch, spare):
    """A recorded step of drafted tokens and its undoing, by what the lengths say was given: replays in which the pages run out for some
    sequences, and for all, restore everything."""
    r = np.random.default_rng(spare)
    p = Pool(r.integers(0, 150, batch).tolist(), 32, 12, spare, seed=batch)
    counts = dev(np.zeros(batch, np.int32))
    total = batch * 90

    def draft():
        before = p.dlengths.clone()
        slots, _, start = qe.kv_extend(counts, p.dtable, p.dlengths, p.dfree, p.dcount, 32, total)
        drafted = p.dlengths.clone()
        qe.kv_extend(before - p.dlengths, p.dtable, p.dlengths, p.dfree, p.dcount, 32, 0)
        return slots, start, drafted

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        draft()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slots, start, drafted = draft()
    refused = 0
    for n in range(5):
        new = i32(r.integers(0, 90, batch))
        counts.copy_(dev(new))
        graph.replay()
        torch.cuda.synchronize()
        table, lengths, free = p.table.copy(), p.lengths.copy(), p.free.copy()
        want = okv.extend(new, table, lengths, free, p.free_count, 32, total)
        assert np.array_equal(host(slots), want[0]) and np.array_equal(host(start), want[2]) and np.array_equal(host(drafted), lengths)
        refused += int((lengths != p.lengths + new).sum())
        assert np.array_equal(host(p.dtable), p.table) and np.array_equal(host(p.dlengths), p.lengths)
        assert int(p.dcount) == spare and np.array_equal(host(p.dfree)[:spare], p.free[:spare])
        owned(host(p.dtable), host(p.dlengths), host(p.dfree), spare, 32)
    assert refused > 0 if spare < 5 or batch > 5 else spare < 40 or refused == 0
