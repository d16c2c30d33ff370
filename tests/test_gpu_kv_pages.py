"""Who holds a page after kv_extend refused some of the sequences: the state itself is looked over, beside the comparison with
the plain form."""
import numpy as np
import pytest
import torch

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
