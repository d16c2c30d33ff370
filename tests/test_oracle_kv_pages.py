"""Who holds a page after calls that refuse some of the sequences, in the plain form of a step's pages (oracle/kv.py)."""
import numpy as np
import pytest

from oracle import kv as okv


def i32(x):
    return np.asarray(x, np.int32)


def owned(table, lengths, free, free_count, page, keep=None):
    """Every page belongs to one row, at a place that its tokens reach, or lies on the stack once; every other entry is -1."""
    pages = list(free[:free_count])
    for b, row in enumerate(table):
        held = max(-(-int(lengths[b]) // page), 0 if keep is None else int(keep[b]))
        pages += list(row[:held])
        assert np.all(row[held:] == -1), b
    assert sorted(pages) == list(range(free.size))


def rows_past_total(batch, seed, page=32, width=9, most=70):
    """Sequences, counts of either sign and a total that cuts off the rows of some: (lengths, counts, total)."""
    r = np.random.default_rng(seed)
    lengths = i32(r.integers(0, page * width - most, batch))
    counts = i32([r.choice([0, 1, r.integers(0, most + 1), -r.integers(0, n + 1)]) for n in lengths])
    return lengths, counts, int(r.integers(0, max(1, np.maximum(counts, 0).sum())))


def pool(lengths, page, width, spare, seed=0):
    held = -(-lengths // page)
    order = i32(np.random.default_rng(seed).permutation(held.sum() + spare))
    table, at = np.full((lengths.size, width), -1, np.int32), 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    free = np.full(order.size, -1, np.int32)
    free[:spare] = order[at:]
    return table, free


def test_rows_past_total_by_hand():
    """Sequence 1's rows pass the total: it stays as it is.  Sequence 2 has no rows, so that it gives its page back and is shorter."""
    lengths = i32([0, 40, 64])
    table = i32([[-1, -1], [0, 1], [2, 3]])
    free = i32([5, 4, -1, -1, -1, -1])
    _, _, start, left, _, bad = okv.extend([5, 10, -40], table, lengths, free, 2, 32, 14)
    assert bad and start.tolist() == [0, 5, 14, 14]
    assert lengths.tolist() == [5, 40, 24] and table.tolist() == [[3, -1], [0, 1], [2, -1]]
    assert left == 2 and free[:2].tolist() == [5, 4]
    owned(table, lengths, free, left, 32)


@pytest.mark.parametrize("batch", [2, 7, 40])
def test_rows_past_total(batch):
    for seed in range(40):
        lengths, counts, total = rows_past_total(batch, seed)
        table, free = pool(lengths, 32, 9, 30, seed)
        before = lengths.copy()
        left = okv.extend(counts, table, lengths, free, 30, 32, total)[3]
        owned(table, lengths, free, left, 32)
        assert np.all(lengths[counts <= 0] == np.maximum(before + counts, 0)[counts <= 0])


def test_taken_back_after_a_refusal():
    """10 tokens, 40 more refused.  By the lengths nothing is taken back; the opposite count would take the 10."""
    lengths, table, free = i32([10, 3]), i32([[1, -1], [0, -1]]), i32([-1, -1])
    before = lengths.copy()
    slots, _, _, left, lacking, bad = okv.extend([40, 2], table, lengths, free, 0, 32, 42)
    assert not bad and lacking == 1 and lengths.tolist() == [10, 5] and np.all(slots[:40] == -1)
    back = before - lengths
    assert back.tolist() == [0, -2]
    left = okv.extend(back, table, lengths, free, left, 32, 0)[3]
    assert lengths.tolist() == [10, 3] and table.tolist() == [[1, -1], [0, -1]] and left == 0
    left = okv.extend([-40, 0], table, lengths, free, left, 32, 0)[3]
    assert lengths.tolist() == [0, 3] and table[0].tolist() == [-1, -1] and free[:left].tolist() == [1]


@pytest.mark.parametrize("batch", [3, 40])
def test_steps_that_refuse_taken_back(batch):
    """Any mixture of new tokens, tokens that go back, pages that run out and rows past the total."""
    for seed in range(40):
        lengths, counts, total = rows_past_total(batch, seed)
        if seed % 2:
            total = int(np.maximum(counts, 0).sum())
        spare = seed % 7
        table, free = pool(lengths, 32, 9, spare, seed)
        first = [x.copy() for x in (table, lengths, free[:spare])]
        left = okv.extend(counts, table, lengths, free, spare, 32, total)[3]
        owned(table, lengths, free, left, 32)
        back = first[1] - lengths
        left = okv.extend(back, table, lengths, free, left, 32, int(np.maximum(back, 0).sum()))[3]
        assert left == spare
        for a, b in zip(first, (table, lengths, free[:spare])):
            assert np.array_equal(a, b)
