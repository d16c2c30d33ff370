"""The plain forms of a serving step (oracle/kv.py) on cases worked out by hand."""
import numpy as np

from oracle import kv as okv


def i32(x):
    return np.asarray(x, np.int32)


def test_extend_by_hand():
    """Page 32.  Sequence 0: 30 -> 70 tokens, wants pages 1 and 2; 1: 64 -> 10, gives its second page back; 2: 0 -> 1."""
    table = i32([[7, -1, -1], [3, 5, -1], [-1, -1, -1]])
    lengths = i32([30, 64, 0])
    free = i32([1, 2, 9, -1, -1, -1, -1, -1, -1, -1])
    slots, positions, start, left, lacking, bad = okv.extend([40, -54, 1], table, lengths, free, 3, 32, 43)
    # the stack is 1 2 9 5 after the page came back; 5, 9 and 2 are taken in this order
    assert table.tolist() == [[7, 5, 9], [3, -1, -1], [2, -1, -1]]
    assert lengths.tolist() == [70, 10, 1] and left == 1 and lacking == 0 and not bad
    assert start.tolist() == [0, 40, 40, 41]
    assert positions[:3].tolist() == [30, 31, 32] and slots[:3].tolist() == [7 * 32 + 30, 7 * 32 + 31, 5 * 32]
    assert slots[39] == 9 * 32 + 5 and (positions[40], slots[40]) == (0, 64) and positions[41:].tolist() == [-1, -1]
    # undone: table, lengths and stack as they were
    okv.extend([-40, 54, -1], table, lengths, free, left, 32, 54)
    assert table.tolist() == [[7, -1, -1], [3, 5, -1], [-1, -1, -1]] and lengths.tolist() == [30, 64, 0]
    assert free[:3].tolist() == [1, 2, 9]


def test_extend_refuses_by_hand():
    """One free page: the first that wants two gets none, the second, which wants one more than is left of them, none either;
    who wants none is served."""
    table, lengths, free = i32([[-1, -1], [-1, -1], [4, -1]]), i32([0, 0, 3]), i32([0, 0, 0, 0, 0])
    slots, positions, start, left, lacking, bad = okv.extend([40, 1, 2], table, lengths, free, 1, 32, 43)
    assert lengths.tolist() == [0, 0, 5] and left == 1 and lacking == 2 and not bad
    assert np.all(slots[:41] == -1) and slots[41:].tolist() == [131, 132] and positions[40] == 0


def test_extend_keeps_by_hand():
    table, lengths, free = i32([[4, 2]]), i32([40]), i32([0, 0, 0, 0, 0])
    okv.extend([-40], table, lengths, free, 0, 32, 0, keep=[1])
    assert table.tolist() == [[4, -1]] and free[0] == 2 and lengths[0] == 0


def test_norm_and_rotation_by_hand():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    w = np.array([1, 2, 3, 4], np.float32)
    # mean square 25 / 4: root 2.5
    y = okv.norm_rotate(x, w, 0.0, None, None, None, False)
    assert np.allclose(y, [[[1.2, 3.2, 0.0, 0.0]]], rtol=1e-6)
    cos, sin = np.array([[1.0, 1.0], [0.0, 0.0]], np.float32), np.array([[0.0, 0.0], [1.0, 1.0]], np.float32)
    a = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    # a quarter turn: (a, b) -> (-b, a)
    assert okv.norm_rotate(a, None, 0.0, np.array([1]), cos, sin, False).tolist() == [[[-3.0, -4.0, 1.0, 2.0, 5.0]]]
    assert okv.norm_rotate(a, None, 0.0, np.array([1]), cos, sin, True).tolist() == [[[-2.0, 1.0, -4.0, 3.0, 5.0]]]
    assert okv.norm_rotate(a, None, 0.0, np.array([0]), cos, sin, True).tolist() == a.tolist()


def test_first_tokens_by_hand():
    """Equal scores: the mean of the visible values.  At position 6 a window of 2 and 3 first tokens see 0, 1, 2, 5, 6."""
    v = np.arange(8, dtype=float).reshape(8, 1, 1)
    out, lse, _ = okv.attention(np.zeros((1, 1, 1)), np.zeros((8, 1, 1)), v, [6], 1.0, window=2, sinks=3)
    assert np.isclose(out[0, 0, 0], 14 / 5) and np.isclose(lse[0, 0], np.log(5))
