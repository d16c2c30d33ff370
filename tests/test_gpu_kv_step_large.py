"""A serving step where offsets pass 32 bits: slots past 2^32, a cache past 4 GiB, positions at the end of a window over
hundreds of thousands of tokens."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from parity import dev, host
from test_gpu_kv import bits, check, draw, f64
from test_gpu_kv_shared import listed  # noqa: F401
from test_gpu_kv_step import tables

pytestmark = pytest.mark.gpu


def i32(x):
    return dev(np.asarray(x, np.int32))


def test_extend_slots_past_32_bits(qe):
    num, page = 40_000_000, 128
    free = torch.arange(num, dtype=torch.int32, device="cuda")
    table, lengths, count = i32(np.full((3, 4), -1)), i32([0, 0, 0]), i32([num])
    slots, positions, start = qe.kv_extend(i32([130, 0, 1]), table, lengths, free, count, page, 131, check=True)
    want = np.concatenate([(num - 1) * page + np.arange(128), (num - 2) * page + np.arange(2), [(num - 3) * page]])
    assert want.min() > 2 ** 32 and np.array_equal(host(slots), want)
    assert host(positions).tolist() == list(range(130)) + [0] and host(start).tolist() == [0, 130, 130, 131] and int(count) == num - 3
    qe.kv_extend(i32([-130, 0, -1]), table, lengths, free, count, page, 0, check=True)
    assert int(count) == num and host(free[-3:]).tolist() == [num - 3, num - 2, num - 1] and bool((table == -1).all())


def test_a_cache_past_4_gib(listed):  # noqa: F811
    """The same tokens in a small cache and at the end of a large one: the same bits everywhere."""
    qe, kv, heads, dim, group, page = listed, 8, 16, 128, 128, 128
    num = (9 << 29) // qe.kv_page_bytes(kv, dim, group, page)                # 4.5 GiB
    big = qe.kv_pages(num, kv, dim, group, page)
    assert big.numel() > 2 ** 32
    small = qe.kv_pages(12, kv, dim, group, page)
    lens = [300, 290, 512]
    rows = np.array([[0, 1, 2, 9], [0, 1, 3, 10], [0, 1, 4, 5]], np.int32)
    cos, sin = (dev(x) for x in tables(600, dim))
    outs = []
    for pages, shift in ((small, 0), (big, num - 12)):
        table, got = rows + np.int32(shift), []
        for b, n in enumerate(lens):
            t = np.arange(0 if b == 0 else 256, n)
            slots = dev(table[b][t // page].astype(np.int64) * page + t % page)
            q, k, v = (draw((t.size, h, dim), 10 * b + h, "bf16").cuda() for h in (heads, kv, kv + 1))
            got.append(qe.kv_append(q, k, v[:, :kv], slots, pages, group=group, positions=i32(t), cos=cos, sin=sin))
            got.extend(qe.kv_read(pages, slots, dim, group=group))
        q = draw((3, heads, dim), 77, "bf16").cuda()
        args = (q, pages, dev(table), i32(lens))
        got.append(qe.kv_attn(*args, group=group, window=100, sinks=40, check=True))
        got.append(qe.kv_attn_shared(*args, i32([0, 3]), i32([2]), group=group, check=True))
        outs.append(got)
    for a, b in zip(*outs):
        assert np.array_equal(bits(a), bits(b))


def test_first_tokens_of_a_long_sequence(qe):
    """One sequence of 600000 tokens, most of whose pages are one page: the records between are not read, and its
    first tokens and window are found where they are."""
    n, page, window, sinks = 600_000, 128, 300, 70
    width = -(-n // page)
    pages = qe.kv_pages(8, 1, 64, 64, page)
    table = np.full((1, width), -1, np.int32)
    t = np.concatenate([np.arange(128), np.arange(n - 3 * page, n)])
    at = np.unique(t // page)
    table[0, at] = np.arange(at.size)
    slots = dev(table[0][t // page].astype(np.int64) * page + t % page)
    k, v = (draw((t.size, 1, 64), s, "bf16").cuda() for s in (1, 2))
    qe.kv_write(k, v, slots, pages)
    held = [f64(x) for x in qe.kv_read(pages, slots, 64)]
    q = draw((2, 4, 64), 3, "bf16").cuda()
    out = qe.kv_attn(q, pages, dev(table), i32([n]), max_q=2, window=window, sinks=sinks, check=True)
    for row, pos in enumerate((n - 2, n - 1)):
        see = (t <= pos) & ((t > pos - window) | (t < sinks))
        part = [x[see] for x in held]
        check(out[row:row + 1], None, q[row:row + 1], [part], [1], 0.125, "bf16")
