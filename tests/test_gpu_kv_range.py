"""Attention over the 4-bit cache where the sizes of values differ widely: a row's result depends, to its
own precision, on the tokens that it sees and the weight that it gives them, whatever else the call reads.

The bound for an output element is that of test_gpu_kv.py, but for its absolute part.  There a term
tokens 2^-34 max |v| over the whole cache stands for probabilities that meet their value scales in
fp16's subnormal range; here it is the row's and the channel group's own.  With p_t the row's
probabilities (after the division by their sum), s_t the group's value scales and Y = max over the
row's visible tokens of p_t s_t, a weight p_t s_t is held in fp16 with the largest at 2^10 or more, so
a step is off by 2^-25 2^-10 Y at most; a code is at most 15 steps from its zero point:
  far = tokens 15 2^-35 Y.
15 s_t is not returned by the library.  The codes of a group span at least 14 steps (each end is
rounded to a step, the two together to 15 +- 1), so 15 s_t <= 15/14 of the spread of the held
values and 0.  fp32's smallest steps add 1e-37 as there.
"""
import numpy as np
import pytest
import torch

from parity import dev
from test_gpu_kv import U_OUT, cache, draw, f64, many_rows

pytestmark = pytest.mark.gpu


def groups_of(v, group):
    """15 s_t at most, for each channel: (tokens, dim)."""
    reach = np.empty_like(v)
    for a in range(0, v.shape[-1], group):
        part = v[..., a:a + group]
        span = np.maximum(part.max(-1), 0.0) - np.minimum(part.min(-1), 0.0)
        reach[..., a:a + group] = 15.0 / 14.0 * span[..., None]
    return reach


def check_rows(out, q, held, nqs, scale, dtype, group, window=0):
    """Every row against fp64 with a bound made of what the row sees alone."""
    u_p = 2.0 ** -21 if dtype == "f32" else 2.0 ** -11
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-37
    first = 0
    for b, (k, v) in enumerate(held):
        n, kv = k.shape[0], max(1, k.shape[1])
        per = q.shape[1] // kv
        x = f64(q[first:first + nqs[b]])
        got = f64(out[first:first + nqs[b]])
        assert np.all(np.isfinite(got)), b
        t = np.arange(n)
        for h in range(q.shape[1]):
            kh, vh = k[:, h // per], v[:, h // per]
            reach = groups_of(vh, group) if n else vh
            for i in range(nqs[b]):
                pos = n - nqs[b] + i
                see = t <= pos
                if window:
                    see &= t > pos - window
                if not see.any():
                    assert not got[i, h].any()
                    continue
                s = scale * (kh[see] @ x[i, h])
                size = abs(scale) * np.abs(x[i, h]).sum() * 3.0 * np.abs(kh[see]).max()
                p = np.exp(s - s.max())
                p /= p.sum()
                ref, mass = p @ vh[see], p @ np.abs(vh[see])
                far = see.sum() * 2.0 ** -35 * (p[:, None] * reach[see]).max(0)
                bound = (u_p + 2.0 ** -19 * (1.0 + size)) * mass + far + U_OUT[dtype] * np.abs(ref) + tiny
                worst = (np.abs(got[i, h] - ref) / bound).max()
                assert worst <= 1.0, (b, h, i, worst)
        first += nqs[b]


def attend_with(qe, change, lens, nqs, heads, kv, dim, group, page, dtype, seed, spare=0, vscale=1.0, positive=False, **kw):
    """A cache whose first sequence gets change(k, v) written over it (fp32 tensors, tokens x kv x dim);
    positive: no query has a negative element."""
    pages, table, held = cache(qe, lens, kv, dim, group, page, dtype, seed, vscale=vscale)
    n = lens[0]
    t = np.arange(n)
    slots = dev(table[0][t // page].astype(np.int64) * page + t % page)
    k, v = (draw((n, kv, dim), seed + 1, dtype).float(), draw((n, kv, dim), seed + 2, dtype, vscale).float())
    change(k, v)
    qe.kv_write(k.cuda(), v.cuda(), slots, pages, group=group)
    held[0] = tuple(f64(x) for x in qe.kv_read(pages, slots, dim, group=group))
    assert all(np.all(np.isfinite(x)) for x in held[0])
    table = np.pad(table, ((0, 0), (0, spare)), constant_values=-1)
    q = draw((sum(nqs), heads, dim), seed + 7, dtype).cuda()
    q = q.abs() if positive else q
    start = dev(np.concatenate([[0], np.cumsum(nqs)]).astype(np.int32))
    out = qe.kv_attn(q, pages, dev(table), dev(np.array(lens, np.int32)), group=group, q_start=start, max_q=max(nqs),
                     check=True, **kw)
    check_rows(out, q, held, nqs, dim ** -0.5, dtype, group, **kw)


# Forms of a call: (sequences, queries, query heads, key heads, room in the table).
FORMS = {
    "few": ([150], [90], 2, 1, 0),
    "wide": ([150], [90], 2, 1, 32768),                 # rows in tiles of 32 where the width allows it
    "many": (*many_rows(16, [150], [140], 64, 64), 16, 16, 0),
}
WIDTHS = [(64, 64), (64, 32), (128, 128), (128, 64), (128, 32), (96, 64), (256, 64)]


def ratios(dtype):
    """Sizes of the large value against the others: 2^20 and 2^30, and the ends of the type's range (the
    values are 2^-10 for fp16, which holds up to 2^16)."""
    return (2.0 ** 20, 2.0 ** 25) if dtype == "f16" else (2.0 ** 20, 2.0 ** 30, 2.0 ** 100)


def base(dtype):
    return 2.0 ** -10 if dtype == "f16" else 1.0


def one_value(v, token, size):
    """The token's values scaled to a largest element of `size`."""
    v[token] *= size / v[token].abs().max()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dim,group", WIDTHS)
def test_a_later_token_leaves_earlier_rows_alone(qe, form, dim, group, dtype):
    """A large value that only the last rows of a tile see."""
    lens, nqs, heads, kv, spare = FORMS[form]
    for size in ratios(dtype):
        print(f"[kv] later {form} {dim} {group} {dtype} {size:g}", flush=True)
        attend_with(qe, lambda k, v: one_value(v, 125, size * base(dtype)), lens, nqs, heads, kv, dim, group, 32, dtype,
                    11, spare, base(dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dim,group", [(64, 64), (128, 64), (128, 32)])
def test_a_token_before_the_window_leaves_later_rows_alone(qe, form, dim, group, dtype):
    """A large value that leaves the window inside of a tile of rows."""
    lens, nqs, heads, kv, spare = FORMS[form]
    size = ratios(dtype)[-1]
    attend_with(qe, lambda k, v: one_value(v, 70, size * base(dtype)), lens, nqs, heads, kv, dim, group, 32, dtype, 12,
                spare, base(dtype), window=17)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dim,group", WIDTHS)
def test_a_token_of_little_weight(qe, form, dim, group, dtype):
    """Large values that the rows see and give nearly no weight, first and last of what they see: keys of
    one sign against queries of the other."""
    lens, nqs, heads, kv, spare = FORMS[form]

    def change(k, v):
        for token in (3, 59):
            one_value(v, token, ratios(dtype)[1] * base(dtype))
            k[token] = -k[token].abs() * 8.0
    attend_with(qe, change, lens, nqs, heads, kv, dim, group, 32, dtype, 13, spare, base(dtype), positive=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dim,group", [(64, 32), (128, 64), (128, 32), (256, 128), (192, 64)])
def test_a_channel_group_leaves_the_others_alone(qe, form, dim, group, dtype):
    """One group of channels large in every token; and which one it is changes along the sequence."""
    lens, nqs, heads, kv, spare = FORMS[form]
    size = ratios(dtype)[-1]

    def first(k, v):
        v[:, :, :group] *= size / 8

    def turns(k, v):
        v[:60, :, :group] *= size / 8
        v[60:, :, group:2 * group] *= size / 8
    for change in (first, turns):
        attend_with(qe, change, lens, nqs, heads, kv, dim, group, 32, dtype, 16, spare, base(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("vscale", [2.0 ** -100, 2.0 ** 119])
def test_values_near_the_ends_of_the_range(qe, form, dtype, vscale):
    """Values near fp32's smallest and largest numbers: no weight vanishes, and sums over tokens that
    pass the largest number have a result that does not."""
    lens, nqs, heads, kv, spare = FORMS[form]

    def change(k, v):
        v.copy_(v.abs().clamp(max=60.0 * vscale))
    attend_with(qe, change, lens, nqs, heads, kv, 64, 32, 32, dtype, 17, spare, vscale)
    attend_with(qe, change, [150], [1], 4, 2, 128, 64, 32, dtype, 18, 0, vscale)
    attend_with(qe, change, [3000], [1], 4, 2, 128, 64, 32, dtype, 19, 0, vscale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_values_before_large_ones(qe, dtype):
    """Tokens of nearly all the weight and tiny values, then, in the same wave, large values of little
    weight: the first ones' weight stays in the sum of the probabilities."""
    def change(k, v):
        v[:200] *= 2.0 ** -70
        k[200:] = -k[200:].abs() * 4.0
        v[200:] *= 2.0 ** 90
    for lens, nqs, heads, kv in (([400], [1], 4, 2), ([3000], [2], 4, 2), (*many_rows(16, [400], [150], 64, 64), 16, 16)):
        attend_with(qe, change, lens, nqs, heads, kv, 64, 64, 32, dtype, 21, positive=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_split_rows_and_a_large_value(qe, dtype):
    """Work split over the tokens: a large value in one split, zeros for values in others."""
    def change(k, v):
        one_value(v, 2500, 2.0 ** 40)
        v[:700] = 0.0
    for group in (32, 64, 128):
        attend_with(qe, change, [2900], [5], 4, 2, 128, group, 64, dtype, 22)
        attend_with(qe, change, [2900, 10], [5, 3], 4, 2, 64, group, 64, dtype, 23, window=2600)
