"""The 4-bit key/value cache on the GPU against its plain CPU form (oracle/kv.py).

Writing is integer work decided by correctly rounded fp32 steps, reading one
correctly rounded product: both are compared bit for bit.

Attention is compared with fp64 arithmetic on the values that the cache holds.
The bound for an output element, with mass = sum_t p_t |v_t| and B = the largest
scale * sum_d |q_d k_td| + |bias| of the head's row (each from the oracle):
  (u_p + 2 u_s (1 + B)) mass + tokens 2^-34 max |v| + u_out |ref| + tiny
 - u_p, what a probability loses: 2^-11 (one fp16 rounding), fp32 calls 2^-21 (two fp16 parts);
   and absolutely half of fp16's smallest step, 2^-25, where the product of a probability and its
   value scale is scaled to at most 2^11 (15 codes of at most 2 max |v| / 15): it shows in a channel
   in which the token that has nearly all the weight is 0;
 - u_s, what a score loses relative to the sums that form it: 2^-20 (fp32 sums of up to
   256 products of codes up to 15, the query's split, the exponential's argument); codes are
   summed before the zero point is taken off, which B counts with the full code range;
 - u_out: 2^-8 bf16, 2^-11 fp16, 2^-23 fp32; tiny: 1e-37, fp16 half its smallest number, 2^-25.
"""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from parity import dev, host

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U_OUT = {"f32": 2.0 ** -23, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def draw(shape, seed, dtype="f32", scale=1.0, spread=True):
    r = np.random.default_rng(seed)
    x = r.standard_normal(shape)
    if spread:
        x = x * np.exp(0.5 * r.standard_normal(shape[1:])) + 0.3 * r.standard_normal(shape[1:])
    return torch.from_numpy((scale * x).astype(np.float32)).to(DT[dtype])


def f64(t):
    return t.detach().cpu().double().numpy()


def rounded(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DT[dtype])


def bits(t):
    t = t.detach().cpu().contiguous()
    return t.view(torch.int32 if t.dtype == torch.float32 else torch.int16).numpy()


# ------------------------------------------------------------------ write
WRITE = [(dim, group) for dim in (8, 40, 64, 80, 96, 120, 128, 160, 192, 200, 256) for group in (32, 64, 128)]


@pytest.mark.parametrize("dim,group", WRITE)
def test_write_bits(qe, dim, group):
    """Codes, scales and zero points of every supported width, whole and partial records."""
    dtype = list(DT)[(dim // 8 + group // 32) % 3]
    tokens, heads, page = 45, 2, 32 if group == 32 else 64
    k, v = draw((tokens, heads, dim), dim + group, dtype), draw((tokens, heads, dim), 2 * dim + 3 * group, dtype)
    pages = qe.kv_pages(4, heads, dim, group, page)
    pages.fill_(0xAB)
    want = host(pages)
    slots = np.arange(page - 5, page - 5 + tokens)         # a partial record, a whole one, a partial one
    okv.write(want, slots, f64(k), f64(v), group)
    qe.kv_write(k.cuda(), v.cuda(), dev(slots), pages, group=group)
    assert np.array_equal(host(pages), want)


@pytest.mark.parametrize("tokens", [0, 1, 31, 32, 33, 64, 97])
@pytest.mark.parametrize("dtype", list(DT))
def test_write_counts(qe, tokens, dtype):
    k, v = draw((tokens, 3, 64), tokens, dtype), draw((tokens, 3, 64), tokens + 1, dtype)
    pages = qe.kv_pages(2, 3, 64, 64, 64)
    pages.fill_(0x5C)
    want = host(pages)
    slots = np.arange(tokens) + 31
    okv.write(want, slots, f64(k), f64(v), 64)
    qe.kv_write(k.cuda(), v.cuda(), dev(slots), pages)
    assert np.array_equal(host(pages), want)


def test_write_scattered_skipped_and_past_the_end(qe):
    r = np.random.default_rng(4)
    slots = r.permutation(96 * 3)[:70]
    slots[[3, 40]] = -1, -(2 ** 40)
    slots[[7, 69]] = 96 * 3, 2 ** 60
    k, v = draw((70, 2, 96), 5, "bf16"), draw((70, 2, 96), 6, "bf16")
    pages = qe.kv_pages(3, 2, 96, 32, 96)
    want = host(pages)
    okv.write(want, slots, f64(k), f64(v), 32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    qe.kv_write(k.cuda(), v.cuda(), dev(slots), pages, group=32, status=status)
    assert np.array_equal(host(pages), want)
    assert int(status) == qe.QE_ERR_ARG
    status.zero_()
    qe.kv_write(k.cuda(), v.cuda(), dev(np.full(70, -1)), pages, group=32, status=status)
    assert np.array_equal(host(pages), want) and int(status) == 0


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shift", [0, 1])
def test_write_and_read_strided(qe, dtype, shift):
    """Slices of a fused projection, at a base that allows 16-byte loads and one that does not;
    outputs into slices, whose neighbours stay."""
    tokens, heads, dim = 40, 3, 72
    buf = draw((tokens, 2 * heads * dim + 50 + shift), 11, dtype, spread=False).cuda()
    k = buf[:, 24 + shift:24 + shift + heads * dim].unflatten(1, (heads, dim))
    v = buf[:, 24 + shift + heads * dim:24 + shift + 2 * heads * dim].unflatten(1, (heads, dim))
    pages = qe.kv_pages(2, heads, dim, 64, 32)
    want = host(pages)
    slots = np.arange(tokens)[::-1].copy() + 7
    okv.write(want, slots, f64(k), f64(v), 64)
    qe.kv_write(k, v, dev(slots), pages)
    assert np.array_equal(host(pages), want)
    out = torch.full((tokens, heads, 2 * dim + 8 + shift), 7.0, dtype=DT[dtype], device="cuda")
    K, V = out[:, :, shift:shift + dim], out[:, :, dim + shift:2 * dim + shift]
    qe.kv_read(pages, dev(slots), dim, K=K, V=V)
    kc, kw = okv.quantize(f64(k), 64)
    vc, vw = okv.quantize(f64(v), 64)
    assert np.array_equal(bits(K), bits(rounded(okv.values(kc, kw, dim, 64), dtype)))
    assert np.array_equal(bits(V), bits(rounded(okv.values(vc, vw, dim, 64), dtype)))
    assert bool((out[:, :, 2 * dim + shift:] == 7.0).all()) and bool((out[:, :, :shift] == 7.0).all())


def test_write_special_values(qe):
    """Zeros, one sign, one value, the ends of the fp32 range, subnormals, NaN and infinities:
    a bad group reads back as NaN, its neighbours do not."""
    dim, group = 64, 32
    x = draw((12, 1, dim), 3).numpy()
    x[0] = 0.0
    x[1] = np.abs(x[1])
    x[2] = -np.abs(x[2])
    x[3] = 3.25
    x[4, 0, 5] = np.nan
    x[5, 0, 40] = np.inf
    x[6, 0, 63] = -np.inf
    x[7, 0, :2] = 3e38, -3e38
    x[8] *= 1e-40
    x[9, 0, 0] = 3.4e38
    x[10] *= 1e36
    x[11] = -0.0
    pages = qe.kv_pages(1, 1, dim, group, 32)
    want = host(pages)
    okv.write(want, np.arange(12), x, -x, group)
    qe.kv_write(dev(x), dev(-x), dev(np.arange(12)), pages, group=group)
    assert np.array_equal(host(pages), want)
    k, v = (host(t)[:, 0] for t in qe.kv_read(pages, dev(np.arange(12)), dim, group=group))
    for row, g in ((4, 0), (5, 1), (6, 1), (7, 0)):
        for y in (k, v):
            assert np.isnan(y[row, 32 * g:32 * g + 32]).all()
            assert np.isfinite(y[row, 32 - 32 * g:64 - 32 * g]).all()
    assert not k[0].any() and not k[11].any()


# ------------------------------------------------------------------ read
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("dim,group", [(8, 32), (64, 32), (80, 32), (96, 64), (128, 128), (168, 64), (256, 128)])
def test_read_bits(qe, dtype, dim, group):
    """Every slot in and out of order, and slots that are not there."""
    tokens, heads, page = 77, 2, 96
    k, v = draw((tokens, heads, dim), dim).numpy(), draw((tokens, heads, dim), group).numpy()
    pages = np.random.default_rng(1).integers(0, 256, host(qe.kv_pages(2, heads, dim, group, page)).shape).astype(np.uint8)
    where = np.random.default_rng(2).permutation(2 * page)[:tokens]
    okv.write(pages, where, k, v, group)
    kc, kw = okv.quantize(k, group)
    vc, vw = okv.quantize(v, group)
    kx, vx = okv.values(kc, kw, dim, group), okv.values(vc, vw, dim, group)
    for order in (np.arange(tokens), np.argsort(where), np.arange(5)):
        K, V = qe.kv_read(dev(pages), dev(where[order]), dim, group=group, dtype=DT[dtype])
        assert np.array_equal(bits(K), bits(rounded(kx[order], dtype)))
        assert np.array_equal(bits(V), bits(rounded(vx[order], dtype)))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    K, V = qe.kv_read(dev(pages), dev(np.array([-1, where[0], 2 * page, 2 ** 50])), dim, group=group,
                      dtype=DT[dtype], status=status)
    assert int(status) == qe.QE_ERR_ARG
    for got, ref in ((K, kx), (V, vx)):
        assert np.array_equal(bits(got[1]), bits(rounded(ref[0], dtype)))
        assert not bool(got[0].any()) and not bool(got[2:].any())


def test_read_a_whole_record_in_order(qe):
    k, v = draw((96, 2, 128), 1).cuda(), draw((96, 2, 128), 2).cuda()
    pages = qe.kv_pages(2, 2, 128, 64, 64)
    qe.kv_write(k, v, torch.arange(96, device="cuda"), pages)
    for order in (torch.arange(96), torch.arange(96).flip(0), torch.arange(32, 64)):
        K, V = qe.kv_read(pages, order.cuda(), 128)
        for got, x in ((K, k), (V, v)):
            c, w = okv.quantize(host(x), 64)
            assert np.array_equal(host(got), okv.values(c, w, 128, 64)[order.numpy()])


# ------------------------------------------------------------------ attention
def cache(qe, lens, kv, dim, group, page, dtype="f32", seed=0, kscale=1.0, vscale=1.0, noise=True):
    """Sequences in shuffled pages of a pool that is full of random bytes elsewhere:
    (pages, table, [(k, v) in fp64])."""
    r = np.random.default_rng(seed)
    width = max(1, max(-(-n // page) for n in lens)) + 1
    num = width * len(lens) + 2
    pages = qe.kv_pages(num, kv, dim, group, page)
    if noise:
        pages.copy_(torch.randint(0, 256, pages.shape, dtype=torch.uint8, device="cuda",
                                  generator=torch.Generator(device="cuda").manual_seed(seed)))
    table = r.permutation(num)[:width * len(lens)].reshape(len(lens), width).astype(np.int32)
    held = []
    for b, n in enumerate(lens):
        t = np.arange(n)
        slots = dev(table[b][t // page].astype(np.int64) * page + t % page)
        k = draw((n, kv, dim), seed + 10 * b + 1, dtype, kscale).cuda()
        v = draw((n, kv, dim), seed + 10 * b + 2, dtype, vscale).cuda()
        qe.kv_write(k, v, slots, pages, group=group)
        held.append(tuple(f64(x) for x in qe.kv_read(pages, slots, dim, group=group)))
    return pages, table, held


def check(out, lse, q, held, nqs, scale, dtype, lens=None, **kw):
    first = 0
    for b, (k, v) in enumerate(held):
        nq = nqs[b]
        x = f64(q[first:first + nq])
        n = k.shape[0]
        pos = n - nq + np.arange(nq)
        ref, ref_lse, mass = okv.attention(x, k, v, pos, scale, **kw)
        got = f64(out[first:first + nq])
        per = q.shape[1] // max(1, k.shape[1])
        size = np.zeros((nq, q.shape[1], 1))
        for h in range(q.shape[1]):
            if n:
                # |k| with the full code range: 15 steps of a group are at most 2 max |k| + its range
                reach = 3.0 * np.abs(k[:, h // per]).max()
                size[:, h, 0] = abs(scale) * np.abs(x[:, h]).sum(-1) * reach
                if kw.get("slopes") is not None:
                    size[:, h, 0] += abs(float(kw["slopes"][h])) * n
        u_p = 2.0 ** -21 if dtype == "f32" else 2.0 ** -11
        far = n * 2.0 ** -34 * np.abs(v).max() if n else 0.0
        bound = (u_p + 2.0 ** -19 * (1.0 + size)) * mass + far + U_OUT[dtype] * np.abs(ref) + (2.0 ** -25 if dtype == "f16" else 1e-37)
        assert np.all(np.isfinite(got)), b
        worst = (np.abs(got - ref) / bound).max() if nq else 0.0
        assert worst <= 1.0, (b, worst)
        if lse is not None:
            l = f64(lse[first:first + nq])
            empty = np.isneginf(ref_lse)
            assert np.array_equal(np.isneginf(l), empty)
            # the sum's own rounding besides the scores'
            tol = 2.0 ** -20 * (1.0 + size[..., 0]) + 2.0 ** -20 * (1.0 + np.abs(np.where(empty, 0, ref_lse)))
            assert np.all(np.abs(np.where(empty, 0, l - ref_lse)) <= tol)
        first += nq


def attend(qe, lens, nqs, heads, kv, dim, group, page, dtype, seed=0, scale=None, kscale=1.0, vscale=1.0,
           qscale=1.0, slopes=False, give_lse=True, spare=0, **kw):
    pages, table, held = cache(qe, lens, kv, dim, group, page, dtype, seed, kscale, vscale)
    table = np.pad(table, ((0, 0), (0, spare)), constant_values=-1)     # pages for sequences that grow
    total = sum(nqs)
    q = draw((total, heads, dim), seed + 7, dtype, qscale).cuda()
    scale = 1.0 / dim ** 0.5 if scale is None else scale
    sl = (2.0 ** (-8.0 * np.arange(1, heads + 1) / heads)).astype(np.float32) if slopes else None
    lse = torch.full((total, heads), 5.0, device="cuda") if give_lse else None
    start = dev(np.concatenate([[0], np.cumsum(nqs)]).astype(np.int32))
    args = dict(group=group, scale=scale, q_start=start, max_q=max(nqs), lse=lse,
                slopes=dev(sl) if slopes else None, **kw)
    out = qe.kv_attn(q, pages, dev(table), dev(np.array(lens, np.int32)), check=True, **args)
    check(out, lse, q, held, nqs, scale, dtype, slopes=sl, **kw)
    return out


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 128, 152, 192, 256])
def test_attention_widths(qe, dim, group):
    """Every width and group; one new token and a few; odd lengths."""
    for dtype in DT:
        print(f"[kv] dim={dim} group={group} {dtype}", flush=True)
        attend(qe, [70, 33], [1, 1], 6, 2, dim, group, 64, dtype, seed=dim)
        attend(qe, [45, 100], [9, 3], 6, 3, dim, group, 32, dtype, seed=dim + 1)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (12, 4), (29, 1), (71, 1), (58, 2), (16, 1), (17, 1)])
def test_attention_head_layouts(qe, heads, kv, dtype):
    attend(qe, [130, 1, 64], [1, 1, 1], heads, kv, 64, 64, 64, dtype, seed=heads)
    attend(qe, [130, 40], [5, 17], heads, kv, 64, 32, 32, dtype, seed=heads + 1)


@pytest.mark.parametrize("n", [0, 1, 2, 31, 32, 33, 63, 64, 65, 255, 256, 257, 1000])
def test_attention_lengths(qe, n):
    attend(qe, [n, 3], [1, 1], 8, 2, 128, 64, 64, "bf16", seed=n)
    attend(qe, [n], [1], 4, 4, 128, 128, 32, "f32", seed=n)


def test_attention_rows_that_see_nothing(qe):
    """More queries than cached tokens, empty sequences, sequences without queries, a window of one."""
    for dtype in DT:
        attend(qe, [3, 0, 20, 9], [7, 4, 0, 9], 4, 2, 64, 32, 32, dtype, seed=1)
        attend(qe, [3, 0, 20, 9], [7, 4, 1, 9], 4, 2, 64, 32, 32, dtype, seed=2, window=1)
        attend(qe, [3, 0, 20, 9], [7, 4, 1, 9], 4, 2, 64, 32, 32, dtype, seed=3, causal=False)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("window", [1, 5, 32, 33, 100, 5000])
def test_attention_windows(qe, window, dtype):
    attend(qe, [257, 90], [1, 1], 6, 2, 64, 64, 64, dtype, seed=window, window=window)
    attend(qe, [257, 90], [70, 41], 6, 2, 96, 32, 32, dtype, seed=window, window=window, slopes=True)


@pytest.mark.parametrize("dtype", list(DT))
def test_attention_slopes_and_no_causal(qe, dtype):
    attend(qe, [300, 17], [1, 1], 20, 20, 80, 32, 32, dtype, seed=3, slopes=True)
    attend(qe, [300, 17], [33, 12], 20, 20, 80, 64, 32, dtype, seed=4, slopes=True)
    attend(qe, [300, 17], [33, 40], 8, 2, 128, 64, 64, dtype, seed=5, causal=False)


@pytest.mark.parametrize("dtype", list(DT))
def test_attention_chunks(qe, dtype):
    """Chunks larger than any tile, at group sizes that share and do not share tiles with tokens."""
    attend(qe, [333], [150], 2, 2, 128, 128, 64, dtype, seed=1)
    attend(qe, [290, 131], [131, 131], 4, 1, 64, 64, 32, dtype, seed=2)
    attend(qe, [200], [200], 3, 1, 128, 64, 64, dtype, seed=3)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("kscale,vscale,qscale", [(1e-6, 1e4, 1e5), (30.0, 1e-6, 1.0), (1e-3, 1e-3, 1e-3)])
def test_attention_magnitudes(qe, dtype, kscale, vscale, qscale):
    """Scores near 0 and near one-hot, values and queries far from 1."""
    if dtype == "f16" and qscale == 1e5:
        pytest.skip("fp16 holds no such queries")
    attend(qe, [140], [1], 8, 2, 64, 64, 64, dtype, seed=1, kscale=kscale, vscale=vscale, qscale=qscale)
    attend(qe, [140], [20], 4, 2, 128, 32, 64, dtype, seed=2, kscale=kscale, vscale=vscale, qscale=qscale)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("nq", [4, 96])
def test_attention_fp32_as_a_whole(qe, nq, group):
    """fp32 calls over many rows: the 2-norm of the error is within 2^-20 of the result's (fp16 parts
    that miss each other by a step in one weight of some thousand are 10 times that, and within the
    bound of a single element)."""
    n, heads, dim = 500, 8, 80
    pages, table, held = cache(qe, [n], heads, dim, group, 32, "f32", 5)
    q = draw((nq, heads, dim), 12, "f32", 0.5).cuda()
    out = qe.kv_attn(q, pages, dev(table), dev(np.array([n], np.int32)), group=group)
    ref, _, _ = okv.attention(f64(q), *held[0], n - nq + np.arange(nq), dim ** -0.5)
    assert np.linalg.norm(f64(out) - ref) <= 2.0 ** -20 * np.linalg.norm(ref)


def test_attention_zero_queries_and_values(qe):
    pages, table, held = cache(qe, [50], 2, 64, 64, 64)
    for dtype in DT:
        q = torch.zeros((1, 4, 64), dtype=DT[dtype], device="cuda")
        out = qe.kv_attn(q, pages, dev(table), dev(np.array([50], np.int32)))
        check(out, None, q, held, [1], 0.125, dtype)


@pytest.mark.parametrize("lens", [[5000], [4097, 9, 2500], [20000]])
def test_attention_long_and_split(qe, lens):
    """Few rows over long caches: work is split over the tokens and joined."""
    for dtype in DT:
        attend(qe, lens, [1] * len(lens), 8, 2, 64, 64, 64, dtype, seed=len(lens))
    attend(qe, lens, [3] * len(lens), 4, 2, 128, 32, 128, "bf16", seed=len(lens) + 5, window=1500)


def test_attention_strides_orders_and_default_queries(qe):
    """Q as a slice of a fused projection, out into a wider buffer, the same number of queries
    for each sequence without q_start; base addresses that allow no wide loads."""
    lens, dim, heads, kv = [40, 71], 72, 4, 2
    pages, table, held = cache(qe, lens, kv, dim, 64, 32, "bf16", 3)
    for shift in (0, 1):
        buf = draw((6, heads * dim + 16 + shift), 5, "bf16", spread=False).cuda()
        q = buf[:, 8 + shift:8 + shift + heads * dim].unflatten(1, (heads, dim))
        wide = torch.full((6, heads, dim + 8 + shift), 3.0, dtype=torch.bfloat16, device="cuda")
        qe.kv_attn(q, pages, dev(table), dev(np.array(lens, np.int32)), out=wide[:, :, shift:shift + dim])
        check(wide[:, :, shift:shift + dim], None, q, held, [3, 3], dim ** -0.5, "bf16")
        assert bool((wide[:, :, dim + shift:] == 3.0).all()) and bool((wide[:, :, :shift] == 3.0).all())
    hm = draw((heads, 6, dim), 6, "bf16").cuda().transpose(0, 1)       # head-major storage
    out = qe.kv_attn(hm, pages, dev(table), dev(np.array(lens, np.int32)))
    check(out, None, hm, held, [3, 3], dim ** -0.5, "bf16")


def test_attention_nan_groups_reach_their_rows_only(qe):
    """A NaN in a cached value or key spoils the rows that see it, not the others; the
    NaNs that lie past a sequence's end or outside of the window spoil none."""
    dim, page = 64, 32
    pages = qe.kv_pages(4, 1, dim, 32, page)
    pages.fill_(0xFF)                                  # every word a NaN, every code 15
    k, v = draw((50, 1, dim), 1).cuda(), draw((50, 1, dim), 2).cuda()
    v[20, 0, 40] = float("nan")
    qe.kv_write(k, v, torch.arange(50, device="cuda"), pages, group=32)
    table = dev(np.array([[0, 1, 2]], np.int32))
    q = draw((50, 2, dim), 3).cuda()
    for lens in (50,):
        L = dev(np.array([lens], np.int32))
        out = qe.kv_attn(q, pages, table, L, group=32)
        assert bool(torch.isfinite(out[:20]).all()) and bool(torch.isfinite(out[20:, :, :32]).all())
        assert bool(torch.isnan(out[20:, :, 32:]).all())
        out = qe.kv_attn(q, pages, table, L, group=32, window=10)
        assert bool(torch.isfinite(out[:20]).all()) and bool(torch.isfinite(out[30:]).all())
        assert bool(torch.isnan(out[20:30, :, 32:]).all())
    k[10, 0, 3] = float("inf")
    qe.kv_write(k, v, torch.arange(50, device="cuda"), pages, group=32)
    out = qe.kv_attn(q, pages, table, dev(np.array([50], np.int32)), group=32, window=5)
    assert bool(torch.isnan(out[10:15]).all()) and bool(torch.isfinite(out[:10]).all())
    assert bool(torch.isfinite(out[15:20]).all())


def test_attention_reports_bad_pages_lengths_and_ranges(qe):
    """Bad device data is reported and counts as absent: page numbers, lengths past the table,
    query ranges past Q."""
    dim = 64
    pages, table, held = cache(qe, [96], 1, dim, 64, 32, seed=1, noise=False)
    q = draw((1, 2, dim), 1).cuda()
    ws = qe.workspace(qe.kv_attn_workspace_size(1, 1, 1, 2, 1, dim), "cuda")
    bad = table.copy()
    bad[0, 1] = 10 ** 6
    out = qe.kv_attn(q, pages, dev(bad), dev(np.array([96], np.int32)), ws=ws)
    assert qe.sync_status(ws) == qe.QE_ERR_ARG and qe.sync_status(ws) == 0
    k, v = held[0]
    keep = np.r_[0:32, 64:96]
    check(out, None, q, [(k[keep], v[keep])], [1], dim ** -0.5, "f32")
    bad[0, 1] = -1
    with pytest.raises(qe.QEError):
        qe.kv_attn(q, pages, dev(bad), dev(np.array([96], np.int32)), ws=ws, check=True)
    out = qe.kv_attn(q, pages, dev(table[:, :3].copy()), dev(np.array([1000], np.int32)), ws=ws)
    assert qe.sync_status(ws) == qe.QE_ERR_ARG
    check(out, None, q, held, [1], dim ** -0.5, "f32")
    out = qe.kv_attn(q, pages, dev(table), dev(np.array([-5], np.int32)), ws=ws)
    assert qe.sync_status(ws) == qe.QE_ERR_ARG and not bool(out.any())
    out = torch.full((1, 2, dim), 9.0, device="cuda")
    qe.kv_attn(q, pages, dev(table), dev(np.array([96], np.int32)), ws=ws, out=out, max_q=1,
               q_start=dev(np.array([5, 9], np.int32)))
    assert qe.sync_status(ws) == qe.QE_ERR_ARG and bool((out == 9.0).all())
    out = qe.kv_attn(q, pages, dev(table), dev(np.array([96], np.int32)), ws=ws, max_q=1,
                     q_start=dev(np.array([0, 400], np.int32)))
    assert qe.sync_status(ws) == qe.QE_ERR_ARG
    check(out, None, q, held, [1], dim ** -0.5, "f32")


# Room in the page table from which rows of few units share tiles of 32 (32768 records of 32
# tokens over all units).
SPARE = 32768


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 128, 152, 256])
def test_attention_wide_tiles(qe, dim, group, dtype):
    """Tables with room for long sequences: rows that end inside of the first, the second and the third tile."""
    attend(qe, [70, 33, 0, 41], [9, 3, 1, 30], 6, 2, dim, group, 64, dtype, seed=dim, spare=SPARE)
    attend(qe, [800, 5000, 9], [1, 1, 1], 29, 1, dim, group, 32, dtype, seed=dim + 1, spare=SPARE)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_wide_tiles_masks(qe, dtype):
    attend(qe, [300, 17], [33, 12], 20, 20, 80, 64, 32, dtype, seed=4, slopes=True, spare=SPARE)
    attend(qe, [300, 17], [33, 40], 8, 2, 128, 64, 64, dtype, seed=5, causal=False, spare=SPARE)
    for window in (1, 33, 3000):
        # (a window bounds what a unit can read, so the units are many here)
        attend(qe, [90, 141], [90, 70], 64 if window < 3000 else 72, 64 if window < 3000 else 72, 64, 32, 32, dtype,
               seed=window, window=window, spare=SPARE)
    attend(qe, [140], [1], 32, 1, 64, 64, 64, dtype, seed=1, kscale=30.0, vscale=1e-6, spare=SPARE)
    attend(qe, [140], [20], 4, 2, 128, 32, 64, dtype, seed=2, kscale=1e-3, vscale=1e-3, qscale=1e-3, spare=SPARE)


def test_attention_wide_tiles_windows(qe):
    """Windows that mask (they bound the records of a unit, so it takes 4096 units of 8)."""
    attend(qe, [150, 4, 5, 6], [120, 1, 2, 1], 256, 256, 64, 32, 32, "bf16", seed=9, window=100, spare=64)


def test_attention_wide_tiles_bad_values_and_pages(qe):
    dim, n = 64, 50
    pages = qe.kv_pages(4, 1, dim, 32, 32)
    pages.fill_(0xFF)
    k, v = draw((n, 1, dim), 1).cuda(), draw((n, 1, dim), 2).cuda()
    v[40, 0, 40] = float("nan")
    qe.kv_write(k, v, torch.arange(n, device="cuda"), pages, group=32)
    table = np.full((1, SPARE), -1, np.int32)
    table[0, :2] = 0, 1
    L = dev(np.array([n], np.int32))
    q = draw((n, 2, dim), 3, "bf16").cuda()
    ws = qe.workspace(qe.kv_attn_workspace_size(n, 1, n, 2, 1, dim), "cuda")
    out = qe.kv_attn(q, pages, dev(table), L, group=32, ws=ws)
    assert qe.sync_status(ws) == 0
    assert bool(torch.isfinite(out[:40]).all()) and bool(torch.isfinite(out[40:, :, :32]).all())
    assert bool(torch.isnan(out[40:, :, 32:]).all())
    table[0, 0] = -1
    out = qe.kv_attn(q, pages, dev(table), L, group=32, ws=ws)
    assert qe.sync_status(ws) == qe.QE_ERR_ARG
    seen = [f64(x)[32:40] for x in qe.kv_read(pages, torch.arange(n, device="cuda"), dim, group=32)]
    assert not bool(out[:32].any())
    check(out[32:40], None, q[32:40], [seen], [8], dim ** -0.5, "bf16")


def many_rows(kv, lens, nqs, group, dim):
    """The sequences and as many short ones beside them as let the call take the form for many rows
    (its rule: 512 workgroups of at most 128 query rows of a key head, at least 128 rows a head)."""
    fill = -(-512 // kv)
    return list(lens) + [7] * fill, list(nqs) + [1] * fill


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 96, 128, 152, 192, 256])
def test_attention_many_rows_widths(qe, dim, group):
    """Every width and group; rows that see nothing, a head's rows in several tiles, empty sequences."""
    for dtype in DT:
        print(f"[kv] many dim={dim} group={group} {dtype}", flush=True)
        lens, nqs = many_rows(16, [131, 33, 0, 200], [131, 60, 2, 35], group, dim)
        attend(qe, lens, nqs, 16, 16, dim, group, 32 if dim % 16 else 64, dtype, seed=dim + group)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("heads,kv", [(12, 4), (29, 1), (40, 8)])
def test_attention_many_rows_shared_heads(qe, heads, kv, dtype):
    lens, nqs = many_rows(kv, [260, 97], [128, 97], 64, 64)
    attend(qe, lens, nqs, heads, kv, 64, 64, 64, dtype, seed=heads)
    attend(qe, lens, nqs, heads, kv, 128, 32, 32, dtype, seed=heads + 1, window=50, slopes=True)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("window", [0, 1, 33, 100, 5000])
def test_attention_many_rows_masks(qe, window, dtype):
    lens, nqs = many_rows(24, [300, 129, 3], [140, 129, 40], 64, 96)
    attend(qe, lens, nqs, 24, 24, 96, 64, 32, dtype, seed=window, window=window, slopes=True)
    attend(qe, lens, nqs, 24, 24, 96, 128, 64, dtype, seed=window + 1, window=window, causal=window != 0)


@pytest.mark.parametrize("dtype", list(DT))
def test_attention_many_rows_all_visible(qe, dtype):
    lens, nqs = many_rows(24, [300, 129, 3], [140, 129, 40], 64, 128)
    attend(qe, lens, nqs, 24, 24, 128, 64, 32, dtype, seed=2, causal=False)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("kscale,vscale,qscale", [(1e-6, 1e4, 1e4), (30.0, 1e-6, 1.0), (1e-3, 1e-3, 1e-3)])
def test_attention_many_rows_magnitudes(qe, dtype, kscale, vscale, qscale):
    if dtype == "f16" and qscale == 1e4:
        pytest.skip("fp16 holds no such queries and values")
    lens, nqs = many_rows(16, [140], [140], 64, 64)
    attend(qe, lens, nqs, 16, 16, 64, 64, 64, dtype, seed=1, kscale=kscale, vscale=vscale, qscale=qscale)


def test_attention_many_rows_fp32_as_a_whole(qe):
    n, heads, dim = 500, 64, 80
    pages, table, held = cache(qe, [n], heads, dim, 64, 32, "f32", 5)
    q = draw((n, heads, dim), 12, "f32", 0.5).cuda()
    out = qe.kv_attn(q, pages, dev(table), dev(np.array([n], np.int32)))
    ref, _, _ = okv.attention(f64(q), *held[0], np.arange(n), dim ** -0.5)
    assert np.linalg.norm(f64(out) - ref) <= 2.0 ** -20 * np.linalg.norm(ref)


def test_attention_many_rows_bad_values_and_pages(qe):
    """NaN and infinite groups spoil the rows that see them, also beside a page that is missing; the
    bytes past a sequence's end spoil none."""
    dim, heads, n = 64, 200, 140
    pages = qe.kv_pages(6, heads, dim, 32, 32)
    pages.fill_(0xFF)
    k, v = draw((n, heads, dim), 1).cuda(), draw((n, heads, dim), 2).cuda()
    v[20, :, 40] = float("nan")
    k[10, :, 3] = float("inf")
    qe.kv_write(k, v, torch.arange(n, device="cuda"), pages, group=32)
    table, L = np.array([[0, 1, 2, 3, 4]], np.int32), dev(np.array([n], np.int32))
    q = draw((n, heads, dim), 3).cuda()
    ws = qe.workspace(qe.kv_attn_workspace_size(n, 1, n, heads, heads, dim), "cuda")
    out = qe.kv_attn(q, pages, dev(table), L, group=32, window=5, ws=ws)
    assert qe.sync_status(ws) == 0
    assert bool(torch.isnan(out[10:15]).all()) and bool(torch.isfinite(out[:10]).all())
    assert bool(torch.isfinite(out[15:20]).all()) and bool(torch.isfinite(out[25:]).all())
    assert bool(torch.isnan(out[20:25, :, 32:]).all()) and bool(torch.isfinite(out[20:25, :, :32]).all())
    for absent in (-1, 10 ** 6):
        table[0, 0] = absent
        out = qe.kv_attn(q, pages, dev(table), L, group=32, ws=ws)
        assert qe.sync_status(ws) == qe.QE_ERR_ARG
        assert not bool(out[:32].any())
        seen = f64(qe.kv_read(pages, torch.arange(n, device="cuda"), dim, group=32)[0]), f64(
            qe.kv_read(pages, torch.arange(n, device="cuda"), dim, group=32)[1])
        check(out[32:], None, q[32:], [tuple(x[32:] for x in seen)], [n - 32], dim ** -0.5, "f32")


def test_attention_is_deterministic_and_replays(qe):
    """The same bits from call to call, on another stream, and from a graph between other work."""
    lens = [3000, 77]
    pages, table, _ = cache(qe, lens, 2, 128, 64, 64, "bf16", 9)
    q = draw((2, 8, 128), 1, "bf16").cuda()
    T, L = dev(table), dev(np.array(lens, np.int32))
    ws = qe.workspace(qe.kv_attn_workspace_size(2, 2, 1, 8, 2, 128), "cuda")
    slots = dev(np.array([table[0, 0] * 64 + 1, table[1, 0] * 64 + 5], np.int64))
    k, v = draw((2, 2, 128), 2, "bf16").cuda(), draw((2, 2, 128), 3, "bf16").cuda()
    out, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")

    def step():
        qe.kv_write(k, v, slots, pages)
        qe.kv_attn(q, pages, T, L, out=out, lse=lse, ws=ws)

    step()
    torch.cuda.synchronize()
    want, want_lse = out.clone(), lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.fill_(0)
        step()
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        out.fill_(1.0)
        lse.fill_(1.0)
        pages[table[0, 0], :, 0, :64] = 0
        torch.cuda.synchronize()
        qe.kv_write(k, v, slots, pages)
        graph.replay()
        torch.cuda.synchronize()
        again = out.clone()
        qe.kv_attn(q, pages, T, L, out=out, ws=ws)
        assert torch.equal(out, again)


def test_cache_past_four_gigabytes(qe):
    """Pages whose bytes lie past 2^32, written, read and attended to."""
    dim, page, heads = 128, 256, 8
    per = qe.kv_page_bytes(heads, dim, 64, page)
    num = (5 << 30) // per
    pages = qe.kv_pages(num, heads, dim, 64, page)
    ids = np.array([[num - 1, 3, num - 2]], np.int32)
    n = 600
    t = np.arange(n)
    slots = dev(ids[0][t // page].astype(np.int64) * page + t % page)
    k, v = draw((n, heads, dim), 1, "bf16").cuda(), draw((n, heads, dim), 2, "bf16").cuda()
    qe.kv_write(k, v, slots, pages)
    K, V = qe.kv_read(pages, slots, dim)
    c, w = okv.quantize(f64(k[::37]), 64)
    assert np.array_equal(host(K)[::37], okv.values(c, w, dim, 64))
    q = draw((1, 16, dim), 3, "bf16").cuda()
    out = qe.kv_attn(q, pages, dev(ids), dev(np.array([n], np.int32)))
    check(out, None, q, [(f64(K), f64(V))], [1], dim ** -0.5, "bf16")
    del pages
    torch.cuda.empty_cache()


def test_binding_refusals(qe):
    pages = qe.kv_pages(2, 2, 64, 64, 64)
    k = torch.zeros((3, 2, 64), device="cuda")
    s = torch.arange(3, device="cuda")
    T, L = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 4, 64), device="cuda")
    for bad in (lambda: qe.kv_pages(1, 2, 60), lambda: qe.kv_pages(1, 2, 264), lambda: qe.kv_pages(1, 2, 64, 48),
                lambda: qe.kv_pages(1, 2, 64, 64, 40), lambda: qe.kv_pages(0, 2, 64),
                lambda: qe.kv_write(k, k, s, pages, group=32), lambda: qe.kv_write(k, k.half(), s, pages),
                lambda: qe.kv_write(k, k, s[:2], pages), lambda: qe.kv_write(k, k, s.int(), pages),
                lambda: qe.kv_write(k[:, :1], k[:, :1], s, pages), lambda: qe.kv_write(k.double(), k.double(), s, pages),
                lambda: qe.kv_write(k.cpu(), k, s, pages), lambda: qe.kv_write(k.transpose(1, 2), k, s, pages),
                lambda: qe.kv_read(pages, s, 128), lambda: qe.kv_read(pages, s, 64, dtype=torch.float64),
                lambda: qe.kv_attn(q, pages, T.long(), L), lambda: qe.kv_attn(q, pages, T, L.long()),
                lambda: qe.kv_attn(q[..., :56], pages, T, L, group=32), lambda: qe.kv_attn(q[0], pages, T, L),
                lambda: qe.kv_attn(q, pages, T, L, q_start=torch.zeros(2, dtype=torch.int32, device="cuda")),
                lambda: qe.kv_attn(q, pages, T, L, max_q=3),
                lambda: qe.kv_attn(q, pages, T, L, slopes=torch.zeros(3, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qe.kv_attn(q[:, :3], pages, T, L), lambda: qe.kv_attn(q, pages, T, L, window=-1),
                lambda: qe.kv_attn(q, pages, T, L, window=4, causal=False),
                lambda: qe.kv_attn(q, pages, T, L, scale=float("nan")),
                lambda: qe.kv_attn(q, pages, T, L, ws=torch.zeros(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(qe.QEError):
            bad()
