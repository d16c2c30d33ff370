"""A step of many sequences around the 4-bit cache: pages and slots (kv_extend), norm, rotation and write (kv_append),
and a run of both with attention, against the plain CPU forms of oracle/kv.py.

Pages, slots and lengths are integers; a query or key is made of fp32 operations that are each correctly rounded, in a
stated order, with a sum in 64 bits that only meets a rounding to 32: everything is compared bit for bit (the two
sums in 64 bits differ by 2^-50 of themselves at most, which moves an fp32 rounding once in 2^25 rows)."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from parity import dev, host
from test_gpu_kv import DT, bits, draw, f64, rounded

pytestmark = pytest.mark.gpu


def i32(x):
    return np.asarray(x, np.int32)


class Pool:
    """Sequences, their table and the free pages, on the CPU and on the GPU."""

    def __init__(self, lengths, page, width, spare, keep=None, seed=0):
        r = np.random.default_rng(seed)
        self.page, batch = page, len(lengths)
        self.keep = None if keep is None else i32(keep)
        held = [max(-(-n // page), 0 if keep is None else keep[b]) for b, n in enumerate(lengths)]
        order = i32(r.permutation(sum(held) + spare))
        self.table = np.full((batch, width), -1, np.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.free = np.full(max(order.size, 1), -1, np.int32)
        self.free[:spare] = order[at:]
        self.free_count, self.lengths = spare, i32(lengths)
        self.upload()

    def upload(self):
        self.dtable, self.dlengths, self.dfree = dev(self.table), dev(self.lengths), dev(self.free)
        self.dcount = dev(i32([self.free_count]))
        self.dkeep = None if self.keep is None else dev(self.keep)

    def step(self, qe, counts, total, **more):
        """The call, compared with the oracle; (slots, positions, q_start, lacking) and whether something was bad."""
        counts = i32(counts)
        lacking = torch.full((1,), -7, dtype=torch.int32, device="cuda")
        ws = qe.workspace(qe.kv_extend_workspace_size(counts.size), "cuda")
        got = qe.kv_extend(dev(counts), self.dtable, self.dlengths, self.dfree, self.dcount, self.page, total, keep=self.dkeep,
                           lacking=lacking, ws=ws, **more)
        want = okv.extend(counts, self.table, self.lengths, self.free, self.free_count, self.page, total, self.keep)
        self.free_count = want[3]
        for g, w, name in zip(got, want, ("slots", "positions", "q_start")):
            assert np.array_equal(host(g), w), name
        assert np.array_equal(host(self.dtable), self.table)
        assert np.array_equal(host(self.dlengths), self.lengths)
        assert np.array_equal(host(self.dfree), self.free)
        assert int(self.dcount) == self.free_count and int(lacking) == want[4]
        assert (qe.sync_status(ws) != qe.QE_OK) == want[5]
        return want


def mixed(r, lengths, keep, page, most):
    """Counts: new tokens, none, and tokens that go back (never into the kept pages)."""
    out = []
    for b, n in enumerate(lengths):
        k = 0 if keep is None else keep[b] * page
        out.append(int(r.choice([0, 1, 1, r.integers(0, most + 1), -r.integers(0, max(n - k, 0) + 1)])))
    return out


# ------------------------------------------------------------------ pages and slots
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("batch,page,most", [(1, 32, 5), (2, 64, 200), (63, 32, 40), (64, 96, 1), (257, 64, 70), (1024, 32, 2),
                                             (1025, 32, 9), (2500, 64, 130), (5000, 32, 1)])
def test_extend_steps(qe, batch, page, most, keep):
    """Three steps and their undoing, which restores everything; padded rows."""
    r = np.random.default_rng(batch + most)
    kept = r.integers(0, 4, batch).tolist() if keep else None
    lengths = [int(r.integers(0, 300)) + (kept[b] * page if keep else 0) for b in range(batch)]
    width = (300 + 3 * most) // page + 8
    p = Pool(lengths, page, width, spare=batch * (3 * most // page + 3), keep=kept, seed=batch)
    first = [x.copy() for x in (p.table, p.lengths, p.free[:p.free_count])]
    done = []
    for n in range(3):
        counts = mixed(r, p.lengths, kept, page, most)
        total = sum(max(c, 0) for c in counts)
        assert not p.step(qe, counts, total + 5 * n)[5]
        done.append(counts)
    for counts in reversed(done):
        assert not p.step(qe, [-c for c in counts], sum(max(-c, 0) for c in counts))[5]
    for a, b in zip(first, (p.table, p.lengths, p.free[:p.free_count])):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("prompt", [1, 31, 33, 2047, 2048, 2049, 40000])
def test_extend_one_prompt(qe, prompt):
    """Both sides of the size from which slots have a launch of their own."""
    p = Pool([0], 32, 1300, spare=1260)
    p.step(qe, [prompt], prompt)
    p.step(qe, [1], 1)
    p.step(qe, [-prompt - 1], 0)
    assert p.lengths[0] == 0 and p.free_count == 1260


@pytest.mark.parametrize("spare", [0, 1, 7, 20, 21])
@pytest.mark.parametrize("pad", [0, 3000])
def test_extend_runs_out(qe, spare, pad):
    """All of a sequence's pages or none, in order; what others give back in the same call counts."""
    lengths = [10, 64, 0, 33, 96, 5, 0]
    counts = [30, 1, 200, -33, 33, 20, 90]
    p = Pool(lengths, 32, 12, spare)
    want = p.step(qe, counts, sum(max(c, 0) for c in counts) + pad)
    assert not want[5] and (want[4] > 0) == (spare + 2 < 1 + 1 + 7 + 2 + 3)
    assert p.lengths[5] == 25                              # wants no page


@pytest.mark.parametrize("pad", [0, 3000])
def test_extend_of_bad_arguments(qe, pad):
    """Sequences that do not fit stay as they are, the others get theirs."""
    lengths, page, width = [-1, 64, 20 * 32, 700 * 32, 5, 2 ** 31 - 1, 40], 32, 21
    p = Pool([0, 64, 20 * 32, 0, 5, 0, 40], page, width, 60)
    p.lengths[:] = lengths
    p.upload()
    assert p.step(qe, [3, 2, 33, 1, 4, 2 ** 31 - 1, 1], 3 + 2 + 33 + 1 + 4 + pad)[5]
    p = Pool([0, 40], page, width, 60)
    p.keep = i32([-1, 22])
    p.upload()
    assert p.step(qe, [5, 5], 10 + pad)[5]
    # rows past `total`
    p = Pool([0, 40, 7], page, width, 60)
    assert p.step(qe, [5, 10, 3], 14)[5]
    assert p.lengths.tolist() == [5, 40, 7]


@pytest.mark.parametrize("count", [-1, 61])
def test_extend_of_a_bad_stack(qe, count):
    p = Pool([0, 40], 32, 10, 60)
    p.free_count = count
    p.upload()
    assert p.step(qe, [40, 40], 80)[5]


def test_extend_of_a_stack_that_overflows(qe):
    """A sequence's pages are free already (a mistake of the program's): what does not fit is lost, nothing else is touched."""
    p = Pool([320, 96], 32, 20, 3)
    p.free_count = p.free.size - 2
    p.upload()
    guard = p.dfree.clone()
    assert p.step(qe, [-320, 1], 1)[5]
    assert guard.numel() == p.dfree.numel()


def test_extend_takes_no_page_that_is_not_there(qe):
    p = Pool([0, 0], 32, 4, 6)
    p.free[[1, 3]] = [-5, 1000]
    p.upload()
    assert p.step(qe, [96, 96], 192)[5]


def test_extend_of_nothing(qe):
    p = Pool([], 32, 4, 6)
    p.step(qe, [], 0)
    p.step(qe, [], 7)
    p = Pool([5], 32, 4, 6)
    p.step(qe, [0], 0)
    p = Pool([0, 0], 32, 0, 6)
    assert p.step(qe, [0, 1], 1)[5]


def test_extend_into_given_tensors_on_a_stream(qe):
    p = Pool([5, 50], 32, 4, 6)
    outs = dict(slots=torch.full((4,), 9, dtype=torch.int64, device="cuda"),
                positions=torch.full((4,), 9, dtype=torch.int32, device="cuda"),
                q_start=torch.full((3,), 9, dtype=torch.int32, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = qe.kv_extend(dev(i32([1, 2])), p.dtable, p.dlengths, p.dfree, p.dcount, 32, 4, stream=side, check=True, **outs)
    torch.cuda.current_stream().wait_stream(side)
    want = okv.extend([1, 2], p.table, p.lengths, p.free, p.free_count, 32, 4)
    for g, o, w in zip(got, outs.values(), want):
        assert g is o and np.array_equal(host(g), w)


def test_extend_reports(qe):
    p = Pool([5], 32, 4, 6)
    with pytest.raises(qe.QEError):
        qe.kv_extend(dev(i32([1000])), p.dtable, p.dlengths, p.dfree, p.dcount, 32, 1000, check=True)


# ------------------------------------------------------------------ norm, rotation, write
def tables(rows, rot):
    turn = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    angle = np.arange(rows)[:, None] * turn
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def append(qe, q, k, v, slots, pages, group, positions=None, cos=None, sin=None, interleaved=False, qw=None, kw=None, eps=1e-6,
           out=None, dtype=None, tell=None):
    """The call and the oracle's pages and queries (rows that are skipped: as out was)."""
    want_pages = host(pages)
    before = None if out is None else f64(out)
    up = lambda x: None if x is None else dev(x)  # noqa: E731
    got = qe.kv_append(q, k, v, dev(slots), pages, group=group, positions=up(positions), cos=up(cos), sin=up(sin),
                       interleaved=interleaved, q_weight=up(qw), k_weight=up(kw), eps=eps, out=out, status=tell)
    how = (eps, positions, cos, sin, interleaved)
    there = np.ones(len(slots), bool)
    if positions is not None:
        there = positions >= 0
        if cos is not None:
            there &= positions < cos.shape[0]
            how = (eps, np.minimum(positions, cos.shape[0] - 1), cos, sin, interleaved)
    okv.write(want_pages, np.where(there, slots, -1), okv.norm_rotate(f64(k), kw, *how), f64(v), group)
    want = okv.norm_rotate(f64(q), qw, *how)
    want = rounded(want, dtype)
    if before is not None:
        want[~torch.from_numpy(there)] = rounded(before, dtype)[~torch.from_numpy(there)]
    return got, want, want_pages, there


SHAPES = [(dim, group) for dim in (8, 40, 64, 80, 96, 120, 128, 160, 192, 200, 256) for group in (32, 64, 128)]


@pytest.mark.parametrize("dim,group", SHAPES)
def test_append_bits(qe, dim, group):
    """Every width: partial and whole records, norms, a part of the channels rotated, either pairing."""
    n = dim // 8 + group // 32
    dtype, heads, kv, tokens, page = list(DT)[n % 3], 3, 2, 45, 64
    q, k = draw((tokens, heads, dim), n, dtype), draw((tokens, kv, dim), n + 1, dtype)
    v = draw((tokens, kv, dim), n + 2, dtype)
    rot = [dim, dim // 2, 2, dim // 4 // 2 * 2][n % 4]
    cos, sin = tables(300, rot)
    r = np.random.default_rng(n)
    weights = [np.exp(0.3 * r.standard_normal(dim)).astype(np.float32) for _ in range(2)]
    pages = qe.kv_pages(4, kv, dim, group, page)
    pages.fill_(0xAB)
    slots = np.arange(page - 5, page - 5 + tokens)
    got, want, want_pages, _ = append(qe, q.cuda(), k.cuda(), v.cuda(), slots, pages, group, i32(r.integers(0, 300, tokens)), cos,
                                      sin, n % 2 == 1, *weights, dtype=dtype)
    assert np.array_equal(host(pages), want_pages)
    assert np.array_equal(bits(got), bits(want))


@pytest.mark.parametrize("rot", [0, 2, 10, 16, 20, 36, 64, 80])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["both", "q", "k", ""])
def test_append_parts(qe, rot, interleaved, norm):
    """Any number of rotated channels, each norm by itself, in place."""
    dim, tokens, dtype = 80, 33, "bf16"
    q, k, v = (draw((tokens, h, dim), rot + h, dtype).cuda() for h in (5, 1, 1))
    cos, sin = tables(50, rot) if rot else (None, None)
    w = np.linspace(0.5, 2.0, dim, dtype=np.float32)
    pages = qe.kv_pages(3, 1, dim, 32, 32)
    before = q.clone()
    got, want, want_pages, _ = append(qe, q, k, v, np.arange(tokens) + 7, pages, 32, i32(np.arange(tokens)), cos, sin, interleaved,
                                      w if norm in ("both", "q") else None, w[::-1].copy() if norm in ("both", "k") else None,
                                      dtype=dtype)
    assert np.array_equal(host(pages), want_pages) and np.array_equal(bits(got), bits(want))
    assert torch.equal(q, before)
    qe.kv_append(q, k, v, dev(np.arange(tokens) + 7), pages, group=32, positions=dev(i32(np.arange(tokens))),
                 cos=None if cos is None else dev(cos), sin=None if sin is None else dev(sin), interleaved=interleaved,
                 q_weight=dev(w) if norm in ("both", "q") else None,
                 k_weight=dev(w[::-1].copy()) if norm in ("both", "k") else None, out=q)
    assert np.array_equal(bits(q), bits(want)) and np.array_equal(host(pages), want_pages)


@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 64, 97, 500])
@pytest.mark.parametrize("dtype", list(DT))
def test_append_counts(qe, tokens, dtype):
    heads, kv, dim = 7, 3, 64
    q, k, v = (draw((tokens, h, dim), tokens + h, dtype).cuda() for h in (heads, kv, kv + 0))
    cos, sin = tables(tokens + 5, dim)
    w = np.linspace(0.5, 2.0, dim, dtype=np.float32)
    pages = qe.kv_pages(9, kv, dim, 64, 64)
    got, want, want_pages, _ = append(qe, q, k, v, np.arange(tokens) + 31, pages, 64, i32(np.arange(tokens) + 5), cos, sin, False, w, w,
                                      dtype=dtype)
    assert np.array_equal(host(pages), want_pages) and np.array_equal(bits(got), bits(want))


@pytest.mark.parametrize("tokens,heads,dim,rot,interleaved", [(1100, 31, 128, 128, False), (2100, 25, 128, 36, False),
                                                              (4100, 13, 96, 96, True), (1500, 19, 256, 128, False)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_runs_of_heads(qe, tokens, heads, dim, rot, interleaved, dtype):
    """Enough tokens and heads that a workgroup goes through two to four heads, the last one through fewer; tokens without
    a position among them, in place."""
    q, k = draw((tokens, heads, dim), 1, dtype).cuda(), draw((tokens, 1, dim), 2, dtype).cuda()
    cos, sin = tables(tokens + 9, rot)
    w = np.linspace(0.5, 2.0, dim, dtype=np.float32)
    positions = i32(np.arange(tokens) + 9)
    positions[::7] = -1
    pages = qe.kv_pages(-(-tokens // 128), 1, dim, 128, 128)
    before = q.clone()
    got, want, want_pages, _ = append(qe, q, k, k, np.arange(tokens), pages, 128, positions, cos, sin, interleaved, w, w, out=q,
                                      dtype=dtype)
    # (append's reference reads q after the call where it is the output: the rows are formed again from the copy)
    want = rounded(okv.norm_rotate(f64(before), w, 1e-6, np.maximum(positions, 0), cos, sin, interleaved), dtype)
    skipped = torch.from_numpy(positions < 0)
    want[skipped] = before.cpu()[skipped]
    assert got is q and np.array_equal(bits(q), bits(want)) and np.array_equal(host(pages), want_pages)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dtype", list(DT))
def test_append_strided(qe, dtype, shift):
    """Slices of a fused projection, aligned and not; the output into a slice whose neighbours stay."""
    tokens, heads, kv, dim = 40, 4, 2, 72
    buf = draw((tokens, (heads + 2 * kv) * dim + 60 + shift), 11, dtype, spread=False).cuda()
    part = lambda a, h: buf[:, 24 + shift + a * dim:24 + shift + (a + h) * dim].unflatten(1, (h, dim))  # noqa: E731
    q, k, v = part(0, heads), part(heads, kv), part(heads + kv, kv)
    cos, sin = tables(60, 36)
    w = np.linspace(0.5, 2.0, dim, dtype=np.float32)
    pages = qe.kv_pages(2, kv, dim, 64, 64)
    room = torch.full((tokens, heads, dim + 8 + shift), 3.0, dtype=DT[dtype], device="cuda")
    got, want, want_pages, _ = append(qe, q, k, v, np.arange(tokens) + 3, pages, 64, i32(np.arange(tokens)), cos, sin, True, w, None,
                                      out=room[..., shift:shift + dim], dtype=dtype)
    assert np.array_equal(host(pages), want_pages) and np.array_equal(bits(got), bits(want))
    assert bool((room[..., shift + dim:] == 3).all()) and bool((room[..., :shift] == 3).all())
    # a token's row many times (stride 0)
    one = k[:1].expand(tokens, kv, dim)
    _, _, want_pages, _ = append(qe, q, one, v, np.arange(tokens) + 3, pages, 64, i32(np.arange(tokens)), cos, sin, dtype=dtype)
    assert np.array_equal(host(pages), want_pages)


def test_append_skips(qe):
    """Rows without a position are left as they were, those without a slot get their query alone."""
    tokens, dtype = 70, "f16"
    q, k, v = (draw((tokens, h, 64), h, dtype).cuda() for h in (3, 2, 2))
    cos, sin = tables(100, 64)
    r = np.random.default_rng(1)
    positions, slots = i32(r.integers(0, 100, tokens)), r.permutation(160)[:tokens]
    positions[[2, 30, 69]] = -1, -2 ** 31, -5
    slots[[3, 31, 68]] = -1, -2 ** 40, -1
    pages = qe.kv_pages(5, 2, 64, 32, 32)
    out = torch.full((tokens, 3, 64), 7.0, dtype=DT[dtype], device="cuda")
    tell = torch.zeros(1, dtype=torch.int32, device="cuda")
    w = np.ones(64, np.float32)
    got, want, want_pages, there = append(qe, q, k, v, slots, pages, 32, positions, cos, sin, False, w, w, out=out, dtype=dtype, tell=tell)
    assert np.array_equal(host(pages), want_pages) and np.array_equal(bits(got), bits(want)) and not there[2]
    assert int(tell) == 0
    positions[5], slots[6] = 100, 160                       # past the tables, past the cache
    out.fill_(7.0)
    got, want, want_pages, there = append(qe, q, k, v, slots, pages, 32, positions, cos, sin, False, w, w, out=out, dtype=dtype, tell=tell)
    assert np.array_equal(host(pages), want_pages) and np.array_equal(bits(got), bits(want)) and not there[5]
    assert int(tell) == qe.QE_ERR_ARG
    # without a rotation a position only says whether the token is there
    out.fill_(7.0)
    got, want, want_pages, _ = append(qe, q, k, v, np.where(slots < 160, slots, -1), pages, 32, positions, qw=w, out=out, dtype=dtype)
    assert np.array_equal(host(pages), want_pages) and np.array_equal(bits(got), bits(want))


@pytest.mark.parametrize("dtype", list(DT))
def test_append_special_values(qe, dtype):
    """Zeros, NaN, infinities, values whose squares pass fp32's range, the smallest ones."""
    dim = 64
    top = float(torch.finfo(DT[dtype]).max)
    rows = np.zeros((9, 1, dim))
    rows[1:] = f64(draw((8, 1, dim), 3, "f32"))
    rows[2, 0, 5] = np.nan
    rows[3, 0, 6] = np.inf
    rows[4, 0, 7] = -np.inf
    rows[5] *= top / 64 if dtype == "f16" else 1e30
    rows[6, 0, :] = top
    rows[7] *= 1e-30 if dtype != "f16" else 1e-6
    x = rounded(rows, dtype).cuda()
    cos, sin = tables(20, dim)
    w = np.linspace(0.5, 2.0, dim, dtype=np.float32)
    for eps in (1e-6, 0.0):
        pages = qe.kv_pages(1, 1, dim, 32, 32)
        got, want, want_pages, _ = append(qe, x, x, x, np.arange(9), pages, 32, i32(np.arange(9)), cos, sin, False, w, w, eps, dtype=dtype)
        g, t = f64(got), f64(want)
        assert np.array_equal(np.isnan(g), np.isnan(t))
        assert np.array_equal(g[~np.isnan(t)], t[~np.isnan(t)])
        assert np.array_equal(host(pages), want_pages)


@pytest.mark.parametrize("dim,group", [(8, 32), (40, 64), (72, 32), (136, 32), (200, 32)])
def test_append_keeps_padding(qe, dim, group):
    """Rows whose norm is infinite or NaN: the record's channels past dim hold 0 all the same."""
    x = f64(draw((4, 1, dim), 3, "f32"))
    x[1], x[2, 0, 3], x[3, 0, 5] = 0.0, np.nan, np.inf
    x = rounded(x, "f32").cuda()
    w = np.linspace(0.5, 2.0, dim, dtype=np.float32)
    pages = qe.kv_pages(1, 1, dim, group, 32)
    _, _, want_pages, _ = append(qe, x, x, x, np.arange(4), pages, group, qw=w, kw=w, eps=0.0, dtype="f32")
    assert np.array_equal(host(pages), want_pages)


def test_append_of_nothing(qe):
    pages = qe.kv_pages(1, 1, 64, 64, 32)
    e = torch.empty(0, 2, 64, device="cuda")
    got = qe.kv_append(e, e[:, :1], e[:, :1], torch.empty(0, dtype=torch.int64, device="cuda"), pages)
    assert got.shape == (0, 2, 64)


def test_append_refusals(qe):
    pages = qe.kv_pages(1, 1, 64, 64, 32)
    q, k = torch.zeros(2, 2, 64, device="cuda"), torch.zeros(2, 1, 64, device="cuda")
    slots, pos = torch.arange(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    t = torch.zeros(4, 32, device="cuda")
    ok = dict(positions=pos, cos=t, sin=t)
    qe.kv_append(q, k, k, slots, pages, **ok)
    for bad in (dict(ok, sin=None), dict(ok, positions=None), dict(ok, cos=t[:3]), dict(ok, cos=t.double(), sin=t.double()),
                dict(ok, positions=pos.long()), dict(ok, positions=pos[:1]), dict(ok, q_weight=t[0]), dict(ok, cos=t.cpu(), sin=t.cpu()),
                dict(ok, out=q.half()), dict(ok, out=q[:1]), dict(ok, cos=torch.zeros(8, 32, device="cuda")[::2], sin=t)):
        with pytest.raises(ValueError):
            qe.kv_append(q, k, k, slots, pages, **bad)
    wide = torch.zeros(4, 33, device="cuda")
    for bad in (dict(ok, cos=wide, sin=wide), dict(ok, cos=t[:0], sin=t[:0]), dict(ok, eps=-1.0), dict(ok, eps=float("nan"))):
        with pytest.raises(qe.QEError):
            qe.kv_append(q, k, k, slots, pages, **bad)
    with pytest.raises(ValueError):
        qe.kv_append(q, k.half(), k, slots, pages, **ok)
    with pytest.raises(ValueError):
        qe.kv_append(q, k, k, slots.int(), pages, **ok)


def test_extend_refusals(qe):
    p = Pool([5, 50], 32, 4, 6)
    counts = dev(i32([1, 1]))
    args = (p.dtable, p.dlengths, p.dfree, p.dcount, 32, 2)
    for bad in ((counts.long(),) + args, (counts[:1],) + args, (counts.cpu(),) + args, (counts, p.dtable.cpu()) + args[1:],
                (counts, p.dtable[:, ::2]) + args[1:], (counts, p.dtable.flatten()) + args[1:], (counts, p.dtable, p.dlengths.long()) + args[2:],
                (counts, p.dtable, p.dlengths, p.dfree.long()) + args[3:], (counts,) + args[:3] + (p.dfree,) + args[4:]):
        with pytest.raises(ValueError):
            qe.kv_extend(*bad)
    for more in (dict(keep=counts.long()), dict(slots=counts), dict(positions=counts[:1]), dict(q_start=counts), dict(lacking=counts)):
        with pytest.raises(ValueError):
            qe.kv_extend(counts, *args, **more)
    for bad in ((48, 2), (0, 2), (32, -1)):
        with pytest.raises((qe.QEError, RuntimeError)):
            qe.kv_extend(counts, *args[:4], *bad)
    with pytest.raises(qe.QEError):
        qe.kv_extend(counts, *args, ws=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert np.array_equal(host(p.dlengths), p.lengths) and np.array_equal(host(p.dtable), p.table)


@pytest.mark.parametrize("graph", [False, True])
def test_append_on_a_stream(qe, graph):
    """A call on a stream of its own, and a recorded one whose tokens change between the replays."""
    tokens, dtype = 40, "bf16"
    q, k, v = (draw((tokens, h, 64), h, dtype).cuda() for h in (4, 2, 3))
    v = v[:, :2]
    cos, sin = tables(100, 64)
    w = np.linspace(0.5, 2.0, 64, dtype=np.float32)
    pages = qe.kv_pages(3, 2, 64, 32, 32)
    slots, positions = dev(np.arange(tokens) + 9), dev(i32(np.arange(tokens)))
    d = [dev(x) for x in (cos, sin, w)]
    call = lambda s=None: qe.kv_append(q, k, v, slots, pages, group=32, positions=positions, cos=d[0], sin=d[1], q_weight=d[2], k_weight=d[2],  # noqa: E731
                                       stream=s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = call(side)
    torch.cuda.current_stream().wait_stream(side)
    out.record_stream(torch.cuda.current_stream())
    if graph:
        rec = torch.cuda.CUDAGraph()
        with torch.cuda.graph(rec):
            out = call()
    for n in range(3 if graph else 1):
        if graph:
            q.copy_(draw(q.shape, 50 + n, dtype).cuda())
            positions.copy_(dev(i32((np.arange(tokens) * 7 + n) % 100 - (np.arange(tokens) == n))))
            rec.replay()
            torch.cuda.synchronize()
        pos = host(positions)
        there = torch.from_numpy(pos >= 0)
        want = rounded(okv.norm_rotate(f64(q), w, 1e-6, pos, cos, sin, False), dtype)
        assert np.array_equal(bits(out.cpu()[there]), bits(want[there]))
        if n == 0:
            expect = np.zeros_like(host(pages))
        okv.write(expect, np.where(pos < 0, -1, np.arange(tokens) + 9), okv.norm_rotate(f64(k), w, 1e-6, pos, cos, sin, False), f64(v), 32)
        if not graph:
            assert np.array_equal(host(pages), expect)
