"""The 4-bit key/value cache of a decoder that this library's layers are used in, as timed cases.

A program that serves a quantized model keeps the keys and values of past tokens in
4 bits as well.  Three operators do that: `kv_write` quantizes the keys and values of
new tokens into a paged cache, `kv_read` gives back the values that the cache stands
for, and `kv_attn` is causal attention over the cache, for one new token of each
sequence or for a chunk of them.  With `own` false, `run` computes the same from
elementary torch operations in fp32; with `own` true it calls the library.

The grid of a group of channels x of one token and head (all steps in fp32):
    lo = min(0, min x), hi = max(0, max x)
    s  = max((hi - lo) / 15, 2^-126), its bit pattern rounded to a multiple of 16
    z  = rint(-lo * (1 / s)),   n = clamp(rint(x * (1 / s)) + z, 0, 15)
and the cache stands for s * (n - z).

The cache is a byte tensor (pages, kv heads, page / 32, record): a record holds 32
consecutive tokens of one head.  With Dp = dim rounded up to 64, 96, 128, 192 or 256
(the channels past dim hold 0), NC = Dp / 32 and NG = ceil(Dp / group) it is, in this order:
    32 key rows of NC * 4 words; word j * NC + c holds channels 8 (4 c + j) .. + 7,
        four bits each, the lowest channel in the lowest bits
    NG x 32 words (group-major): the bit pattern of the key group's s, z in its low four bits
    Dp / 4 x 32 half-words: channels 4 u .. + 3 of the value of each of the 32 tokens
    NG x 32 words for the value groups
Token t of a sequence lies in page table[t // page], its slot is table[t // page] * page + t % page.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
TINY = 2.0 ** -126


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # ---- write, then read back what the cache holds of these tokens
        # one new token of one sequence: the smallest call, latency alone
        dict(name="store_1", kind="store", seqs=1, tokens=1, kv_heads=8, dim=128, group=64, page=64,
             dtype="bf16", start=1000),
        # fp32 activations as the layers of this library have them, at a head size that is padded,
        # an odd number of heads and of tokens, starting inside a record
        dict(name="store_1003_f32", kind="store", seqs=1, tokens=1003, kv_heads=5, dim=80, group=32,
             page=32, dtype="f32", start=37),
        # a prompt's chunk for grouped heads
        dict(name="store_2048", kind="store", seqs=1, tokens=2048, kv_heads=8, dim=128, group=64,
             page=64, dtype="bf16", start=4096),
        # a batch of prompts with a key head for each of the 32 query heads of a 4096-wide layer
        dict(name="store_8x4096", kind="store", seqs=8, tokens=4096, kv_heads=32, dim=128, group=128,
             page=128, dtype="f16", start=0),
        # ---- read a cached prefix back
        # a short prefix of a model with one key head (71 query heads of 64, width 4544)
        dict(name="read_777", kind="read", tokens=777, kv_heads=1, dim=64, group=32, page=32,
             dtype="f32"),
        # a long document's prefix
        dict(name="read_131072", kind="read", tokens=131072, kv_heads=8, dim=128, group=64, page=64,
             dtype="bf16"),
        # ---- attention, one new token for each sequence
        # one user, short context: latency
        dict(name="decode_1x500", kind="attn", seqs=1, q=1, length=500, ragged=False, heads=32,
             kv_heads=8, dim=128, group=64, page=64, dtype="bf16", window=0, slopes=False),
        # 71 query heads on one key head, odd lengths
        dict(name="decode_7x1999_mqa", kind="attn", seqs=7, q=1, length=1999, ragged=True, heads=71,
             kv_heads=1, dim=64, group=32, page=32, dtype="f16", window=0, slopes=False),
        # a serving batch of uneven lengths at the 14848-wide layer: 232 query heads on 8 key heads
        dict(name="decode_64x8192", kind="attn", seqs=64, q=1, length=8192, ragged=True, heads=232,
             kv_heads=8, dim=64, group=64, page=64, dtype="bf16", window=0, slopes=False),
        # two users with very long contexts, whole cache read once
        dict(name="decode_2x262144", kind="attn", seqs=2, q=1, length=262144, ragged=False, heads=32,
             kv_heads=8, dim=128, group=128, page=128, dtype="bf16", window=0, slopes=False),
        # ---- attention of a chunk of a prompt over everything before it and itself
        # uneven fp32 chunks with a window and position slopes, at a padded head size
        dict(name="chunk_5x211_f32", kind="attn", seqs=5, q=211, length=1501, ragged=True, heads=20,
             kv_heads=20, dim=80, group=32, page=32, dtype="f32", window=700, slopes=True),
        # a chunk of 2048 tokens at the end of 16384, a key head for each query head: bound by its products
        dict(name="chunk_2048_of_16384", kind="attn", seqs=1, q=2048, length=16384, ragged=False,
             heads=32, kv_heads=32, dim=128, group=128, page=64, dtype="bf16", window=0, slopes=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "read", "decode", "decode", "chunk", "chunk"])
    dim = rng.choice([40, 64, 64, 80, 96, 104, 128, 128, 128, 160, 192, 256])
    case = dict(kind=kind, dim=dim, group=rng.choice([32, 64, 128]), page=rng.choice([32, 64, 96, 128, 256]),
                dtype=rng.choice(["f32", "f16", "bf16", "bf16"]))
    if kind == "store":
        seqs, kv = rng.choice([1, 1, 2, 5, 16, 64]), rng.choice([1, 2, 5, 8, 12, 32])
        most = 2 ** 26 // (seqs * kv * dim)
        return dict(case, seqs=seqs, tokens=_log(rng, 1, min(8192, most)), kv_heads=kv, start=rng.randrange(0, 3000))
    if kind == "read":
        kv = rng.choice([1, 2, 5, 8, 12, 32])
        return dict(case, tokens=_log(rng, 1, min(131072, 2 ** 26 // (kv * dim))), kv_heads=kv)
    kv = rng.choice([1, 2, 4, 5, 8, 16, 32])
    per = rng.choice([1, 1, 2, 4, 7, 8, 16, 29, 71])
    while per * kv > 256:
        per = rng.choice([1, 2, 4, 7, 8])
    case.update(kind="attn", heads=per * kv, kv_heads=kv, ragged=rng.random() < 0.5,
                window=rng.choice([0, 0, 0, rng.randrange(1, 2000)]), slopes=rng.random() < 0.25)
    if kind == "decode":
        seqs = _log(rng, 1, 64)
        length = _log(rng, 1, min(262144, max(64, 2 ** 28 // (seqs * kv * dim), 64)))
        length = min(length, max(1, 2 ** 29 // (seqs * per * kv)))
        return dict(case, seqs=seqs, q=rng.choice([1, 1, 1, 2, 4]), length=length)
    seqs = rng.choice([1, 1, 1, 2, 3, 6])
    q = _log(rng, 2, 4096 // seqs)
    most = min(2 ** 28 // (seqs * kv * dim), 2 ** 29 // (seqs * q * per * kv))
    return dict(case, seqs=seqs, q=q, length=max(1, min(int(q * rng.uniform(0.8, 8.0)) + rng.randrange(0, 500), most)))


# ---------------------------------------------------------------- the cache's layout
def _sizes(dim, group):
    dp = next(d for d in (64, 96, 128, 192, 256) if d >= dim)
    ng = -(-dp // group)
    return dp, ng, 32 * (dp + 8 * ng)


def _quantize(x, dp, group):
    """x (..., dim) -> codes int32 (..., dp) and words int32 (..., NG)."""
    ng = -(-dp // group)
    x = torch.nn.functional.pad(x.float(), (0, ng * group - x.shape[-1]))
    x = x.view(*x.shape[:-1], ng, group)
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    bits = ((hi - lo) / 15.0).clamp(min=TINY).view(torch.int32)
    bits = (bits + 8) & ~15
    inv = 1.0 / bits.view(torch.float32)
    z = torch.round(-lo * inv).clamp(0, 15)
    n = (torch.round(x * inv[..., None]) + z[..., None]).clamp(0, 15).int()
    return n.flatten(-2)[..., :dp], bits | z.int()


def _key_bytes(n):
    """Codes (..., dp) -> key rows (..., dp / 2) bytes in the record's order."""
    nc = n.shape[-1] // 32
    n = n.view(*n.shape[:-1], nc, 4, 4, 2)          # c, j, byte, nibble
    b = (n[..., 0] | (n[..., 1] << 4)).to(torch.uint8)
    return b.transpose(-3, -2).flatten(-3)


def _value_halves(n):
    """Codes (..., dp) -> (..., dp / 4) half-words (int16)."""
    n = n.view(*n.shape[:-1], n.shape[-1] // 4, 4)
    h = n[..., 0] | (n[..., 1] << 4) | (n[..., 2] << 8) | (n[..., 3] << 12)
    return h.to(torch.int16)


def _put(pages, slots, k, v, group):
    """Quantizes k, v (tokens, heads, dim) into the slots of the pages."""
    dim, heads = k.shape[-1], k.shape[1]
    dp, ng, rec = _sizes(dim, group)
    at, t = slots // 32, slots % 32
    per = pages.shape[2]
    page, r = at // per, at % per
    h = torch.arange(heads, device=slots.device)
    base = ((page[:, None] * heads + h) * per + r[:, None])      # record of (token, head)
    flat = pages.view(-1, rec)
    kn, kw = _quantize(k, dp, group)
    vn, vw = _quantize(v, dp, group)
    rows = flat[:, :16 * dp].view(-1, 32, dp // 2)
    rows[base, t[:, None]] = _key_bytes(kn)
    o = 16 * dp
    flat[:, o:o + 128 * ng].view(torch.int32).view(-1, ng, 32)[base, :, t[:, None]] = kw
    o += 128 * ng
    flat[:, o:o + 16 * dp].view(torch.int16).view(-1, dp // 4, 32)[base, :, t[:, None]] = _value_halves(vn)
    o += 16 * dp
    flat[:, o:].view(torch.int32).view(-1, ng, 32)[base, :, t[:, None]] = vw


def _grid(n, words, group):
    """Codes (..., dp) uint8 and words (..., NG) int32 -> s (n - z) in fp32."""
    dp, ng = n.shape[-1], words.shape[-1]
    s, z = (words & ~15).view(torch.float32), (words & 15).float()
    if ng == 1:
        return (n.float() - z) * s
    sub = dp if dp % group else group          # (a last group of half the size: repeat, then cut)
    if sub == group:
        n = n.view(*n.shape[:-1], ng, group)
        return ((n.float() - z[..., None]) * s[..., None]).flatten(-2)
    s, z = s.repeat_interleave(group, -1)[..., :dp], z.repeat_interleave(group, -1)[..., :dp]
    return (n.float() - z) * s


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1)


def _unpack(rec, dim, group):
    """Records (..., bytes) -> keys and values (..., 32, dim) in fp32."""
    dp, ng, _ = _sizes(dim, group)
    o = 16 * dp
    kn = _nibbles(rec[..., :o].unflatten(-1, (32, 4, dp // 32, 4)))            # token, j, c, byte, nibble
    kn = kn.transpose(-4, -3).flatten(-4)
    kw = rec[..., o:o + 128 * ng].contiguous().view(torch.int32).unflatten(-1, (ng, 32)).transpose(-1, -2)
    o += 128 * ng
    vn = _nibbles(rec[..., o:o + 16 * dp].unflatten(-1, (dp // 4, 32, 2)))     # unit, token, byte, nibble
    vn = vn.transpose(-4, -3).flatten(-3)
    o += 16 * dp
    vw = rec[..., o:].contiguous().view(torch.int32).unflatten(-1, (ng, 32)).transpose(-1, -2)
    return (_grid(kn, kw.contiguous(), group)[..., :dim], _grid(vn, vw.contiguous(), group)[..., :dim])


def _get(pages, slots, dim, group):
    """Keys and values (tokens, heads, dim), fp32, of the slots."""
    heads, per = pages.shape[1], pages.shape[2]
    dp, ng, rec = _sizes(dim, group)
    at, t = slots // 32, (slots % 32)[:, None]
    base = (at // per)[:, None] * heads + torch.arange(heads, device=slots.device)
    base = base * per + (at % per)[:, None]
    flat = pages.view(-1, rec)
    kn = _nibbles(flat[:, :16 * dp].view(-1, 32, dp // 2)[base, t].unflatten(-1, (4, dp // 32, 4)))
    kn = kn.transpose(-4, -3).flatten(-4)
    o = 16 * dp
    kw = flat[:, o:o + 128 * ng].view(torch.int32).view(-1, ng, 32)[base, :, t]
    o += 128 * ng
    vn = flat[:, o:o + 16 * dp].view(torch.int16).view(-1, dp // 4, 32)[base, :, t]
    vn = _nibbles(vn.contiguous().view(torch.uint8)).flatten(-2)
    o += 16 * dp
    vw = flat[:, o:].view(torch.int32).view(-1, ng, 32)[base, :, t]
    return _grid(kn, kw.contiguous(), group)[..., :dim], _grid(vn, vw.contiguous(), group)[..., :dim]


# ---------------------------------------------------------------- inputs
def _activations(g, tokens, heads, dim, dtype, keys):
    """Keys have a few channels that are much larger than the others and a mean of their own."""
    x = torch.randn(tokens, heads, dim, generator=g, device=DEV)
    if keys:
        size = torch.exp(0.3 * torch.randn(heads, dim, generator=g, device=DEV))
        big = torch.rand(heads, dim, generator=g, device=DEV) < 0.04
        x = (x + torch.randn(heads, dim, generator=g, device=DEV) * 0.5) * torch.where(big, 5.0 * size, size)
    return x.to(dtype)


def _new_pages(num, case):
    rec = _sizes(case["dim"], case["group"])[2]
    return torch.zeros(num, case["kv_heads"], case["page"] // 32, rec, dtype=torch.uint8, device=DEV)


def _table(g, seqs, width, spare):
    """The pages of the sequences, in no order among the pool's."""
    return torch.randperm(seqs * width + spare, generator=g, device=DEV)[:seqs * width].view(seqs, width).int()


def _slots(table, start, tokens, page):
    t = torch.arange(start, start + tokens, device=DEV)
    return (table.long()[:, t // page] * page + t % page).flatten()


def _lengths(case, seed):
    """Cached tokens and new queries of each sequence: between a quarter of the longest and it, between one
    query and all, dealt to the sequences by the seed (their sums are the case's)."""
    seqs, length, q = case["seqs"], case["length"], case["q"]
    if not case["ragged"]:
        return [length] * seqs, [q] * seqs
    part = [1.0 if seqs == 1 else i / (seqs - 1) for i in range(seqs)]
    ls = [max(1, int(length * (0.25 + 0.75 * f))) for f in part]
    qs = [1 + int((q - 1) * f) for f in part]
    rng = random.Random(seed)
    rng.shuffle(ls)
    rng.shuffle(qs)
    return ls, qs


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, dim, kv, page = DTYPES[case["dtype"]], case["dim"], case["kv_heads"], case["page"]
    st = dict(case=case, group=case["group"], dim=dim, dtype=dt)
    if case["kind"] == "store":
        seqs, n = case["seqs"], case["tokens"]
        width = -(-(case["start"] + n) // page)
        # keys and values are slices of a fused projection's output, as a layer hands them over
        both = torch.cat([_activations(g, seqs * n, kv, dim, dt, True), _activations(g, seqs * n, kv, dim, dt, False)], 1)
        table = _table(g, seqs, width, 3)
        st.update(k=both[:, :kv], v=both[:, kv:], pages=_new_pages(seqs * width + 3, case),
                  slots=_slots(table, case["start"], n, page))
        return st
    if case["kind"] == "read":
        n = case["tokens"]
        seqs, most = 1, n
    else:
        ls, qs = _lengths(case, seed)
        seqs, most = case["seqs"], max(ls)
    width = -(-most // page)
    table = _table(g, seqs, width, 2)
    pages = _new_pages(seqs * width + 2, case)
    step = max(1, 2 ** 25 // (seqs * kv * dim))
    for a in range(0, most, step):
        b = min(most, a + step)
        _put(pages, _slots(table, a, b - a, page), _activations(g, seqs * (b - a), kv, dim, dt, True),
             _activations(g, seqs * (b - a), kv, dim, dt, False), case["group"])
    if case["kind"] == "read":
        st.update(pages=pages, slots=_slots(table, 0, n, page))
        return st
    heads = case["heads"]
    start = torch.tensor([0] + qs).cumsum(0).int().to(DEV)
    total = sum(qs)
    st.update(pages=pages, table=table, lengths=torch.tensor(ls, dtype=torch.int32, device=DEV), q_start=start,
              max_q=max(qs), q=_activations(g, total, heads, dim, dt, False) * 0.5, window=case["window"],
              slopes=2.0 ** (-8.0 * torch.arange(1, heads + 1, device=DEV) / heads) if case["slopes"] else None)
    return st


# ---------------------------------------------------------------- one pass
def _attend(st):
    q, table, lengths, start = st["q"], st["table"].long(), st["lengths"], st["q_start"]
    dim, mq = st["dim"], st["max_q"]
    seqs, total, heads = table.shape[0], q.shape[0], q.shape[1]
    kv = st["pages"].shape[1]
    rec = st["pages"][table].transpose(1, 2).flatten(2, 3)                   # seqs, kv, records, bytes
    k, v = (x.flatten(2, 3) for x in _unpack(rec, dim, st["group"]))         # seqs, kv, tokens, dim
    i = torch.arange(mq, device=q.device)
    nq = start[1:] - start[:-1]
    rows = (start[:-1, None] + i).clamp(max=total - 1)
    qs = q[rows.long()].float().view(seqs, mq, kv, heads // kv, dim).transpose(1, 2).flatten(2, 3)
    s = torch.matmul(qs * (1.0 / math.sqrt(dim)), k.transpose(-1, -2)).view(seqs, kv, mq, heads // kv, -1)
    t = torch.arange(s.shape[-1], device=q.device)
    back = (lengths - nq)[:, None, None] + i[:, None] - t                    # how far before the query token t lies
    if st["slopes"] is not None:
        s = s - st["slopes"].view(kv, 1, -1, 1) * back[:, None, :, None, :].float()
    hide = back < 0
    if st["window"]:
        hide = hide | (back >= st["window"])
    s = s.masked_fill_(hide[:, None, :, None, :], -math.inf)
    p = torch.exp_(s.sub_(s.amax(-1, keepdim=True).clamp(min=-3.0e38)))
    o = torch.matmul(p.flatten(2, 3), v) / p.sum(-1).flatten(2, 3).clamp(min=1e-30)[..., None]
    o = o.view(seqs, kv, mq, heads // kv, dim).transpose(1, 2).flatten(2, 3)  # seqs, mq, heads, dim
    at = torch.arange(total, device=q.device)
    b = torch.searchsorted(start[1:].contiguous(), at, right=True)
    return o[b, at - start[b]].to(q.dtype)


def run(st):
    if own:
        return _run_own(st)
    if st["case"]["kind"] == "attn":
        return {"out": _attend(st)}
    if st["case"]["kind"] == "store":
        _put(st["pages"], st["slots"], st["k"], st["v"], st["group"])
    k, v = _get(st["pages"], st["slots"], st["dim"], st["group"])
    return {"k": k.to(st["dtype"]), "v": v.to(st["dtype"])}


def _run_own(st):
    import paper_2309_01885_amd as P
    if st["case"]["kind"] == "attn":
        if "ws" not in st:      # the program keeps its workspace between the calls
            st["ws"] = P.workspace(P.kv_attn_workspace_size(st["q"].shape[0], st["table"].shape[0], st["max_q"],
                                                            st["q"].shape[1], st["pages"].shape[1], st["dim"]), DEV)
        return {"out": P.kv_attn(st["q"], st["pages"], st["table"], st["lengths"], group=st["group"],
                                 q_start=st["q_start"], max_q=st["max_q"], window=st["window"],
                                 slopes=st["slopes"], ws=st["ws"])}
    if st["case"]["kind"] == "store":
        P.kv_write(st["k"], st["v"], st["slots"], st["pages"], group=st["group"])
    k, v = P.kv_read(st["pages"], st["slots"], st["dim"], group=st["group"], dtype=st["dtype"])
    return {"k": k, "v": v}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    dim, kv = case["dim"], case["kv_heads"]
    held = 2 * (dim / 2 + 4 * -(-dim // case["group"]))          # bytes of a token and head in the cache
    if case["kind"] != "attn":
        n = case["tokens"] * case.get("seqs", 1)
        # store: inputs in, cache out and in again, values out; read: cache in, values out
        passes = 2 if case["kind"] == "store" else 1
        return {"bytes": n * kv * passes * (held + 2 * dim * size) + 8.0 * n, "flops": n * kv * 2 * dim * 4.0 * passes}
    seen = pairs = total = 0.0
    for length, q in zip(*_lengths(case, 0)):                    # (ragged lengths: those of seed 0)
        w = case["window"] or length + q
        first = max(0, length - q - w + 1)
        seen += max(0, length - first)
        pairs += sum(max(0, min(length - q + i + 1, w)) for i in range(q))
        total += q
    return {"bytes": seen * kv * held + 2.0 * total * case["heads"] * dim * size,
            "flops": 4.0 * dim * case["heads"] * pairs}


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_grid(x, group):
    """s, n, z of the last axis by the definition (fp32 decides the integers), group by group."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for a in range(0, x.shape[-1], group):
        y = x[..., a:a + group].to(torch.float32)
        zero = torch.zeros_like(y[..., :1])
        both = torch.cat([y, zero], -1)
        lo, hi = both.min(-1, keepdim=True).values, both.max(-1, keepdim=True).values
        s = torch.maximum((hi - lo) / 15, torch.full_like(lo, TINY))
        word = s.view(torch.int32)
        s = (torch.div(word + 8, 16, rounding_mode="floor") * 16).view(torch.float32)
        inv = torch.ones_like(s) / s
        z = torch.clamp(torch.round(-lo * inv), 0, 15)
        n = torch.clamp(torch.round(y * inv) + z, 0, 15)
        out[..., a:a + group] = s.double() * (n.double() - z.double())
    return out


def _exact_cache(pages, page_ids, head, dim, group):
    """Keys and values (tokens, dim) of one head's pages in 64 bits, channel by channel from the layout."""
    dp, ng, rec = _sizes(dim, group)
    r = pages[page_ids, head].reshape(-1, rec)
    k = torch.empty(r.shape[0] * 32, dim, dtype=torch.float64, device=r.device)
    v = torch.empty_like(k)
    row = torch.arange(32, device=r.device)

    def word(off):
        b = [r[:, off + 4 * row + e].long() for e in range(4)]
        w = (b[0] + 256 * b[1] + 65536 * b[2] + 16777216 * b[3])
        z = w % 16
        bits = w - z
        exponent, fraction = bits // 8388608, bits % 8388608
        return torch.ldexp(1.0 + fraction.double() / 8388608.0, (exponent - 127).int()), z.double()

    kw = [word(16 * dp + 128 * a) for a in range(ng)]
    vw = [word(32 * dp + 128 * ng + 128 * a) for a in range(ng)]
    for d in range(dim):
        octet = d // 8
        at = row * (dp // 2) + 4 * ((octet % 4) * (dp // 32) + octet // 4) + d % 8 // 2
        n = (r[:, at].long() // (16 if d % 2 else 1)) % 16
        s, z = kw[d // group]
        k[:, d] = (s * (n.double() - z)).flatten()
        at = 16 * dp + 128 * ng + 64 * (d // 4) + 2 * row + d % 4 // 2
        n = (r[:, at].long() // (16 if d % 2 else 1)) % 16
        s, z = vw[d // group]
        v[:, d] = (s * (n.double() - z)).flatten()
    return k, v


def exact(case, seed):
    st = prepare(case, seed)
    dim, group, page = case["dim"], case["group"], case["page"]
    if case["kind"] == "store":
        return {"k": _exact_grid(st["k"], group), "v": _exact_grid(st["v"], group)}
    pages = st["pages"]
    if case["kind"] == "read":
        ids = st["slots"][::page] // page
        heads = [_exact_cache(pages, ids, h, dim, group) for h in range(case["kv_heads"])]
        n = case["tokens"]
        return {"k": torch.stack([k[:n] for k, _ in heads], 1), "v": torch.stack([v[:n] for _, v in heads], 1)}
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    per = case["heads"] // case["kv_heads"]
    ls, qs = _lengths(case, seed)
    first = 0
    for b, (length, nq) in enumerate(zip(ls, qs)):
        ids = st["table"][b, :-(-length // page)].long()
        for h in range(case["kv_heads"]):
            k, v = (x[:length] for x in _exact_cache(pages, ids, h, dim, group))
            for a in range(0, nq, 256):
                e = min(nq, a + 256)
                where = torch.arange(a, e, device=DEV) + (length - nq)
                token = torch.arange(length, device=DEV)
                see = token[None, :] <= where[:, None]
                if case["window"]:
                    see &= token[None, :] > where[:, None] - case["window"]
                for j in range(per):
                    head = h * per + j
                    x = st["q"][first + a:first + e, head].double() @ k.T / math.sqrt(dim)
                    if st["slopes"] is not None:
                        x = x + st["slopes"][head].double() * (token[None, :] - where[:, None])
                    x = torch.where(see, x, -math.inf)
                    top = x.max(-1, keepdim=True).values
                    p = torch.where(see, torch.exp(x - torch.where(torch.isinf(top), 0.0, top)), 0.0)
                    mass = p.sum(-1, keepdim=True)
                    out[first + a:first + e, head] = (p @ v) / torch.where(mass > 0, mass, 1.0)
        first += nq
    return {"out": out}
