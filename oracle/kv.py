"""The 4-bit key/value cache on the CPU: grid, record layout and attention, plainly.

The grid is decided in fp32, step by step as include/qe.h states it (it decides
integers); attention is in fp64 from the values that the cache stands for.
"""
import numpy as np

F = np.float32
WIDTHS = (64, 96, 128, 192, 256)


def sizes(dim, group):
    """(Dp, groups, bytes of a record)."""
    dp = next(w for w in WIDTHS if w >= dim)
    ng = -(-dp // group)
    return dp, ng, 32 * dp // 2 * 2 + 2 * 32 * 4 * ng


def quantize_group(x):
    """One group (1-D, any float type) -> (codes, scale bits, zero point)."""
    x = np.asarray(x).astype(F)
    with np.errstate(over="ignore", invalid="ignore"):
        lo, hi = min(F(0), x.min()), max(F(0), x.max())
        span = F(hi - lo)
        if not np.all(np.isfinite(x)) or not np.isfinite(span):
            return np.zeros(x.size, np.uint8), np.uint32(0x7fc00000), 0
        s = np.maximum(F(span * F(1 / 15)), F(2.0 ** -126))
        bits = np.uint32((int(s.view(np.uint32)) + 8) // 16 * 16)
        inv = F(F(1) / bits.view(F))
        z = np.clip(np.rint(F(-lo * inv)), 0, 15)
        n = np.clip(np.rint((x * inv).astype(F)) + z, 0, 15)
    return n.astype(np.uint8), bits, int(z)


def quantize(x, group):
    """(..., dim) -> codes (..., Dp), words (..., NG); channels past dim hold 0."""
    x = np.asarray(x)
    dim = x.shape[-1]
    dp, ng, _ = sizes(dim, group)
    padded = np.zeros(x.shape[:-1] + (ng * group,), x.dtype)
    padded[..., :dim] = x
    flat = padded.reshape(-1, ng, group)
    codes = np.zeros((flat.shape[0], ng * group), np.uint8)
    words = np.zeros((flat.shape[0], ng), np.uint32)
    for r in range(flat.shape[0]):
        for g in range(ng):
            n, bits, z = quantize_group(flat[r, g])
            codes[r, g * group:(g + 1) * group] = n
            words[r, g] = bits | np.uint32(z)
    return codes[:, :dp].reshape(x.shape[:-1] + (dp,)), words.reshape(x.shape[:-1] + (ng,))


def values(codes, words, dim, group):
    """s (n - z) in fp32 (one rounding)."""
    s = (words & np.uint32(0xfffffff0)).view(F)
    z = (words & np.uint32(15)).astype(F)
    at = np.arange(dim) // group
    with np.errstate(invalid="ignore"):
        return s[..., at] * (codes[..., :dim].astype(F) - z[..., at])


def put(pages, slot, head, k_codes, k_words, v_codes, v_words, group):
    """Writes one token of one head; pages: uint8 (pages, heads, page / 32, record)."""
    dp, ng = k_codes.size, k_words.size
    per = pages.shape[2]
    rec = pages[slot // (32 * per), head, slot // 32 % per]
    t = slot % 32
    nc = dp // 32
    vals = 16 * dp + 128 * ng
    for d in range(0, dp, 2):
        octet, byte = d // 8, d % 8 // 2
        rec[t * dp // 2 + 4 * (octet % 4 * nc + octet // 4) + byte] = k_codes[d] | k_codes[d + 1] << 4
        rec[vals + 64 * (d // 4) + 2 * t + d % 4 // 2] = v_codes[d] | v_codes[d + 1] << 4
    for g in range(ng):
        a = 16 * dp + 4 * (32 * g + t)
        rec[a:a + 4] = np.array([k_words[g]], "<u4").view(np.uint8)
        a = vals + 16 * dp + 4 * (32 * g + t)
        rec[a:a + 4] = np.array([v_words[g]], "<u4").view(np.uint8)


def write(pages, slots, k, v, group):
    """In place: tokens x heads x dim into the slots (negative or past the end: skipped)."""
    limit = pages.shape[0] * pages.shape[2] * 32
    kc, kw = quantize(k, group)
    vc, vw = quantize(v, group)
    for t, slot in enumerate(slots):
        if 0 <= slot < limit:
            for h in range(k.shape[1]):
                put(pages, int(slot), h, kc[t, h], kw[t, h], vc[t, h], vw[t, h], group)


def attention(q, k, v, pos, scale, causal=True, window=0, slopes=None, sinks=0):
    """q (nq, heads, dim) at positions pos over k, v (tokens, kv heads, dim), all in fp64:
    (out, lse, mass) with mass = sum_t p_t |v_t|, what an error of the p_t acts on."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    nq, heads, dim = q.shape
    per = heads // k.shape[1]
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((nq, heads), -np.inf)
    t = np.arange(k.shape[0])
    for h in range(heads):
        kh, vh = k[:, h // per], v[:, h // per]
        for i in range(nq):
            see = np.ones(t.size, bool)
            if causal:
                see &= t <= pos[i]
            if window:
                see &= (t > pos[i] - window) | (t < sinks)
            if not see.any():
                continue
            s = scale * (kh[see] @ q[i, h])
            if slopes is not None:
                s = s + float(slopes[h]) * (t[see] - pos[i])
            top = s.max()
            p = np.exp(s - top)
            total = p.sum()
            out[i, h] = p @ vh[see] / total
            mass[i, h] = p @ np.abs(vh[see]) / total
            lse[i, h] = top + np.log(total)
    return out, lse, mass


def extend(counts, table, lengths, free, free_count, page, total, keep=None):
    """A step's pages and slots, sequence by sequence and token by token; in place on table, lengths and free.
    Returns (slots, positions, q_start, free_count, lacking, bad)."""
    width, num, batch = table.shape[1], free.size, len(counts)
    keep = [0] * batch if keep is None else keep
    bad = not 0 <= free_count <= num
    free_count = min(max(free_count, 0), num)
    plan = []
    for b in range(batch):
        old, k = int(lengths[b]), int(keep[b])
        new = max(old + int(counts[b]), 0)
        wrong = old < 0 or old > width * page or k < 0 or k > width or new > min(width * page, 2 ** 31 - 1)
        held, want = (0, 0) if wrong else (max(-(-old // page), k), max(-(-new // page), k))
        plan.append((old, old if wrong else new, held, want, wrong))
        bad |= wrong
    back = [(b, j) for b, (_, _, held, want, _) in enumerate(plan) for j in range(want, held)]
    top = free_count + len(back)
    for r, (b, j) in enumerate(back):
        if top - 1 - r < num:
            free[top - 1 - r] = table[b, j]
        table[b, j] = -1
    have = min(top, num)
    bad |= top > num
    slots, positions = np.full(total, -1, np.int64), np.full(total, -1, np.int32)
    q_start = np.zeros(batch + 1, np.int32)
    needed = taken = row = 0
    for b, (old, new, held, want, wrong) in enumerate(plan):
        n, need = max(int(counts[b]), 0), max(want - held, 0)
        needed += need
        got = not wrong and (need == 0 or needed <= have) and (n == 0 or row + n <= total)
        if got:
            for j in range(need):
                at = top - 1 - (needed - need + j)
                table[b, held + j] = free[at] if at < num else -1
            taken = max(taken, needed if need else 0)
            lengths[b] = new
        for i in range(0 if wrong else max(0, min(n, total - row))):
            positions[row + i] = old + i
            if got:
                p = int(table[b, (old + i) // page])
                if 0 <= p < num:
                    slots[row + i] = p * page + (old + i) % page
                else:
                    bad = True
        row += n
        q_start[b + 1] = min(row, total)
    bad |= row > total
    return slots, positions, q_start, have - taken, max(needed - have, 0), bad


def norm_rotate(x, weight, eps, positions, cos, sin, interleaved):
    """(tokens, heads, dim) of any float type -> fp32: every step one fp32 rounding, the sum of squares in fp64."""
    y = np.asarray(x).astype(F)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if weight is not None:
            d = y.astype(np.float64)
            r = (1.0 / np.sqrt((d * d).sum(-1, keepdims=True) / y.shape[-1] + eps)).astype(F)
            y = (y * r).astype(F) * weight.astype(F)
        if cos is None:
            return y
        c, s = (t[np.maximum(positions, 0)][:, None] for t in (cos, sin))
        half = cos.shape[1]
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        z = y.copy()
        z[..., a] = y[..., a] * c - y[..., b] * s
        z[..., b] = y[..., b] * c + y[..., a] * s
    return z
