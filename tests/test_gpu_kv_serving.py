"""kv_extend, kv_append and attention together, as a serving loop uses them: sequences behind a shared prompt that decode, draft
and go back, in a replayed graph whose inputs change, against the CPU forms of each part (pages, lengths and cache bit for
bit, attention within the bound of test_gpu_kv.py's head)."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from parity import dev, host
from test_gpu_kv import DT, bits, check, draw, f64, rounded
from test_gpu_kv_shared import listed  # noqa: F401
from test_gpu_kv_step import tables

pytestmark = pytest.mark.gpu

HEADS, KV, DIM, GROUP, PAGE, PREFIX = 8, 2, 64, 64, 32, 3


def i32(x):
    return dev(np.asarray(x, np.int32))


class Server:
    """Five sequences whose first three pages are one prompt; the CPU's copy of everything beside the GPU's."""

    def __init__(self, qe, dtype, attend):
        self.qe, self.dtype, self.attend = qe, dtype, attend
        r = np.random.default_rng(1)
        num, width = 40, 9
        order = r.permutation(num).astype(np.int32)
        self.table = np.full((5, width), -1, np.int32)
        self.table[:, :PREFIX] = order[:PREFIX]
        self.free = np.full(num, -1, np.int32)
        self.free[:num - PREFIX] = order[PREFIX:]
        self.free_count = num - PREFIX
        self.lengths = np.full(5, PREFIX * PAGE, np.int32)
        self.keep = np.full(5, PREFIX, np.int32)
        self.cos, self.sin = tables(400, DIM)
        self.w = [np.exp(0.2 * r.standard_normal(DIM)).astype(np.float32) for _ in range(2)]
        self.pages = qe.kv_pages(num, KV, DIM, GROUP, PAGE)
        self.want = host(self.pages)
        self.d = {n: dev(getattr(self, n)) for n in ("table", "free", "lengths", "keep", "cos", "sin")}
        self.d.update(free_count=i32([self.free_count]), qw=dev(self.w[0]), kw=dev(self.w[1]))
        t = np.arange(PREFIX * PAGE)
        slots = self.table[0][t // PAGE].astype(np.int64) * PAGE + t % PAGE
        q, k, v = (draw((t.size, h, DIM), 90 + h, dtype) for h in (HEADS, KV, KV + 1))
        self.append(q.cuda(), k.cuda(), v[:, :KV].cuda(), dev(slots), i32(t))
        self.write(k, v[:, :KV], slots, t)
        self.ws = {}

    def append(self, q, k, v, slots, positions):
        d = self.d
        return self.qe.kv_append(q, k, v, slots, self.pages, group=GROUP, positions=positions, cos=d["cos"], sin=d["sin"], q_weight=d["qw"],
                                 k_weight=d["kw"])

    def write(self, k, v, slots, positions):
        okv.write(self.want, np.where(positions < 0, -1, slots), self.turn(k, self.w[1], positions), f64(v), GROUP)

    def turn(self, x, w, positions):
        return okv.norm_rotate(f64(x), w, 1e-6, positions, self.cos, self.sin, False)

    def step(self, counts, q, k, v, max_q):
        """The three calls."""
        total, d = q.shape[0], self.d
        if not self.ws:
            self.ws = dict(step=self.qe.workspace(self.qe.kv_extend_workspace_size(5), "cuda"),
                           attn=self.qe.workspace(self.qe.kv_attn_shared_workspace_size(total, 5, max_q, HEADS, KV, DIM, 1), "cuda"))
        slots, positions, start = self.qe.kv_extend(counts, d["table"], d["lengths"], d["free"], d["free_count"], PAGE, total, keep=d["keep"],
                                                    ws=self.ws["step"])
        turned = self.append(q, k, v, slots, positions)
        return turned, self.attend(self, turned, start, max_q), positions

    def verify(self, counts, q, k, v, got, window=0, sinks=0):
        turned, out, positions = got
        slots, pos, start, self.free_count, lacking, bad = okv.extend(counts, self.table, self.lengths, self.free, self.free_count, PAGE,
                                                                      q.shape[0], self.keep)
        assert not bad and not lacking
        for n in ("table", "lengths", "free"):
            assert np.array_equal(host(self.d[n]), getattr(self, n)), n
        assert np.array_equal(host(positions), pos)
        self.write(k.cpu(), v.cpu(), slots, pos)
        assert np.array_equal(host(self.pages), self.want)
        there = torch.from_numpy(pos >= 0)
        assert np.array_equal(bits(turned.cpu()[there]), bits(rounded(self.turn(q.cpu(), self.w[0], pos), self.dtype)[there]))
        held, nqs = [], []
        for b, n in enumerate(self.lengths):
            t = np.arange(n)
            at = dev(self.table[b][t // PAGE].astype(np.int64) * PAGE + t % PAGE)
            held.append(tuple(f64(x) for x in self.qe.kv_read(self.pages, at, DIM, group=GROUP)))
            nqs.append(int(start[b + 1] - start[b]))
        assert self.qe.sync_status(self.ws["step"]) == 0 and self.qe.sync_status(self.ws["attn"]) == 0
        check(out, None, turned, held, nqs, DIM ** -0.5, self.dtype, window=window, sinks=sinks)


def over_shared(s, q, start, max_q):
    return s.qe.kv_attn_shared(q, s.pages, s.d["table"], s.d["lengths"], s.groups, s.shared, group=GROUP, q_start=start, max_q=max_q,
                               ws=s.ws["attn"])


def over_window(s, q, start, max_q):
    return s.qe.kv_attn(q, s.pages, s.d["table"], s.d["lengths"], group=GROUP, q_start=start, max_q=max_q, window=50, sinks=10, ws=s.ws["attn"])


def rows(total, seed, dtype):
    q, k, v = (draw((total, h, DIM), seed + h, dtype).cuda() for h in (HEADS, KV, KV + 1))
    return q, k, v[:, :KV]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("how", ["shared", "window"])
def test_serving_loop(listed, how, dtype):  # noqa: F811
    s = Server(listed, dtype, over_shared if how == "shared" else over_window)
    s.groups, s.shared = i32([0, 5]), i32([PREFIX])
    masks = {} if how == "shared" else dict(window=50, sinks=10)
    # prompts of their own behind the shared one, one sequence without; rows that are padding
    counts = [5, 40, 1, 0, 33]
    q, k, v = rows(82, 10, dtype)
    s.verify(counts, q, k, v, s.step(i32(counts), q, k, v, 40), **masks)
    # decoding, drafts of up to four tokens and their undoing, from one graph
    s.ws, static, inputs = {}, i32([0] * 5), rows(12, 20, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(static, *inputs, 4)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = s.step(static, *inputs, 4)
    for n, counts in enumerate([[1, 1, 1, 1, 1], [4, 1, 0, 4, 3], [-3, 1, 1, -4, 0], [1, -42, 4, 2, -1], [0, 1, 0, 0, -30], [4, 1, 1, 1, 4]]):
        static.copy_(i32(counts))
        fresh = rows(12, 100 + 10 * n, dtype)
        for a, b in zip(inputs, fresh):
            a.copy_(b)
        graph.replay()
        s.verify(counts, *fresh, got, **masks)
        torch.cuda.synchronize()
