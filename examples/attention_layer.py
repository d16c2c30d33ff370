"""A quantized attention layer served from a 4-bit key/value cache.

    python examples/attention_layer.py [--hidden 4096 --heads 32 --kv-heads 8 --steps 16]

The layer's projection is quantized to 4 bits on calibration activations (gram, grid_minmax,
cd_sweep).  Prompts of different lengths are then read in chunks: their tokens get pages and slots
(kv_extend), queries and keys are rotated by their positions on the way into the cache (kv_append)
and attend to what it holds (kv_attn with q_start).  Every sequence goes on a token at a
time, all three calls recorded once as a HIP graph and replayed.  Prints what the cache holds per token and how far
the layer's outputs lie from those of an unquantized cache and of the unquantized layer.  Weights
and activations are synthetic.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2309_01885_amd as P  # noqa: E402


def quantize_weight(W, X, bits=4, sweeps=5):
    """W (outputs x inputs, fp32) on the grid that QuantEase finds for activations X (inputs x tokens)."""
    Sigma = P.gram(X, damp=0.01)
    scale, zero = P.grid_minmax(W, bits)
    W_hat, R = torch.empty_like(W), torch.empty_like(W)
    codes = torch.zeros(W.shape, dtype=torch.uint8, device=W.device)
    P.cd_sweep(W, Sigma, bits, scale, zero, W_hat, codes, R, sweeps)
    return W_hat


class PagedCache:
    """Sequences of one layer in fixed-size pages of a pool, taken on the GPU as the sequences grow."""

    def __init__(self, sequences, max_len, kv_heads, dim, group=64, page=64):
        width = -(-max_len // page)
        self.pages = P.kv_pages(sequences * width, kv_heads, dim, group, page)
        self.free = torch.randperm(sequences * width, device="cuda").int()
        self.free_count = torch.full((1,), sequences * width, dtype=torch.int32, device="cuda")
        self.table = torch.full((sequences, width), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.lacking = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = P.workspace(P.kv_extend_workspace_size(sequences), "cuda")
        self.group, self.page = group, page

    def extend(self, counts, total):
        """Pages for counts[b] (int32, device) more tokens of sequence b: slots, positions and q_start of the `total` tokens."""
        return P.kv_extend(counts, self.table, self.lengths, self.free, self.free_count, self.page, total, lacking=self.lacking,
                           ws=self.ws)


def rotation(positions, dim):
    """Cosines and sines of the positions' angles (fp32)."""
    turn = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * turn
    return angle.cos().float(), angle.sin().float()


class AttentionLayer:
    def __init__(self, W, heads, kv_heads, dim, dtype, positions):
        self.W, self.heads, self.kv_heads, self.dim = W.to(dtype), heads, kv_heads, dim
        self.cos, self.sin = rotation(positions, dim)

    def project(self, x):
        """Query, keys and values as slices of the fused projection (no copies)."""
        y = (x @ self.W.t()).unflatten(1, (self.heads + 2 * self.kv_heads, self.dim))
        return y.split([self.heads, self.kv_heads, self.kv_heads], dim=1)

    def attend(self, x, cache, counts, max_q, ws=None):
        """Writes the tokens x, counts[b] of sequence b, into the cache and lets them attend to their sequences."""
        slots, positions, q_start = cache.extend(counts, x.shape[0])
        q, k, v = self.project(x)
        q = P.kv_append(q, k, v, slots, cache.pages, group=cache.group, positions=positions, cos=self.cos, sin=self.sin)
        return P.kv_attn(q, cache.pages, cache.table, cache.lengths, group=cache.group, q_start=q_start, max_q=max_q, ws=ws)


def turned(x, cos, sin):
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def plain(layer, xs):
    """The same layer over whole sequences with an unquantized cache, in fp32."""
    outs = []
    for x in xs:
        q, k, v = (t.float() for t in layer.project(x))
        q, k = (turned(t, layer.cos[:x.shape[0], None], layer.sin[:x.shape[0], None]) for t in (q, k))
        k, v = (t.repeat_interleave(layer.heads // layer.kv_heads, dim=1) for t in (k, v))
        n = x.shape[0]
        s = torch.einsum("qhd,thd->hqt", q, k) / layer.dim ** 0.5
        s = s.masked_fill(torch.ones(n, n, device="cuda", dtype=torch.bool).triu(1), -float("inf"))
        outs.append(torch.einsum("hqt,thd->qhd", s.softmax(-1), v))
    return outs


def distance(a, b):
    return float((a.float() - b.float()).norm() / b.float().norm())


def serve(layer, xs, prompts, chunk, group=64, page=64):
    """Outputs of all tokens of xs: prompts[b] of them read in chunks, the others one by one."""
    n_seq, total = len(xs), [x.shape[0] for x in xs]
    cache = PagedCache(n_seq, max(total), layer.kv_heads, layer.dim, group, page)
    outs, held = [[] for _ in xs], [0] * n_seq
    while any(h < p for h, p in zip(held, prompts)):
        counts = [min(chunk, p - h) for h, p in zip(held, prompts)]
        y = layer.attend(torch.cat([x[h:h + c] for x, h, c in zip(xs, held, counts)]), cache,
                         torch.tensor(counts, dtype=torch.int32, device="cuda"), max(counts))
        held = [h + c for h, c in zip(held, counts)]
        for b, part in enumerate(y.split(counts)):
            outs[b].append(part)
    # decoding: the graph reads its tokens and counts from fixed buffers and moves lengths and pages itself
    x_in = torch.stack([x[p] for x, p in zip(xs, prompts)])
    counts = torch.zeros(n_seq, dtype=torch.int32, device="cuda")           # the warm-up adds no token
    ws = P.workspace(P.kv_attn_workspace_size(n_seq, n_seq, 1, layer.heads, layer.kv_heads, layer.dim), "cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.attend(x_in, cache, counts, 1, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.attend(x_in, cache, counts, 1, ws=ws)
    counts.fill_(1)
    for step in range(total[0] - prompts[0]):
        x_in.copy_(torch.stack([x[p + step] for x, p in zip(xs, prompts)]))
        graph.replay()
        for b in range(n_seq):
            outs[b].append(y[b:b + 1].clone())
    if P.sync_status(ws) != P.QE_OK or P.sync_status(cache.ws) != P.QE_OK or int(cache.lacking):
        raise RuntimeError("the cache's page table or lengths are damaged, or its pages used up")
    return [torch.cat(o) for o in outs], cache


def run(hidden=4096, heads=32, kv_heads=8, dim=128, prompts=(300, 1000, 1, 777), steps=16, chunk=256,
        calibration=8192, group=64, page=64, dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    mix = normal(hidden, hidden) / hidden ** 0.5 * torch.exp(0.5 * normal(hidden))
    W = normal((heads + 2 * kv_heads) * dim, hidden) / hidden ** 0.5
    W_hat = quantize_weight(W, (normal(calibration, hidden) @ mix).t().contiguous())
    xs = [(normal(p + steps, hidden) @ mix).to(dtype) for p in prompts]
    longest = max(prompts) + steps
    layer = AttentionLayer(W_hat, heads, kv_heads, dim, dtype, longest)
    got, cache = serve(layer, xs, list(prompts), chunk, group, page)
    kept = plain(layer, xs)
    full = plain(AttentionLayer(W, heads, kv_heads, dim, dtype, longest), xs)
    per_token = P.kv_page_bytes(kv_heads, dim, group, page) / page
    return {"bytes_per_token": per_token, "bytes_per_token_16_bit": 4.0 * kv_heads * dim, "held": cache.lengths.tolist(),
            "cache": [distance(a, b) for a, b in zip(got, kept)],
            "weights": [distance(a, b) for a, b in zip(kept, full)],
            "both": [distance(a, b) for a, b in zip(got, full)]}


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("dim", 128), ("steps", 16), ("chunk", 256),
                        ("group", 64), ("page", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    r = run(**vars(ap.parse_args()))
    print(f"cache: {r['bytes_per_token']:.0f} bytes a token (16-bit: {r['bytes_per_token_16_bit']:.0f})")
    print("relative error of the outputs, per sequence (tokens; 4-bit cache; 4-bit weights; both)")
    for row in zip(r["held"], r["cache"], r["weights"], r["both"]):
        print("  %6d  %.4f  %.4f  %.4f" % row)


if __name__ == "__main__":
    main()
