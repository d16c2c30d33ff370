"""Calls on a stream that is not torch's current one, with buffers that the call makes: the results are
those of a call on the current stream, also where that one is behind."""
import numpy as np
import pytest
import torch

from parity import dev
from test_gpu_kv import cache, draw

pytestmark = pytest.mark.gpu


def test_kv_attn_and_read_on_another_stream(qe):
    """Splits along the tokens (sums and statistics go through the workspace), while the current stream is busy and
    takes memory of the same sizes."""
    pages, table, _ = cache(qe, [3000], 2, 128, 64, 64, "bf16", 9)
    q = draw((1, 8, 128), 1, "bf16").cuda()
    T, L = dev(table), dev(np.array([3000], np.int32))
    slots = dev(table[0][np.arange(500) // 64].astype(np.int64) * 64 + np.arange(500) % 64)
    lse = torch.empty((1, 8), device="cuda")
    want = qe.kv_attn(q, pages, T, L, lse=lse, check=True).clone()
    want_lse, (want_k, want_v) = lse.clone(), qe.kv_read(pages, slots, 128)
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        torch.cuda._sleep(2000000)
        lse.record_stream(side)
        out = qe.kv_attn(q, pages, T, L, lse=lse, stream=side)
        k, v = qe.kv_read(pages, slots, 128, stream=side)
        size = qe.kv_attn_workspace_size(1, 1, 1, 8, 2, 128)
        for _ in range(4):
            torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        side.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert torch.equal(k, want_k) and torch.equal(v, want_v)
        out = qe.kv_attn(q, pages, T, L, stream=side, check=True)
        assert torch.equal(out, want)


def test_quantizer_calls_on_another_stream(qe):
    g = torch.Generator(device="cuda").manual_seed(3)
    W = torch.randn(96, 160, device="cuda", generator=g)
    X = torch.randn(160, 1024, device="cuda", generator=g)

    def calls(stream):
        S = qe.gram(X, damp=0.01, stream=stream)
        scale, zero = qe.grid_minmax(W, 4, stream=stream)
        top = qe.topk_abs(W, 50, stream=stream)
        cols = qe.topk_columns(W, 3, stream=stream)
        csr = qe.outliers_csr(top[0], top[1], top[2], stream=stream)
        obj = qe.objective(W, top[0], S, stream=stream)
        lam = torch.tensor(qe.lambda_max(S, stream=stream))
        return [S, scale, zero, *top, *cols, *csr, obj, lam]

    want = [t.clone() for t in calls(None)]
    side = torch.cuda.Stream()
    for _ in range(2):
        torch.cuda.synchronize()
        torch.cuda._sleep(2000000)
        got = calls(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
