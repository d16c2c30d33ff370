"""kv_attn_shared behind more than 2^29 tokens, in a table that names one page over and over."""
import numpy as np
import pytest
import torch

from parity import dev, host
from test_gpu_kv_shared import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per,slopes", [(2, False), (2, True), (64, False)])
def test_shared_behind_2_to_29_tokens(qe, per, slopes):
    """512 pages of 2^20 tokens that are all one, of zeros, then a page (shared as well) whose 32 first tokens score 40 above the others
    and have the value 3; 5 tokens of zeros of a sequence's own.  Weight of the zeros: 2^29 + 2^20 of about 32 e^39.5 = 4.5e18,
    2^-32 of it, so that every output is 3 up to the roundings: the value's code (3 = 15 steps of fp32(3 / 15), 2^-20), the
    weight (fp16, 2^-11) and the output (bf16, 2^-8).  Slopes take the tokens' true distance, 2^20, off at 2^-21 each.  lse is right
    within 2^-10: the scores' codes and sums are (2^-19 of 40), and the sum's logarithm."""
    page, dim, width = 1 << 20, 64, 514
    pages = qe.kv_pages(4, 1, dim, 64, page)
    pages.zero_()
    k, v = torch.zeros(32, 1, dim, device="cuda"), torch.full((32, 1, dim), 3.0, device="cuda")
    k[:, 0, 0] = 15.0
    qe.kv_write(k, v, dev(np.arange(32) + page), pages)
    table = np.zeros((2, width), np.int32)
    table[:, 512] = 1
    table[:, 513] = 2, 3
    n = 513 * page + 5
    assert n > 2 ** 29
    q = torch.zeros(2, per, dim, device="cuda", dtype=torch.bfloat16)
    q[:, :, 0] = 8.0
    slope = 2.0 ** -21 if slopes else 0.0
    sl = torch.full((per,), slope, device="cuda") if slopes else None
    want = 40.0 + np.log(np.exp(slope * (512.0 * page + np.arange(32) - (n - 1))).sum())
    args = (q, pages, dev(table), i32([n, n]))
    need = qe.kv_attn_shared_workspace_size(2, 2, 1, per, 1, dim, 1)
    for call in (lambda lse: qe.kv_attn(*args, scale=1 / 3, slopes=sl, lse=lse, check=True),
                 lambda lse: qe.kv_attn_shared(*args, i32([0, 2]), i32([513]), scale=1 / 3, slopes=sl, lse=lse, check=True,
                                               ws=qe.workspace(need, "cuda"))):
        lse = torch.zeros(2, per, device="cuda")
        out = call(lse)
        assert np.all(np.abs(host(out.float()) - 3.0) <= 3.0 * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -20))
        assert np.all(np.abs(host(lse) - want) <= 2.0 ** -10)
