"""kv_attn_shared where the first sequences of a group have no queries: a serving loop's idle place, whose row of the table was
reset, at the front of a group that goes on.  The others' shared pages are read all the same."""
import numpy as np
import pytest
import torch

from parity import dev
from test_gpu_kv import DT, check, draw
from test_gpu_kv_shared import family, i32, listed  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nqs,heads,kv,wide", [([0, 0, 1, 2, 0, 1, 0, 1], 8, 2, 0), ([0, 0, 70, 90, 0, 40, 60, 0], 4, 2, 30000)])
def test_idle_sequences_in_front(listed, nqs, heads, kv, wide, causal, dtype):  # noqa: F811
    """Few rows and many; a group whose first two are idle and one that ends with an idle one."""
    pages, table, lens, held, groups, shared = family(listed, [(4, [128, 130, 300, 290]), (3, [96, 200, 190, 150])], kv, 64, 64, 32, dtype,
                                                      seed=3)
    idle = [b for b, n in enumerate(nqs) if n == 0]
    table[idle] = -1
    table = np.pad(table, ((0, 0), (0, max(0, wide - table.shape[1]))), constant_values=-1)
    for left in (0, 128):                                  # (the idle places' lengths: reset, or as they were)
        lens = [left if b in idle else n for b, n in enumerate(lens)]
        total = sum(nqs)
        q = draw((total, heads, 64), 5, dtype).cuda()
        lse = torch.full((total, heads), 5.0, device="cuda")
        out = listed.kv_attn_shared(q, pages, dev(table), i32(lens), i32(groups), i32(shared), max_q=max(nqs), causal=causal, lse=lse,
                                    q_start=i32(np.concatenate([[0], np.cumsum(nqs)])), check=True)
        check(out, lse, q, held, nqs, 0.125, dtype, causal=causal)
