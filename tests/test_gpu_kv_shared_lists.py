"""kv_attn_shared's lists where the public call takes them by its own rule, and as many groups as they hold.  That a call does take
them shows in its workspace: kv_attn's is refused then."""
import numpy as np
import pytest
import torch

from parity import dev
from test_gpu_kv import DT, check, draw
from test_gpu_kv_shared import attend, family, i32, listed  # noqa: F401

pytestmark = pytest.mark.gpu


def takes_lists(qe, q, pages, table, lens, groups, shared, dim, group, kv, max_q=None, **more):
    """Whether the call refuses kv_attn's workspace."""
    total, batch = q.shape[0], len(lens)
    size = qe.kv_attn_workspace_size(total, batch, max_q or total // batch, q.shape[1], kv, dim)
    try:
        qe.kv_attn_shared(q, pages, table, i32(lens), groups, shared, group=group, max_q=max_q, ws=qe.workspace(size, "cuda"), **more)
    except qe.QEError as e:
        assert e.code == qe.QE_ERR_WORKSPACE
        return True
    return False


# heads, key heads, dim, group, sequences, queries of each, shared tokens, the table's width in tokens.  By the rule at kSaves in
# kv_shared.hip the lists are taken where the saved tiles of 16 rows x key heads x records of the table are 20000 or more: 21 x 4 x 290,
# 12 x 8 x 375 and 13 x 5 x 625 are, 21 x 4 x 125 is not; or where the shared part has the many-row form alone.
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("heads,kv,dim,group,seqs,nq,shared,room,lists",
                         [(8, 4, 64, 64, 24, 1, 8960, 9280, True), (32, 8, 128, 64, 16, 1, 640, 12000, True),
                          (8, 4, 64, 32, 24, 1, 640, 4000, False), (8, 1, 64, 64, 5, 40, 640, 64000, True),
                          (15, 5, 80, 32, 16, 1, 320, 20000, True)])
def test_by_the_calls_own_rule(qe, heads, kv, dim, group, seqs, nq, shared, room, lists, dtype):
    page = 64
    parts = [(shared // page, [shared + 1 + 9 * y for y in range(seqs)])]
    pages, table, lens, held, groups, pages_shared = family(qe, parts, kv, dim, group, page, dtype, seed=1)
    assert table.shape[1] <= room // page
    table = dev(np.pad(table, ((0, 0), (0, room // page - table.shape[1])), constant_values=-1))
    q = draw((seqs * nq, heads, dim), 3, dtype).cuda()
    args = (pages, table, lens, i32(groups), i32(pages_shared))
    assert takes_lists(qe, q, *args, dim, group, kv) == lists
    lse = torch.full((seqs * nq, heads), 5.0, device="cuda")
    out = qe.kv_attn_shared(q, args[0], args[1], i32(lens), *args[3:], group=group, lse=lse, check=True)
    check(out, lse, q, held, [nq] * seqs, dim ** -0.5, dtype)
    for _ in range(2):
        assert torch.equal(qe.kv_attn_shared(q, args[0], args[1], i32(lens), *args[3:], group=group), out)


@pytest.mark.parametrize("pairs,alone", [(300, 723), (0, 1024), (1, 1023), (1024, 0), (500, 524), (512, 0), (0, 512), (1, 511), (500, 525), (1025, 0)])
def test_many_groups(listed, pairs, alone):  # noqa: F811
    """Pairs behind one page, pairs behind two, sequences alone, 512 to 1024 groups of them in the lists (which hold 1024) and
    1025, where the call is kv_attn's; fewer and more sequences than the plan has threads."""
    parts = [(1 + y % 2, [33 + y % 40, 40 + y % 55]) for y in range(pairs)] + [(0, [1 + y % 70]) for y in range(alone)]
    order = np.random.default_rng(1).permutation(len(parts))
    parts = [parts[y] for y in order]
    parts = [(p, [max(n, 32 * p) for n in ls]) for p, ls in parts]
    pages, table, lens, held, groups, shared = family(listed, parts, 1, 64, 64, 32, "f16", seed=6)
    seqs = len(lens)
    q = draw((seqs, 2, 64), 9, "f16").cuda()
    args = (q, pages, dev(table), lens, i32(groups), i32(shared))
    assert takes_lists(listed, *args, 64, 64, 1) == (len(parts) <= 1024)
    out = listed.kv_attn_shared(q, pages, dev(table), i32(lens), *args[4:], check=True)
    check(out, None, q, held, [1] * seqs, 0.125, "f16")
