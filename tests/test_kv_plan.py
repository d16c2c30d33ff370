"""How many splits along the tokens an attention call over the 4-bit cache takes, as its workspace shows it:
256 bytes of status, then, where it splits, fp32 sums and two statistics for the rows of every unit and split."""
import pytest


@pytest.fixture(scope="module")
def Q():
    import paper_2309_01885_amd.qe as Q
    Q.load()
    return Q


def up(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("batch,splits", [(1, 96), (2, 48), (4, 24), (8, 12), (16, 6), (32, 3), (48, 2), (49, 3), (64, 3), (95, 2),
                                          (96, 1), (200, 1)])
def test_splits_of_single_tokens(Q, batch, splits):
    """8 key heads of 128 with 4 query heads each: a unit a sequence and key head, tiles of 16 rows; 768 workgroups,
    1536 where that would leave long units whole."""
    rows = batch * 8 * splits * 16
    want = 256 + (up(rows * 128 * 4) + up(rows * 2 * 4) if splits > 1 else 0)
    assert Q.kv_attn_workspace_size(batch, batch, 1, 32, 8, 128) == want
