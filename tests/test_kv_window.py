"""Windows that a C int does not hold reach the library as what they mean.  Without a GPU: the library call is
replaced by a record of its arguments."""
import pytest
import torch

import paper_2309_01885_amd.qe as Q


@pytest.mark.parametrize("window,passed", [(0, 0), (1, 1), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1),
                                           (2 ** 32, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1), (2 ** 40 + 7, 2 ** 31 - 1),
                                           (-1, -1), (-2 ** 31, -2 ** 31), (-2 ** 32, -1), (5 - 2 ** 32, -1)])
def test_windows(monkeypatch, window, passed):
    got = []
    call = Q.SIGNATURES["qe_kv_attn"][1]

    class Lib:
        def qe_kv_attn(self, *args):
            assert call[20] is Q._int
            got.append(Q._int(args[20]).value)
            return 0

        def qe_kv_attn_workspace_size(self, *args):
            return 256

    monkeypatch.setattr(Q, "load", lambda: Lib())
    monkeypatch.setattr(Q, "_pages", lambda pages, dim, group: (4, 64, 2, -1))
    monkeypatch.setattr(Q, "_raw_stream", lambda dev, stream: 0)
    Q.kv_attn(torch.ones((3, 4, 64)), torch.ones((4, 2, 2, 64), dtype=torch.uint8), torch.ones((3, 1), dtype=torch.int32),
              torch.ones(3, dtype=torch.int32), window=window)
    assert got == [passed]
