"""The decoding loop's status word (no GPU): every call of a step that can raise flags is given it."""
import pytest
import torch

from paper_2609_21858_gb300 import decode
from test_decode import session


@pytest.mark.parametrize("branching", [(2, 3), (1, 1, 1)])
def test_draft_lists_raise_their_flags(branching, monkeypatch):
    s, rows = session(branching), []

    def lists(x, weight, key, ctx, pos, K, status=None, **kw):
        assert status is s.status
        rows.append(x.shape[0])
        return dict(tok=torch.ones(x.shape[0], K, dtype=torch.int32), ndist=torch.ones(x.shape[0], dtype=torch.int32))

    monkeypatch.setattr(decode.pps, "lmhead_draft_list", lists)
    s._draft()
    assert rows == [3 * (hi - lo) for lo, hi in s.levels]
