"""pps_verify_chain whose sequences all lie outside the nodes: what the stream runs next finds the call at its end."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_chain import BF, _cuda  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_seq", [1, 5, 64])
@pytest.mark.parametrize("named", [False, True])
def test_the_workspace_is_free_after_a_call_of_bad_sequences(n_seq, named):
    """Enough rows that their sums take long beside a grid that has nothing to do."""
    n, n_draft, V, gamma = 400, 350, 128256, 5
    p, q = (torch.zeros(r, V, dtype=BF, device="cuda") for r in (n, n_draft))
    i32 = dict(dtype=torch.int32, device="cuda")
    off = torch.full((n_seq + 1,), n + 1, **i32)  # each sequence begins past the nodes
    rows, tok, u = torch.full((n,), -1, **i32), torch.zeros(n_draft, **i32), torch.zeros(n_draft, device="cuda")
    noise = torch.ones(n_seq, V, device="cuda")
    ws = pps.chain_workspace(n, n_draft, n_seq)
    kw = dict(stream=torch.cuda.current_stream()) if named else {}
    for _ in range(5):
        status = torch.zeros(1, **i32)
        torch.cuda.synchronize()
        got = pps.verify_chain(p, q, gamma, off, rows, tok, u, noise, ws=ws, status=status, **kw)
        ws.fill_(0xab)
        torch.cuda.synchronize()
        assert bool((ws == 0xab).all())
        assert int(status) == pps.FLAG_INDEX
        assert not bool(got["accept_len"].any()) and not bool(got["n_emitted"].any()) and bool((got["emitted"] == -1).all())
        # the call's own scratch goes back to the allocator with the call
        size = ws.numel()
        pps.verify_chain(p, q, gamma, off, rows, tok, u, noise, **kw)
        block = torch.full((size,), 0xcd, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert bool((block == 0xcd).all())
        del block
