"""pps_verify_chain's accept_prob: every draft row has a value, 0 where no node of a chain names it."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_chain import BF, F32, _chains, _check, _cuda, _law  # noqa: F401

pytestmark = pytest.mark.gpu


def used(p, dirty):
    """The allocator's free blocks hold `dirty`, so that an output nobody writes shows."""
    blocks = [torch.full((n,), dirty, device="cuda") for n in (4, 64, 128, 256, 512, 1024)]
    del blocks


def both(*args, **kw):
    """Through the extension and through Python, over memory of two kinds."""
    for dirty in (3.25, float("nan")):
        used(args[0], dirty)
        yield pps.verify_chain(*args, **kw)
        used(args[0], dirty)
        yield pps.verify_chain(*args, stream=torch.cuda.current_stream(), **kw)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gamma", [0, 1, 2, 5, 9])
def test_chains_longer_than_gamma(dt, gamma):
    args = list(_chains([5, 0, 3, 7, 1], 700, dt, 3))
    p, q, _, off, rows, tok, u, noise = args
    args[2] = gamma
    named = set()
    for s in range(5):
        for j in range(min(int(off[s + 1] - off[s]) - 1, gamma)):
            named.add(int(rows[int(off[s]) + j]))
    others = torch.tensor([r not in named for r in range(q.shape[0])], device="cuda")
    for got in both(*args):
        _check(*args, got=got)
        assert bool((got["accept_prob"][others] == 0).all())
        assert bool((got["accept_prob"][~others] > 0).all())


def test_rows_of_no_chain():
    p, q, gamma, off, rows, tok, u, noise = _chains([2, 2, 2], 100, BF, 5, permute=False)
    rows = rows.clone()
    rows[3] = -1  # the second chain ends at its root; its second node still names its row
    off = torch.tensor([0, 3, 6, 10], dtype=torch.int32, device="cuda")  # the third sequence lies outside the nodes
    for got in both(p, q, gamma, off, rows, tok, u, noise):
        prob = got["accept_prob"].tolist()
        assert prob[2] == 0 and prob[4:] == [0, 0] and min(prob[0], prob[1], prob[3]) > 0
    out = dict(accept_len=torch.empty(3, dtype=torch.int32, device="cuda"),
               n_emitted=torch.empty(3, dtype=torch.int32, device="cuda"),
               emitted=torch.empty(3, 3, dtype=torch.int32, device="cuda"),
               accept_prob=torch.full((9,), 7.0, device="cuda"))
    pps.verify_chain(p, q, gamma, off, rows, tok, u, noise, out=out)
    assert out["accept_prob"][:6].tolist() == prob and out["accept_prob"][6:].tolist() == [7.0] * 3


def test_more_draft_rows_than_threads():
    """40000 rows of a drafter, of which two chains name three."""
    p, q, gamma, off, rows, tok, u, noise = _chains([2, 1], 64, F32, 7, permute=False)
    big = torch.zeros(40000, 64, device="cuda")
    at = torch.tensor([39999, 0, 20000], device="cuda")
    big[at] = q
    rows = torch.tensor([39999, 0, -1, 20000, -1], dtype=torch.int32, device="cuda")
    toks, us = torch.zeros(40000, dtype=torch.int32, device="cuda"), torch.zeros(40000, device="cuda")
    toks[at], us[at] = tok, u
    args = (p, big, gamma, off, rows, toks, us, noise)
    for got in both(*args):
        _check(*args, got=got)
        assert int((got["accept_prob"] != 0).sum()) == 3


def test_no_sequences():
    p, q, gamma, _, _, tok, u, noise = _chains([2, 1], 64, F32, 9)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    for got in both(p[:0], q, gamma, torch.zeros(1, dtype=torch.int32, device="cuda"), none, tok, u, noise):
        assert got["accept_prob"].tolist() == [0, 0, 0] and got["accept_len"].numel() == 0
