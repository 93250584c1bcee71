"""pps_verify_chain at temperatures near the ends of fp32: a law of one token, and a uniform one."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_chain import BF, F32, _chains, _check, _cuda  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [1, 9, 4096, 30001])
@pytest.mark.parametrize("T", [1e-45, 1e-39, 4e-39, 1e-30, 1e-5])
def test_the_largest_logit_is_the_law(dt, V, T):
    p, q, gamma, off, rows, tok, u, noise = _chains([3, 0, 2], V, dt, V, permute=False)
    for x in (p, q):  # one largest logit a row (bf16 has ties)
        i = torch.randint(0, V, (x.shape[0], 1), device="cuda")
        x.scatter_(1, i, 40.0)
    q[0] = p[0]  # a draft that is accepted
    best, drafted = p.argmax(-1), q.argmax(-1).int()
    for got in (pps.verify_chain(p, q, gamma, off, rows, drafted, u, noise, temperature=T),
                pps.verify_chain(p, q, gamma, off, rows, drafted, u, noise, temperature=T, stream=torch.cuda.current_stream())):
        for s, a, b in ((0, 0, 4), (1, 4, 5), (2, 5, 8)):
            said = []
            for c in range(a, b):
                said.append(int(best[c]))
                r = int(rows[c])
                if r < 0 or int(drafted[r]) != said[-1]:
                    break
            assert got["emitted"][s].tolist() == said + [-1] * (gamma + 1 - len(said)), (s, T)
            assert int(got["accept_len"][s]) == len(said) - 1 and int(got["n_emitted"][s]) == len(said)
        same = drafted == best[torch.tensor([0, 1, 2, 5, 6], device="cuda")].int()
        assert torch.equal(got["accept_prob"], same.float())


@pytest.mark.parametrize("dt", [BF, F32])
def test_a_uniform_law(dt):
    args = _chains([3, 0, 2], 500, dt, 11)
    _check(*args, T=3e38, exempt=1)
