"""The decoding loop's token-level coupling: the drafted tokens, both models' logits and the random numbers that it hands to
pps_verify_chain are those of the text, and what it says follows from them."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_21858_gb300 import decode
from paper_2609_21858_gb300.decode import Decoder, Session
from test_gpu_chain import _check
from test_gpu_decode import plain

pytestmark = pytest.mark.gpu


def near(got, want, tol):
    """Rows of logits, by the norm of their differences."""
    err = (got.double() - want).norm(dim=-1) / want.norm(dim=-1)
    assert err.max().item() < tol, err.tolist()


@pytest.mark.parametrize("gamma,temperature", [(1, 1.0), (4, 0.7), (5, 1.3)])
def test_every_step(gamma, temperature, monkeypatch):
    layers, V, n_seq = 2, 640, 4
    m = Decoder(V, 128, layers, 4, 2, 64, max_pos=512, seed=5)
    s = Session(m, (1,) * gamma, n_seq, 220, key=13, temperature=temperature, page_size=8)
    rng = np.random.default_rng(1)
    s.prefill([rng.integers(0, V, k).tolist() for k in (1, 3, 20, 70)])
    seen = []
    verify = decode.pps.verify_chain

    def spy(*args, status=None):
        got = verify(*args, status=status)
        seen.append((args, got))
        return got

    monkeypatch.setattr(decode.pps, "verify_chain", spy)
    drawn, skipped, accepted = [], 0, 0
    for _ in range(6):
        before = s.tokens()
        v = s.step(coupling=True)
        (p, q, g, off, rows, tok, u, noise, T), got = seen[-1]
        assert g == gamma and T == temperature and got is v and off.numel() == n_seq + 1
        assert bool(((u >= 0) & (u < 1)).all()) and bool((noise[:, :V] > 0).all())
        drawn += [u.clone(), noise.clone()]
        _check(p, q, g, off, rows, tok, u, noise, T=T, got=got, exempt=1)
        for i in range(n_seq):
            nodes = range(int(off[i]), int(off[i + 1]))
            assert len(nodes) == gamma + 1 and int(rows[nodes[-1]]) == -1
            row = rows[nodes[0]:nodes[-1]].long()
            drafted = tok[row].tolist()
            text = before[i] + drafted
            at = torch.arange(len(before[i]) - 1, len(text), device=s.device)  # the node's tokens
            # The target: each stage of a layer rounds to bf16, 2^-8 of its value at most: eight of them per layer and as
            # many in what fed them.  Logits of another context differ by their own size.
            near(p[nodes[0]:nodes[-1] + 1], plain(m, text)[1][at], 8 * (layers + 1) * 2.0 ** -8)
            # the drafter: the head on the token's normed embedding, which is rounded twice at most
            x = m.embed[torch.tensor(text, device=s.device)[at[:-1]].long()].double()
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
            near(q[row], x @ m.head.double().T, 2 * 2.0 ** -8)
            # the drafted tokens are the keyed race's on the drafter's law
            key = np.full(gamma, int(s.key[i]), np.uint64)
            win, _, _, margin = oracle.target_rows((q[row].double() / T).float().cpu().numpy(), key, np.zeros(gamma, np.uint64),
                                                   (at[:-1] + 1).cpu().numpy().astype(np.uint32))
            assert np.all((win == np.array(drafted)) | (margin < 1e-5))
            n = int(got["accept_len"][i])
            assert got["emitted"][i].tolist()[:n] == drafted[:n] and int(got["n_emitted"][i]) == n + 1
            accepted += n
        after = s.tokens()
        for i in range(n_seq):
            n = int(got["n_emitted"][i])
            assert after[i] == before[i] + got["emitted"][i].tolist()[:n]
    assert accepted > 0
    # other random numbers in every step
    for a in range(0, len(drawn), 2):
        for b in range(a + 2, len(drawn), 2):
            assert not torch.equal(drawn[a], drawn[b]) and not torch.equal(drawn[a + 1], drawn[b + 1])
