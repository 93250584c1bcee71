"""The decoding loop on the GPU: after speculative steps, the cache holds what a plain pass in 64 bits over the emitted
text gives, and the emitted tokens are that pass's own races."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_21858_gb300 import synth
from paper_2609_21858_gb300.decode import Decoder, Session, main

pytestmark = pytest.mark.gpu


def plain(m, text):
    """Keys and values of every layer [n, kv heads, d] and the logits, in 64 bits, over one whole text."""
    f = lambda x: x.double()
    norm = lambda x: x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    n, hd = len(text), m.head_dim
    x = f(m.embed)[torch.tensor(text, device=m.embed.device).long()]
    c, s = (t[:, None] for t in f(m.rope[:n]).split(hd // 2, dim=1))

    def turn(y, w):
        if w is not None:
            y = norm(y) * f(w)
        a, b = y[..., :hd // 2], y[..., hd // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], dim=-1)

    out = []
    unseen = torch.triu(torch.ones(n, n, dtype=torch.bool, device=x.device), 1)
    for wqkv, wo, (qn, kn) in zip(m.wqkv, m.wo, m.qk):
        q, k, v = (norm(x) @ f(wqkv).T).view(n, -1, hd).split([m.heads, m.kv_heads, m.kv_heads], dim=1)
        q, k = turn(q, qn), turn(k, kn)
        out.append((k, v))
        g = m.heads // m.kv_heads
        score = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(g, 1)) * hd ** -0.5
        w = score.masked_fill(unseen, -torch.inf).softmax(-1)
        x = x + torch.einsum("hij,jhd->ihd", w, v.repeat_interleave(g, 1)).reshape(n, -1) @ f(wo).T
    return out, norm(x) @ f(m.head).T


# Every stage of a layer (norm, projection, rotated key, weights, result, projection, sum) rounds once to bf16, 2^-9 of its
# value at most; eight roundings per layer and as many in what fed them, added up in the worst direction.
def rounding(layers):
    return 8 * (layers + 1) * 2.0 ** -9


@pytest.mark.parametrize("branching,coupling,qk_norm", [((4, 1, 1), False, True), ((2, 2, 2), False, False),
                                                        ((1, 1, 1, 1), False, True), ((1, 1, 1), True, True),
                                                        ((8, 3, 1), False, True)])
def test_cache_and_tokens(branching, coupling, qk_norm):
    layers, V = 2, 640
    m = Decoder(V, 128, layers, 4, 2, 64, max_pos=512, qk_norm=qk_norm, seed=3)
    n_seq = 4
    s = Session(m, branching, n_seq, 220, key=11, page_size=8)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, V, k).tolist() for k in (1, 2, 17, 140)]
    s.prefill(prompts)
    accepted = 0
    for _ in range(8):
        accepted += int(s.step(coupling)["accept_len"].sum())
    texts = s.tokens()
    assert accepted > 0  # some draft went through
    total = agree = 0
    for q, text in enumerate(texts):
        n = len(text) - 1  # the last token is not in the cache
        assert text[:len(prompts[q])] == prompts[q] and n == int(s.length[q]) and n >= len(prompts[q]) - 1 + 8
        assert min(text) >= 0 and max(text) < V
        kv, logits = plain(m, text[:n])
        pos = torch.arange(n, device=s.device)
        slot = s.cache.slots(torch.full_like(pos, q), pos)
        for l, (k, v) in enumerate(kv):
            for mine, want in ((s.cache.k[l], k), (s.cache.v[l], v)):
                got = mine.view(-1, m.kv_heads, m.head_dim)[slot].double()
                err = (got - want).norm(dim=-1) / want.norm(dim=-1)
                assert err.max().item() < rounding(l + 1), (q, l, err.max().item(), err.argmax().item())
        if not coupling:
            # the race of every emitted position on the plain logits: the same token but where the race is close
            at = np.arange(len(prompts[q]) - 1, n)
            key = np.full(at.size, int(s.key[q]), np.uint64)
            win, _, _, margin = oracle.target_rows(logits[at].float().cpu().numpy(), key, np.zeros(at.size, np.uint64),
                                                   (at + 1).astype(np.uint32))
            emitted = np.array(text)[at + 1]
            # logits of order 2: an error of rounding(layers) of their vector's norm, spread over its elements
            close = margin < 4 * 2 * rounding(layers)
            assert np.all((win == emitted) | close)
            total, agree = total + at.size, agree + int((win == emitted).sum())
    if not coupling:
        assert agree >= 0.8 * total, (agree, total)


def test_steps_repeat():
    """The same session twice gives the same bits."""
    def go():
        m = Decoder(500, 64, 2, 4, 1, 16, seed=1)
        s = Session(m, (3, 2), 3, 120, key=5)
        s.prefill([[1, 2, 3], [4], [5, 6]])
        for _ in range(4):
            s.step()
        return s.tokens(), s.cache.k.clone(), s.cache.v.clone()
    (a, k, v), (b, k2, v2) = go(), go()
    assert a == b and torch.equal(k, k2) and torch.equal(v, v2)


def test_command(capsys):
    main(["--steps", "3", "--sequences", "3"])
    main(["--steps", "3", "--sequences", "3", "--branching", "1,1", "--coupling"])
    assert capsys.readouterr().out.count("accepted per step") == 2
