"""The decoding loop over a cache of 4 bits, over a pool of pages, and with laws on the target's logits: these calls together, as a
server makes them."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_21858_gb300 import pps
from paper_2609_21858_gb300.decode import Decoder, Session, main
from q4_format import held
from test_gpu_decode import plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def run(branching, coupling=False, steps=8, n_seq=4, prompts=None, **kw):
    m = Decoder(640, 128, 2, 4, 2, 64, max_pos=512, seed=3)
    s = Session(m, branching, n_seq, 220, key=11, page_size=8, **kw)
    rng = np.random.default_rng(0)
    prompts = prompts or [rng.integers(0, 640, k).tolist() for k in (1, 2, 17, 60)[:n_seq]]
    s.prefill(prompts)
    for _ in range(steps):
        s.step(coupling)
    return s, prompts


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("branching,coupling", [((4, 1, 1), False), ((1, 1, 1), False), ((1, 1, 1), True)])
def test_a_pool_changes_nothing_but_the_pages(bits, branching, coupling):
    a, _ = run(branching, coupling, bits=bits)
    b, _ = run(branching, coupling, bits=bits, pool=70)
    assert a.tokens() == b.tokens()
    # every page is a sequence's or free, once, and a sequence has those its tokens need
    rows, n = b.cache.pages.tolist(), [len(x) for x in b.tokens()]
    used = [p for r in rows for p in r if p >= 0]
    free = b.cache.free_list[:int(b.cache.free_count)].tolist()
    assert sorted(used + free) == list(range(70))
    assert b.cache.held.tolist() == [-(-(x - 1) // 8) for x in n] == [sum(p >= 0 for p in r) for r in rows]


@pytest.mark.parametrize("branching,coupling", [((4, 1, 1), False), ((1, 1, 1, 1), True)])
def test_the_4_bit_cache_holds_the_text(branching, coupling):
    s, _ = run(branching, coupling, bits=4, pool=80)
    m = s.model
    for q, text in enumerate(s.tokens()):
        n = len(text) - 1
        kv, _ = plain(m, text[:n])
        pos = torch.arange(n, device=s.device)
        slot = s.cache.slots(torch.full_like(pos, q), pos)
        got = pps.kv_read_q4(s.cache.layers[0], slot)
        # the first layer's keys and values have passed no attention yet: those of a plain pass but for roundings to bf16 before
        # them (embedding's norm and projection, 2^-9 each), which move a number across a code's border at most
        for x, want in zip(got, kv[0]):
            value, scale = held(want)
            off = (x.double() - want).abs().unflatten(-1, (-1, 16))
            assert bool((off <= (1.0 + 2.0 ** -3) * scale[..., None] + 2.0 ** -5 * want.abs().unflatten(-1, (-1, 16))).all())


def test_a_pool_that_runs_out_is_told():
    s, _ = run((3, 1), steps=1, pool=14)
    s.tokens()
    with pytest.raises(RuntimeError, match="flags"):
        for _ in range(12):
            s.step()
        s.tokens()
    assert int(s.status) & pps.FLAG_POOL


@pytest.mark.parametrize("branching,coupling", [((4, 1, 1), False), ((1, 1, 1), False), ((1, 1, 1), True)])
def test_laws_that_forbid_and_favour(branching, coupling):
    # only even tokens may follow, and of these one is favoured beyond all others until it has been said
    n, V = 4, 640
    bits = torch.zeros(V, dtype=torch.int64)
    bits[0::2] = 1
    words = (bits.view(-1, 32) << torch.arange(32)).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).cuda()
    laws = dict(allowed=lambda tok: words.expand(tok.numel(), -1), presence=torch.full((n,), 100.0, device="cuda"),
                bias_off=torch.arange(n + 1, dtype=torch.int32, device="cuda"),
                bias_tok=torch.tensor([10, 20, 30, 40], dtype=torch.int32, device="cuda"), bias_val=torch.full((n,), 60.0, device="cuda"))
    s, prompts = run(branching, coupling, prompts=[[1], [3, 5], [7] * 17, [9, 11]], laws=laws, bits=4, pool=90)
    for q, text in enumerate(s.tokens()):
        new = text[len(prompts[q]):]
        assert new[0] == 10 * (q + 1) and all(x % 2 == 0 for x in new)
        assert len(set(new)) == len(new)  # presence outweighs every logit: no token twice


def test_a_penalised_token_by_the_oracle():
    """The emitted tokens are the keyed race of the shaped logits of a plain pass."""
    n, V = 4, 640
    rep, freq = 1.3, 0.4
    laws = dict(repetition=torch.full((n,), rep, device="cuda"), frequency=torch.full((n,), freq, device="cuda"))
    s, prompts = run((4, 1, 1), laws=laws, pool=90)
    total = agree = 0
    for q, text in enumerate(s.tokens()):
        m = len(text) - 1
        _, logits = plain(s.model, text[:m])
        at = np.arange(len(prompts[q]) - 1, m)
        rows = logits[torch.as_tensor(at).cuda()].clone()
        for i, p in enumerate(at):
            seen = torch.tensor(text[:p + 1], device="cuda")
            said = torch.bincount(seen, minlength=V) > 0
            out = torch.bincount(seen[len(prompts[q]):], minlength=V)
            rows[i] = torch.where(said, torch.where(rows[i] > 0, rows[i] / rep, rows[i] * rep), rows[i]) - freq * out
        key = np.full(at.size, int(s.key[q]), np.uint64)
        win, _, _, margin = oracle.target_rows(rows.float().cpu().numpy(), key, np.zeros(at.size, np.uint64), (at + 1).astype(np.uint32))
        emitted = np.array(text)[at + 1]
        close = margin < 4 * 2 * 8 * 3 * 2.0 ** -9  # as test_gpu_decode has it, for two layers
        assert np.all((win == emitted) | close)
        total, agree = total + at.size, agree + int((win == emitted).sum())
    assert agree >= 0.8 * total, (agree, total)


def test_command(capsys):
    main(["--steps", "3", "--sequences", "3", "--bits", "4", "--pool", "200", "--repetition", "1.2"])
    main(["--steps", "3", "--sequences", "3", "--branching", "1,1", "--coupling", "--bits", "4"])
    assert capsys.readouterr().out.count("accepted per step") == 2
