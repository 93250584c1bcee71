"""The decoding loop where the pool has no pages left for a sequence: it stands still, and goes on when pages come back."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from paper_2609_21858_gb300.decode import Decoder, Session
from test_gpu_decode import plain, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


@pytest.mark.parametrize("branching,coupling", [((3, 1, 1), False), ((1, 1, 1), False), ((1, 1, 1), True)])
def test_a_sequence_without_pages_stands_still(branching, coupling):
    s = Session(Decoder(640, 128, 2, 4, 2, 64, max_pos=512, seed=4), branching, 2, 300, key=5, page_size=8, pool=13)
    s.prefill([[7 * i % 640 for i in range(17)], [3 * i % 640 for i in range(60)]])  # 2 and 8 pages
    stood = torch.zeros(2, dtype=torch.int64, device="cuda")
    for _ in range(30):
        length, text = s.length.clone(), s.text.clone()
        v = s.step(coupling)
        still = v["n_emitted"] == 0
        stood += still
        assert torch.equal(s.length, length + v["n_emitted"])
        assert bool((v["emitted"][still] == -1).all()) and not bool(v["accept_len"][still].any())
        assert torch.equal(s.text[still], text[still])
        # whatever the text says is in pages that the sequence holds
        assert bool((s.cache.held * 8 >= s.length).all())
        assert int(s.cache.held.sum()) + int(s.cache.free_count) == 13
    assert bool((stood > 0).all()) and int(s.status) == pps.FLAG_POOL
    # the second sequence ends: its pages let the first go on
    s.length[1] = 0
    s.cache.trim(s.length)
    s.status.zero_()
    before = int(s.length[0])
    for _ in range(4):
        s.step(coupling)
    s.length[1] = 0  # (it has begun anew)
    text = s.tokens()[0]
    n = len(text) - 1
    assert n >= before + 4 and all(0 <= x < 640 for x in text)
    pos = torch.arange(n, device="cuda")
    slot = s.cache.slots(torch.zeros_like(pos), pos)
    kv, _ = plain(s.model, text[:n])
    for cached, want in zip((s.cache.k[0], s.cache.v[0]), kv[0]):
        got = cached.view(-1, 2, 64)[slot].double()
        assert bool(((got - want).norm(dim=-1) < rounding(1) * want.norm(dim=-1)).all())
