"""The target-side calls where element offsets pass 2^31 and 2^32: large caches, many tokens, many rows of logits."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_chain import _check

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    pps.lib()
    yield
    torch.cuda.empty_cache()


def rn(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(BF)


def test_a_cache_of_more_than_2_32_elements():
    n_pages, page, kv, d = 16400, 256, 8, 128
    kc, vc = (torch.empty(n_pages, page, kv, d, dtype=BF, device="cuda") for _ in range(2))
    assert kc.numel() > 2 ** 32
    mine = torch.tensor([16399, 0, 8191, 16384, 8192], **I32)  # around 2^31 and 2^32 elements too
    n = 5 * page - 3
    q, k, v = rn(1, n, 16, d), rn(2, n, kv, d), rn(3, n, kv, d)
    at = torch.arange(n, device="cuda")
    slot = mine.long()[at // page] * page + at % page
    got = pps.kv_append(q, k, v, at.int(), slot, kc, vc, None)
    assert torch.equal(got, q)
    assert torch.equal(kc[mine.long()].flatten(0, 1)[:n], k) and torch.equal(vc[mine.long()].flatten(0, 1)[:n], v)
    status = torch.zeros(1, **I32)
    out = pps.paged_attention(q[-2:], kc, vc, mine[None], torch.tensor([n], **I32), torch.tensor([0, 2], **I32), status=status)
    assert int(status) == 0
    w = torch.einsum("ihd,jhd->hij", q[-2:].double(), k.double().repeat_interleave(2, 1)) * d ** -0.5
    w[:, 0, n - 1] = -torch.inf
    p = w.softmax(-1)
    want = torch.einsum("hij,jhd->ihd", p, v.double().repeat_interleave(2, 1))
    size = torch.einsum("hij,jhd->ihd", p, v.double().abs().repeat_interleave(2, 1))
    # the weights and the result are each rounded once to bf16, 2^-8 at most
    assert bool(((out.double() - want).abs() <= 1.01 * 2.0 ** -8 * (want.abs() + size) + 1e-4 * size).all())


def test_more_than_2_31_elements_of_new_tokens():
    n, heads, kv, d = 360000, 32, 8, 128
    qkv = torch.empty(n, heads + 2 * kv, d, dtype=BF, device="cuda")
    assert qkv.numel() > 2 ** 31
    some = torch.tensor([0, 1, 174762, 174763, 349525, 349526, n - 1], device="cuda")
    qkv.zero_()
    qkv[some] = rn(4, len(some), heads + 2 * kv, d)
    q, k, v = qkv.split([heads, kv, kv], dim=1)
    kc, vc = (torch.empty(len(some), 16, kv, d, dtype=BF, device="cuda") for _ in range(2))
    slot = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    slot[some] = 16 * torch.arange(len(some), device="cuda") + 5
    out = pps.kv_append(q, k, v, torch.zeros(n, **I32), slot, kc, vc, None)
    assert torch.equal(out[some], q[some]) and not bool(out[2:100000].any())
    assert torch.equal(kc[:, 5], k[some]) and torch.equal(vc[:, 5], v[some])


def test_more_than_2_31_elements_of_queries():
    """A sequence of one key per token: each gets its value."""
    n, heads, kv, d, page = 530000, 32, 8, 128, 8
    q = torch.empty(n, heads, d, dtype=BF, device="cuda").fill_(0.5)
    assert q.numel() > 2 ** 31
    kc, vc = rn(5, 1000, page, kv, d), rn(6, 1000, page, kv, d)
    pages = (torch.arange(n, device="cuda") % 1000).int()[:, None]
    out = pps.paged_attention(q, kc, vc, pages, torch.ones(n, **I32), torch.arange(n + 1, **I32))
    for a in range(0, n, 100000):
        b = min(a + 100000, n)
        want = vc[pages[a:b, 0].long(), 0].repeat_interleave(heads // kv, 1)
        assert torch.equal(out[a:b], want)


def test_rows_of_logits_past_2_31_elements():
    n, n_draft, V, stride, gamma = 17000, 16900, 700, 131072, 4
    p, q = (torch.empty(r, stride, dtype=BF, device="cuda")[:, :V] for r in (n, n_draft))
    assert n_draft * stride > 2 ** 31
    p.zero_(), q.zero_()
    seqs, at = [0, 8190, 16382, 16995], []
    for s in seqs:
        at += list(range(s, s + 5))
    p[at] = 2 * rn(7, len(at), V)
    rows = torch.full((n,), -1, **I32)
    last = torch.arange(16, device="cuda") + (n_draft - 16)  # the last draft rows, four to a sequence
    for i, s in enumerate(seqs):
        rows[s:s + 4] = last[4 * i:4 * i + 4].int()
        q[last[4 * i:4 * i + 4]] = p[s:s + 4] + 0.5 * rn(8 + i, 4, V)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    tok = torch.zeros(n_draft, **I32)
    tok[last] = q[last].float().argmax(-1).int()
    u = torch.rand(n_draft, generator=g, device="cuda")
    noise = torch.rand(1, V, generator=g, device="cuda").clamp(min=1e-9).log().neg().clamp(min=1e-9)
    for s in seqs:
        off = torch.tensor([s, s + 5], **I32)
        got = pps.verify_chain(p, q, gamma, off, rows, tok, u, noise)
        _check(p, q, gamma, off, rows, tok, u, noise, got=got)
