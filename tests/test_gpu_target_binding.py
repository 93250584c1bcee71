"""The two ways through the binding of the target-side calls (the extension, and Python when a stream is named) give the
same bits, and both follow use_library."""
import pytest
import torch

from paper_2609_21858_gb300 import pps

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def both(call):
    """Results of the call without a stream and on the current one by name."""
    a = call()
    b = call(stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    return a, b


@pytest.fixture(params=[10, 7])
def rounds(request):
    pps.use_library(request.param)
    yield request.param
    pps.use_library(10)


def test_calls_agree(rounds):
    g = torch.Generator(device="cuda")
    g.manual_seed(rounds)
    rn = lambda *s, dt=torch.bfloat16: torch.randn(s, generator=g, device="cuda").to(dt)
    i32 = dict(dtype=torch.int32, device="cuda")
    n, heads, kv_heads, d = 9, 6, 2, 64
    kc, vc = rn(6, 16, kv_heads, d), rn(6, 16, kv_heads, d)
    caches = [(kc.clone(), vc.clone()) for _ in range(2)]
    q, k, v = rn(n, heads, d), rn(n, kv_heads, d), rn(n, kv_heads, d)
    pos, slot = torch.arange(n, **i32), torch.arange(n, device="cuda") + 30
    rope = pps.rope_table(64, d)
    it = iter(caches)
    qs = both(lambda **kw: pps.kv_append(q, k, v, pos, slot, *next(it), rope, **kw))
    assert torch.equal(*qs) and torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])
    assert not torch.equal(caches[0][0], kc)
    kc, vc = caches[0]
    pages = torch.tensor([[5, 1, 0], [2, 3, 4]], **i32)
    kv_len, q_off = torch.tensor([33, 48], **i32), torch.tensor([0, 4, 9], **i32)
    outs = both(lambda **kw: pps.paged_attention(qs[0], kc, vc, pages, kv_len, q_off, **kw))
    assert torch.equal(*outs) and bool(outs[0].any())
    V, gamma = 300, 3
    p, ql = rn(8, V), rn(6, V)
    seq_off, rows = torch.tensor([0, 4, 8], **i32), torch.tensor([0, 1, 2, -1, 3, 4, 5, -1], **i32)
    tok, u = torch.randint(0, V, (6,), generator=g, **i32), torch.rand(6, generator=g, device="cuda")
    noise = torch.rand(2, V, generator=g, device="cuda") + 0.01
    a, b = both(lambda **kw: pps.verify_chain(p, ql, gamma, seq_off, rows, tok, u, noise, **kw))
    own = {name: torch.full_like(x, 77) for name, x in a.items() if name != "accept_prob"}
    assert pps.verify_chain(p, ql, gamma, seq_off, rows, tok, u, noise, out=own) is own
    for name, x in a.items():
        assert torch.equal(x, b[name])
        assert name == "accept_prob" or torch.equal(x, own[name])


@pytest.mark.parametrize("named", [False, True])
def test_refusals_agree(named):
    """What the extension hands on is refused in the same words either way."""
    kw = dict(stream=torch.cuda.current_stream()) if named else {}
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    q, kc = z(2, 4, 64), z(3, 16, 2, 64)
    pages, kv, off = torch.zeros(1, 2, **i32), torch.tensor([5], **i32), torch.tensor([0, 2], **i32)
    with pytest.raises(TypeError, match="kv_len"):
        pps.paged_attention(q, kc, kc, pages, kv.long(), off, **kw)
    with pytest.raises(ValueError, match="mask"):
        pps.paged_attention(q, kc, kc, pages, kv, off, mask=torch.zeros(3, 1, **i32), **kw)
    with pytest.raises(pps.PPSError):
        pps.paged_attention(q, z(3, 12, 2, 64), z(3, 12, 2, 64), pages, kv, off, **kw)
    with pytest.raises(TypeError, match="slot"):
        pps.kv_append(q, q[:, :2], q[:, :2], torch.arange(2, **i32), torch.arange(2, **i32), kc, kc.clone(), None, **kw)
