"""pps_kv_append against the formulas in 64 bits: norm, rotation, cache slots, layouts and alignments."""
import pytest
import torch

from paper_2609_21858_gb300 import pps

pytestmark = pytest.mark.gpu

BF, F16 = torch.bfloat16, torch.float16
U = {BF: 2.0 ** -8, F16: 2.0 ** -11}  # unit roundoff


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def _turned(x, weight, eps, rope, pos, interleaved):
    """The definition in 64 bits, and the size of the terms of each channel."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    size = x.abs().clone()
    y = x.clone()
    if rope is not None:
        rot = rope.shape[1]
        row = rope.double()[pos.long().clamp(0, rope.shape[0] - 1)]
        c, s = row[:, None, :rot // 2], row[:, None, rot // 2:]
        i = torch.arange(rot // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def _close(got, want, size, dt):
    # one rounding of the result, and fp32 arithmetic on the terms (a dozen roundings of 2^-24, the norm's sum among them)
    err = (got.double() - want).abs()
    tol = U[dt] * want.abs() + 2.0 ** -19 * size + 2.0 ** -25
    assert bool((err <= tol).all()), f"worst excess {(err - tol).max().item():.3g}"


def _inputs(n, hq, hk, d, dt, seed, offset=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    width = (hq + 2 * hk) * d
    flat = (torch.randn(n * width + offset, generator=g, device="cuda") * 1.5).to(dt)
    qkv = flat[offset:].view(n, width)
    q, k, v = (x.view(n, -1, d) for x in qkv.split([hq * d, hk * d, hk * d], dim=1))
    return g, q, k, v


# (tokens, heads, kv heads, channels, rot, page, dtype): rot in thirds of a vector, odd pages, one token, wide heads
CASES = [(1, 32, 8, 128, 128, 16, BF), (37, 28, 4, 128, 128, 16, F16), (300, 14, 2, 64, 32, 64, BF),
         (5, 3, 1, 80, 80, 8, BF), (9, 20, 4, 80, 40, 16, F16), (17, 2, 2, 8, 8, 3, BF), (11, 4, 4, 24, 10, 5, F16),
         (6, 5, 1, 256, 256, 16, BF), (130, 12, 12, 64, 64, 32, F16), (4, 1, 1, 256, 0, 1, BF), (7, 6, 3, 72, 2, 7, BF),
         (6000, 8, 2, 16, 16, 128, BF)]


@pytest.mark.parametrize("n,hq,hk,d,rot,page,dt", CASES)
@pytest.mark.parametrize("norm,interleaved,layout,offset", [(False, False, "token", 0), (True, False, "head", 0),
                                                            (True, True, "token", 0), (False, True, "head", 3),
                                                            (True, False, "token", 4)])
def test_against_the_formulas(n, hq, hk, d, rot, page, dt, norm, interleaved, layout, offset):
    g, q, k, v = _inputs(n, hq, hk, d, dt, n + d + rot, offset)
    max_pos = 70000
    rope = pps.rope_table(max_pos, rot) if rot else None
    pos = torch.randint(0, max_pos, (n,), generator=g, device="cuda", dtype=torch.int32)
    n_pages = -(-n // page) + 2
    shape = (n_pages, hk, page, d) if layout == "head" else (n_pages, page, hk, d)
    caches = [torch.randn(shape, generator=g, device="cuda").to(dt) for _ in range(2)]
    if layout == "head":
        caches = [c.transpose(1, 2) for c in caches]
    before = [c.clone() for c in caches]
    slot = torch.randperm(n_pages * page, generator=g, device="cuda")[:n].contiguous()
    slot[n // 2::3] = -1  # tokens that are not written
    w = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2)] if norm else [None, None]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = pps.kv_append(q, k, v, pos, slot, *caches, rope, q_norm=w[0], k_norm=w[1], eps=1e-5,
                        interleaved=interleaved, status=status)
    assert int(status.item()) == 0
    _close(out, *_turned(q, w[0], 1e-5, rope, pos, interleaved), dt)
    kept = slot >= 0
    page_of, in_page = slot[kept] // page, slot[kept] % page
    want, size = _turned(k, w[1], 1e-5, rope, pos, interleaved)
    _close(caches[0][page_of, in_page], want[kept], size[kept], dt)
    assert torch.equal(caches[1][page_of, in_page], v[kept])
    for c, b in zip(caches, before):  # nothing else has changed
        c[page_of, in_page] = b[page_of, in_page]
        assert torch.equal(c, b)


def test_queries_in_place_and_one_norm():
    n, hq, hk, d = 50, 8, 2, 128
    g, q, k, v = _inputs(n, hq, hk, d, BF, 5)
    rope, pos = pps.rope_table(100, d), torch.arange(n, device="cuda", dtype=torch.int32)
    kc, vc = (torch.zeros(4, 16, hk, d, dtype=BF, device="cuda") for _ in range(2))
    slot = torch.arange(n, device="cuda")
    w = torch.full((d,), 0.5, dtype=BF, device="cuda")
    want, size = _turned(q, w, 1e-6, rope, pos, False)
    out = pps.kv_append(q, k, v, pos, slot, kc, vc, rope, q_norm=w, out=q)
    assert out.data_ptr() == q.data_ptr()
    _close(q, want, size, BF)
    _close(kc.view(-1, hk, d)[:n], *_turned(k, None, 0, rope, pos, False), BF)


def test_positions_and_slots_out_of_range_are_flagged_and_harmless():
    n, hq, hk, d = 6, 4, 2, 64
    _, q, k, v = _inputs(n, hq, hk, d, BF, 8)
    rope = pps.rope_table(10, d)
    kc, vc = (torch.zeros(3, 16, hk, d, dtype=BF, device="cuda") for _ in range(2))  # slots 32..47 (page 2) lie outside the views
    slot = torch.tensor([0, 32, 2 ** 40, -5, 31, 3], device="cuda")
    for bad_pos, bad_slot in ((True, False), (False, True)):
        pos = torch.tensor([0, 1, 2, 3, 10 if bad_pos else 9, -1 if bad_pos else 5], dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kc.zero_(), vc.zero_()
        at = slot if bad_slot else torch.arange(n, device="cuda")
        out = pps.kv_append(q, k, v, pos, at, kc[:2], vc[:2], rope, status=status)
        assert int(status.item()) == pps.FLAG_INDEX
        _close(out, *_turned(q, None, 0, rope, pos, False), BF)
        assert not bool(kc[2].any()) and not bool(vc[2].any())
        if bad_slot:
            assert torch.equal(vc.view(-1, hk, d)[[0, 31, 3]], v[[0, 4, 5]]) and int(vc.view(48, -1).any(1).sum()) == 3


def test_non_finite_values_stay_in_their_head():
    n, hq, hk, d = 4, 2, 2, 64
    _, q, k, v = _inputs(n, hq, hk, d, BF, 9)
    q, k, v = q.clone(), k.clone(), v.clone()
    q[1, 0, 3], k[2, 1, 0], v[0, 0, 0] = float("nan"), float("inf"), float("-inf")
    rope, pos = pps.rope_table(10, d), torch.arange(n, dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros(1, 16, hk, d, dtype=BF, device="cuda") for _ in range(2))
    w = torch.ones(d, dtype=BF, device="cuda")
    out = pps.kv_append(q, k, v, pos, torch.arange(n, device="cuda"), kc, vc, rope, q_norm=w, k_norm=w)
    finite = torch.isfinite(out).all(-1)
    assert not bool(finite[1, 0]) and int((~finite).sum()) == 1
    finite = torch.isfinite(kc[0, :n]).all(-1)
    assert not bool(finite[2, 1]) and int((~finite).sum()) == 1
    assert torch.equal(vc[0, :n], v)


def test_another_stream_and_no_tokens():
    n, hq, hk, d = 33, 4, 2, 128
    _, q, k, v = _inputs(n, hq, hk, d, F16, 10)
    rope, pos = pps.rope_table(64, d), torch.arange(n, dtype=torch.int32, device="cuda")
    slot = torch.arange(n, device="cuda")
    kc, vc = (torch.zeros(3, 16, hk, d, dtype=F16, device="cuda") for _ in range(2))
    want = pps.kv_append(q, k, v, pos, slot, kc, vc, rope)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
    side.wait_stream(torch.cuda.current_stream())
    got = pps.kv_append(q, k, v, pos, slot, kc2, vc2, rope, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(kc, kc2) and torch.equal(vc, vc2)
    none = pps.kv_append(q[:0], k[:0], v[:0], pos[:0], slot[:0], kc, vc, rope)
    assert none.shape == (0, hq, d)


def test_refusals():
    n, hq, hk, d = 4, 4, 2, 64
    _, q, k, v = _inputs(n, hq, hk, d, BF, 11)
    rope, pos = pps.rope_table(16, d), torch.zeros(n, dtype=torch.int32, device="cuda")
    slot = torch.arange(n, device="cuda")
    kc, vc = (torch.zeros(1, 16, hk, d, dtype=BF, device="cuda") for _ in range(2))
    ok = dict(q=q, k=k, v=v, pos=pos, slot=slot, k_cache=kc, v_cache=vc, rope=rope)
    pps.kv_append(**ok)
    for bad in (dict(q=q.float()), dict(k=k.half()), dict(pos=pos.long()), dict(slot=slot.int()), dict(rope=rope.double()),
                dict(k_cache=kc[0]), dict(v_cache=vc.half()), dict(q_norm=torch.ones(d, device="cuda")), dict(q=q.cpu())):
        with pytest.raises(TypeError):
            pps.kv_append(**{**ok, **bad})
    for bad in (dict(k=k[:3]), dict(v=v[:, :1]), dict(pos=pos[:3]), dict(slot=slot[:3]), dict(v_cache=vc[:, :8]),
                dict(out=q[:, :2]), dict(q_norm=torch.ones(d - 1, dtype=BF, device="cuda")), dict(k=k[..., :32])):
        with pytest.raises(ValueError):
            pps.kv_append(**{**ok, **bad})
    with pytest.raises(pps.PPSError) as e:
        pps.kv_append(**{**ok, "rope": pps.rope_table(16, d + 2)})
    assert e.value.code == pps.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        pps.rope_table(16, 7)
