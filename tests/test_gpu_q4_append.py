"""pps_kv_append_q4 and pps_kv_read_q4 against the format's definition in 64 bits."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from q4_format import held, values
from test_gpu_append import BF, F16, U, _close, _inputs, _turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def _cache(g, n_pages, page, hk, d, layout, unit):
    def one(n):
        shape = (n_pages, hk, page, n) if layout == "head" else (n_pages, page, hk, n)
        x = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
        return x.transpose(1, 2) if layout == "head" else x
    units = [0.25 + torch.rand(hk, generator=g, device="cuda") for _ in range(2)] if unit else [None, None]
    return pps.CacheQ4(one(d // 2), one(d // 2), one(pps.q4_scale_bytes(d)), one(pps.q4_scale_bytes(d)), *units)


def _near(codes, scales, unit, want, size):
    """Values held of numbers `want` that fp32 arithmetic gets up to 2^-19 of `size` (a dozen roundings of 2^-24 on terms
    of that size): within half a step of the scale that is held, and the scale within half of its own step."""
    u = 1.0 if unit is None else unit.double()[:, None, None]
    b = scales[..., :want.shape[-1] // 16]
    s = values(torch.full_like(codes, 0x22), scales).unflatten(-1, (-1, 16))[..., :1] * u  # (code 2: one)
    v, w, off = (x.unflatten(-1, (-1, 16)) for x in (values(codes, scales, unit), want, 2.0 ** -19 * size + 2.0 ** -40))
    top, slack = w.abs().amax(-1, keepdim=True) / 6, off.amax(-1, keepdim=True)
    step = torch.maximum(s * 2.0 ** -3, torch.full_like(s, 2.0 ** -9) * u)  # a step of e4m3 is 2^-3 of a number or less
    assert bool(((s - top.clamp(max=448.0 * 1.0000001 * (u if unit is not None else 1.0))).abs() <= step / 2 + slack).all())
    m = torch.where(s > 0, w.abs() / s, 0.0)
    half = torch.where(m <= 2, 0.25, torch.where(m <= 4, 0.5, 1.0)) * s
    assert bool(((v - w).abs() <= torch.where(s > 0, half, w.abs()) * 1.0001 + off).all())
    assert b.shape[-1] == want.shape[-1] // 16


CASES = [(1, 32, 8, 128, 128, 16, BF), (37, 28, 4, 128, 128, 16, F16), (300, 14, 2, 64, 32, 64, BF),
         (5, 3, 1, 80, 80, 8, BF), (9, 20, 4, 80, 40, 16, F16), (17, 2, 2, 16, 8, 3, BF), (11, 4, 4, 48, 10, 5, F16),
         (6, 5, 1, 256, 256, 16, BF), (130, 12, 12, 64, 64, 32, F16), (4, 1, 1, 256, 0, 1, BF), (7, 6, 3, 112, 2, 7, BF),
         (6000, 8, 2, 32, 16, 128, BF), (3, 2, 1, 176, 96, 16, F16)]


@pytest.mark.parametrize("n,hq,hk,d,rot,page,dt", CASES)
@pytest.mark.parametrize("norm,interleaved,layout,offset,unit", [(False, False, "head", 0, False), (True, False, "token", 0, True),
                                                                 (True, True, "head", 0, False), (False, True, "token", 3, True),
                                                                 (True, False, "head", 4, False)])
def test_against_the_formulas(n, hq, hk, d, rot, page, dt, norm, interleaved, layout, offset, unit):
    g, q, k, v = _inputs(n, hq, hk, d, dt, n + d + rot, offset)
    max_pos = 70000
    rope = pps.rope_table(max_pos, rot) if rot else None
    pos = torch.randint(0, max_pos, (n,), generator=g, device="cuda", dtype=torch.int32)
    n_pages = -(-n // page) + 2
    cache = _cache(g, n_pages, page, hk, d, layout, unit)
    before = [t.clone() for t in cache[:4]]
    slot = torch.randperm(n_pages * page, generator=g, device="cuda")[:n].contiguous()
    slot[n // 2::3] = -1  # tokens that are not written
    w = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2)] if norm else [None, None]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = pps.kv_append_q4(q, k, v, pos, slot, cache, rope, q_norm=w[0], k_norm=w[1], eps=1e-5,
                           interleaved=interleaved, status=status)
    assert int(status.item()) == 0
    _close(out, *_turned(q, w[0], 1e-5, rope, pos, interleaved), dt)
    kept = slot >= 0
    at = slot[kept] // page, slot[kept] % page
    want, size = _turned(k, w[1], 1e-5, rope, pos, interleaved)
    _near(cache.k[at], cache.k_scale[at], cache.k_unit, want[kept], size[kept])
    got, (want, scale) = values(cache.v[at], cache.v_scale[at]), held(v[kept].double(), cache.v_unit)
    assert torch.equal(got, want)  # values pass no rounding before the format's own
    for c, b in zip(cache[:4], before):  # nothing else has changed (of the scales' rows, nor their unused bytes)
        if c.shape[-1] == d // 2:
            c[at] = b[at]
        else:
            c[at][..., :d // 16], x = b[at][..., :d // 16], c[at]
            x[..., :d // 16] = b[at][..., :d // 16]
            c[at] = x
        assert torch.equal(c, b)


@pytest.mark.parametrize("dt", [BF, F16])
@pytest.mark.parametrize("hk,d,page,layout,unit", [(8, 128, 16, "head", False), (3, 80, 5, "token", True), (1, 16, 1, "head", True),
                                                   (40, 256, 8, "token", False), (2, 64, 64, "head", True)])
def test_reading_back(dt, hk, d, page, layout, unit):
    g = torch.Generator(device="cuda").manual_seed(hk + d)
    cache = _cache(g, 6, page, hk, d, layout, unit)
    for t in (cache.k_scale, cache.v_scale):  # every scale, but for the largest, which fp16 may not hold times a unit
        t[(t % 128 > 110) & (t % 128 < 127)] = 50
    slot = torch.randint(-1, 6 * page, (777,), generator=g, device="cuda")
    k, v = pps.kv_read_q4(cache, slot, dtype=dt)
    for got, codes, scales, u in ((k, cache.k, cache.k_scale, cache.k_unit), (v, cache.v, cache.v_scale, cache.v_unit)):
        at = slot.clamp(min=0) // page, slot.clamp(min=0) % page
        s = values(torch.full_like(codes[at], 0x22), scales[at])  # unit * scale, then * code, each rounded to 32 bits
        if u is not None:
            s = (s.float() * u[:, None]).double()
        one = torch.zeros_like(scales[at])
        one[:] = 0x38
        want = (s.float() * values(codes[at], one).float()).to(dt)
        want[slot < 0] = 0
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    out = torch.full((2, 777, hk, d + 8), 3.0, dtype=dt, device="cuda")
    again = pps.kv_read_q4(cache, slot, dtype=dt, out=(out[0, :, :, :d], out[1, :, :, :d]))
    assert torch.equal(torch.nan_to_num(again[0]), torch.nan_to_num(k)) and bool((out[..., d:] == 3).all())


def test_what_is_appended_reads_back_and_float8_scales():
    n, hq, hk, d = 100, 8, 2, 64
    g, q, k, v = _inputs(n, hq, hk, d, BF, 3)
    cache = pps.cache_q4(8, 16, hk, d)
    cache = cache._replace(k_scale=cache.k_scale.view(torch.float8_e4m3fn), v_scale=cache.v_scale.view(torch.float8_e4m3fn))
    slot = torch.randperm(128, generator=g, device="cuda")[:n]
    pps.kv_append_q4(q, k, v, torch.zeros(n, dtype=torch.int32, device="cuda"), slot, cache, pps.rope_table(4, d))
    got = pps.kv_read_q4(cache, slot)
    for x, y in zip(got, (k, v)):  # position 0: no rotation; values of 6 bits are exact in bf16
        assert torch.equal(x.double(), held(y.double())[0])


def test_positions_and_slots_out_of_range_are_flagged_and_harmless():
    n, hq, hk, d = 6, 4, 2, 64
    _, q, k, v = _inputs(n, hq, hk, d, BF, 8)
    rope = pps.rope_table(10, d)
    whole = pps.cache_q4(3, 16, hk, d)
    cache = pps.CacheQ4(*(t[:2] for t in whole[:4]))  # slots 32..47 (page 2) lie outside the views
    slot = torch.tensor([0, 32, 2 ** 40, -5, 31, 3], device="cuda")
    for bad_pos, bad_slot in ((True, False), (False, True)):
        pos = torch.tensor([0, 1, 2, 3, 10 if bad_pos else 9, -1 if bad_pos else 5], dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        for t in whole[:4]:
            t.zero_()
        at = slot if bad_slot else torch.arange(n, device="cuda")
        out = pps.kv_append_q4(q, k, v, pos, at, cache, rope, status=status)
        assert int(status.item()) == pps.FLAG_INDEX
        _close(out, *_turned(q, None, 0, rope, pos, False), BF)
        assert not any(bool(t[2].any()) for t in whole[:4])
        if bad_slot:
            want, _ = held(v.double())
            assert torch.equal(values(whole.v, whole.v_scale).flatten(0, 1)[[0, 31, 3]], want[[0, 4, 5]])
            assert int(whole.v_scale.flatten(0, 1).flatten(1).any(1).sum()) == 3
    status.zero_()
    k2, v2 = pps.kv_read_q4(cache, slot, status=status)
    assert int(status.item()) == pps.FLAG_INDEX and not bool(k2[[1, 2, 3]].any()) and bool(v2[[0, 4, 5]].any())


def test_blocks_that_are_not_finite_zero_or_out_of_the_scales_range():
    n, hq, hk, d = 4, 2, 2, 64
    _, q, k, v = _inputs(n, hq, hk, d, BF, 9)
    q, k, v = q.clone(), k.clone(), v.clone()
    k[2, 1, 0], v[0, 0, 17], v[1, 0, 5] = float("inf"), float("nan"), float("-inf")
    v[2, 0, :16] = 0
    v[2, 1] *= 1e-6   # a scale that rounds to zero
    v[3, 0] *= 1e6    # one past the largest
    cache = pps.cache_q4(1, 16, hk, d)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    pps.kv_append_q4(q, k, v, pos, torch.arange(n, device="cuda"), cache, pps.rope_table(10, d))
    got, (want, _) = values(cache.v, cache.v_scale)[0, :n], held(v.double())
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and int(torch.isnan(got).sum()) == 32
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    assert not bool(got[2, 1].any()) and not bool(got[2, 0, :16].any())
    bad = torch.isnan(values(cache.k, cache.k_scale)[0, :n]).unflatten(-1, (-1, 16)).any(-1)
    assert bool(bad[2, 1, 0]) and bool(bad[2, 1, 2]) and int(bad.sum()) == 2  # channel 0 and its partner of the rotation, 32


def test_another_stream_a_graph_and_no_tokens():
    n, hq, hk, d = 33, 4, 2, 128
    _, q, k, v = _inputs(n, hq, hk, d, F16, 10)
    rope, pos = pps.rope_table(64, d), torch.arange(n, dtype=torch.int32, device="cuda")
    slot = torch.arange(n, device="cuda")
    a, b, c = (pps.cache_q4(3, 16, hk, d) for _ in range(3))
    want = pps.kv_append_q4(q, k, v, pos, slot, a, rope)
    read = pps.kv_read_q4(a, slot, dtype=F16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pps.kv_append_q4(q, k, v, pos, slot, b, rope, stream=side)
    again = pps.kv_read_q4(b, slot, dtype=F16, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(x, y) for x, y in zip(read, again))
    torch.cuda.synchronize()
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(want)
    with torch.cuda.graph(graph):
        pps.kv_append_q4(q, k, v, pos, slot, c, rope, out=out)
    graph.replay()
    assert torch.equal(out, want) and all(torch.equal(x, y) for x, y in zip(a[:4], c[:4]))
    assert pps.kv_append_q4(q[:0], k[:0], v[:0], pos[:0], slot[:0], a, rope).shape == (0, hq, d)
    assert pps.kv_read_q4(a, slot[:0])[0].shape == (0, hk, d)


def test_refusals():
    n, hq, hk, d = 4, 4, 2, 64
    _, q, k, v = _inputs(n, hq, hk, d, BF, 11)
    rope, pos = pps.rope_table(16, d), torch.zeros(n, dtype=torch.int32, device="cuda")
    slot = torch.arange(n, device="cuda")
    cache = pps.cache_q4(1, 16, hk, d)
    ok = dict(q=q, k=k, v=v, pos=pos, slot=slot, cache=cache, rope=rope)
    pps.kv_append_q4(**ok)
    half = torch.ones(hk, dtype=BF, device="cuda")
    for bad in (dict(q=q.float()), dict(k=k.half()), dict(pos=pos.long()), dict(slot=slot.int()), dict(rope=rope.double()),
                dict(cache=cache.k), dict(cache=None), dict(cache=cache._replace(k=cache.k.int())), dict(q=q.cpu()),
                dict(cache=cache._replace(v_scale=cache.v_scale.to(torch.float16))), dict(cache=cache._replace(k_unit=half)),
                dict(cache=cache._replace(v=None)), dict(slot=None), dict(pos=None), dict(k=[1])):
        with pytest.raises(TypeError):
            pps.kv_append_q4(**{**ok, **bad})
    wide = torch.zeros(1, 16, hk, 8, dtype=torch.uint8, device="cuda")
    for bad in (dict(k=k[:3]), dict(v=v[:, :1]), dict(pos=pos[:3]), dict(slot=slot[:3]), dict(out=q[:, :2]),
                dict(cache=cache._replace(v=cache.v[:, :8])), dict(cache=cache._replace(k_scale=wide)),
                dict(cache=cache._replace(k=cache.k.contiguous())), dict(cache=cache._replace(k_unit=torch.ones(1, device="cuda"))),
                dict(cache=cache._replace(v_scale=cache.v_scale.contiguous()))):
        with pytest.raises(ValueError):
            pps.kv_append_q4(**{**ok, **bad})
    for bad in (dict(slot=slot.int()), dict(cache=3), dict(dtype=torch.float32), dict(slot=slot.cpu())):
        with pytest.raises(TypeError):
            pps.kv_read_q4(**{**dict(cache=cache, slot=slot), **bad})
    with pytest.raises(pps.PPSError) as e:
        pps.kv_append_q4(**{**ok, "rope": pps.rope_table(16, d + 2)})
    assert e.value.code == pps.ERR_INVALID_ARG
    for d in (8, 24, 272):
        with pytest.raises(ValueError):
            pps.cache_q4(1, 16, 2, d)
