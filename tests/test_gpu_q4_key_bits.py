"""Keys held in 4 bits and the queries of the same call, bit by bit against the formula's operations in 32 bits one by one."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from q4_format import values
from test_gpu_append import BF, F16, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()


def _rotated(x, rope, pos, interleaved):
    """In fp32, a kernel for each operation, so that nothing joins a product and a sum."""
    x, rot = x.float(), rope.shape[1]
    row = rope[pos.long()][:, None]
    c, s = row[..., :rot // 2], row[..., rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    p, q = torch.sub(torch.mul(a, c), torch.mul(b, s)), torch.add(torch.mul(a, s), torch.mul(b, c))
    turned = torch.stack([p, q], dim=-1).flatten(-2) if interleaved else torch.cat([p, q], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _held(x, unit):
    """Of fp32 channels, the values in units and the scales that the format's definition gives, in fp32.  Divisors are tensors:
    a division by a Python number is a product with its reciprocal."""
    z = x if unit is None else x * (torch.ones_like(unit) / unit)[:, None]
    z = z.unflatten(-1, (-1, 16))
    top = z.abs().amax(-1, keepdim=True)
    scale = (top / torch.full_like(top, 6.0)).clamp(max=448.0).to(torch.float8_e4m3fn).float()
    m = torch.where(scale > 0, z / scale, 0.0).clamp(-6.0, 6.0)
    step = torch.where(m.abs() < 2, 0.5, torch.where(m.abs() < 4, 1.0, 2.0))  # (powers of two: exact)
    return (torch.round(m / step) * step * scale).flatten(-2).double(), scale[..., 0].double()


# (tokens, heads, kv heads, channels, rot): of 16-byte, 8-byte and single-channel moves by rot and the offset of the inputs
@pytest.mark.parametrize("dt", [BF, F16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,hq,hk,d,rot,offset,unit", [(40000, 2, 4, 128, 128, 0, True), (40000, 1, 2, 128, 64, 0, False),
                                                       (30000, 3, 2, 80, 40, 0, True), (30000, 2, 2, 64, 64, 4, False),
                                                       (20000, 1, 2, 128, 128, 1, True), (50000, 4, 1, 48, 10, 0, False)])
def test_keys_and_queries_are_those_of_products_and_sums_rounded_one_by_one(n, hq, hk, d, rot, offset, unit, interleaved, dt):
    g, q, k, v = _inputs(n, hq, hk, d, dt, n + d + rot + offset, offset)
    rope = pps.rope_table(100000, rot)
    pos = torch.randint(0, 100000, (n,), generator=g, device="cuda", dtype=torch.int32)
    cache = pps.cache_q4(-(-n // 16), 16, hk, d)
    if unit:
        cache = cache._replace(k_unit=0.25 + torch.rand(hk, generator=g, device="cuda"))
    out = pps.kv_append_q4(q, k, v, pos, torch.arange(n, device="cuda"), cache, rope, interleaved=interleaved)
    assert torch.equal(out, _rotated(q, rope, pos, interleaved).to(dt))
    codes, scales = (x.flatten(0, 1)[:n] for x in (cache.k, cache.k_scale))
    want, scale = _held(_rotated(k, rope, pos, interleaved), cache.k_unit)
    ones = values(torch.full_like(codes, 0x22), scales).unflatten(-1, (-1, 16))[..., 0]
    assert torch.equal(ones, scale)
    assert torch.equal(values(codes, scales), want)


def test_scales_next_to_a_border():
    """Largest magnitudes whose sixth lies next to the middle of two scales, where a product with 1 / 6 rounds to the other one."""
    n, d = 64, 16
    border = torch.tensor(7.1249995, device="cuda").view(torch.int32)
    top = (border - n // 2 + torch.arange(n, dtype=torch.int32, device="cuda")).view(torch.float32)
    k = torch.zeros(n, 1, d, dtype=F16, device="cuda")
    k[:, 0, 0] = 2.0
    rope = torch.zeros(n, d, device="cuda")
    rope[:, 0] = top / 2  # in a cosine's place: the rotated channel is the largest, exactly
    cache = pps.cache_q4(n // 16, 16, 1, d)
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    pps.kv_append_q4(k, k, k, at, at.long(), cache, rope)
    want = (top / torch.full_like(top, 6.0)).to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(cache.k_scale.flatten(0, 1)[:, 0, 0], want) and len(set(want.tolist())) == 2
