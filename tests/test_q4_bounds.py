"""How far a channel held in 4 bits is off: the bounds that include/pps.h states, of the definition and (on the GPU) of what is held."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from q4_format import held, values

# fp32 roundings of z, its sixth and its quotient, beside the bounds in exact arithmetic
ROUND = 1 + 4 * 2.0 ** -24


def blocks(lo, hi, dt, n=6000, device="cpu"):
    """[n, 16] blocks of numbers of dt whose largest magnitude lies in [lo, hi], evenly over its logarithm, both ends among them; the others are spread
    from a sixth of it on, where codes are farthest apart."""
    g = torch.Generator().manual_seed(int(hi * 64))
    top = torch.logspace(0, 1, n, base=hi / lo, dtype=torch.float64) * lo
    x = (top[:, None] * (1 / 6 + 5 / 6 * torch.rand(n, 16, generator=g, dtype=torch.float64)) * (1 - 2 * torch.randint(0, 2, (n, 16), generator=g)))
    x[:, 0] = top
    x = x.to(dt).double()
    x[0, 0], x[-1, 0] = torch.tensor([lo, hi], dtype=torch.float64).to(dt).double()
    return x.clamp(-hi, hi).to(device)


def check(x, v, unit=1.0):
    """x: what was to be held, v: what is."""
    x, v = x / unit, v / unit
    top, off = x.abs().amax(-1), (x - v).abs().amax(-1)
    normal, low, zero, high = (top >= 6 * 2.0 ** -6) & (top <= 2688), (top < 6 * 2.0 ** -6) & (top > 6 * 2.0 ** -10), top <= 6 * 2.0 ** -10, top > 2688
    assert bool((off <= 3 / 17 * top * ROUND)[normal].all())
    assert bool((off <= top / 3 * ROUND)[low].all())
    assert not bool(v[zero].any())
    big = (x.abs() > 2688) & high[:, None]
    assert bool((v[big].abs() == 2688).all())
    return normal, low, zero, high, off / top


RANGES = [(6 * 2.0 ** -6, 2688.0), (6 * 2.0 ** -10, 6 * 2.0 ** -6), (2.0 ** -14, 6 * 2.0 ** -10), (2688.0, 60000.0)]


@pytest.mark.parametrize("lo,hi", RANGES)
def test_the_definition(lo, hi):
    x = blocks(lo, hi, torch.float32, 40000)
    kind = check(x, held(x[:, None])[0][:, 0])
    worst = kind[4].max().item()
    # the bounds are not generous either
    assert worst > {RANGES[0]: 0.175, RANGES[1]: 0.32, RANGES[2]: 0.99, RANGES[3]: 0.9}[(lo, hi)]


@pytest.mark.gpu
@pytest.mark.parametrize("unit", [1.0, 0.0625, 0.001])
@pytest.mark.parametrize("lo,hi", RANGES)
def test_what_is_held(lo, hi, unit):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    x = blocks(lo * unit, hi * unit, torch.bfloat16, device="cuda")
    n = x.shape[0]
    v = x.view(n, 1, 16).bfloat16()
    x = v.double()[:, 0]
    cache = pps.cache_q4(-(-n // 16), 16, 1, 16)
    u = torch.full((1,), unit, device="cuda")
    cache = cache._replace(k_unit=u, v_unit=u)
    pps.kv_append_q4(v, v, v, None, torch.arange(n, device="cuda"), cache, None)
    for codes, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        got = values(codes.flatten(0, 1)[:n], scales.flatten(0, 1)[:n])[:, 0]
        check(x, got * float(u), float(u))
