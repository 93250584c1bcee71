"""pps_kv_append with heads whose last unit has one vector (head_dim - rot an odd multiple of 8): what is not finite in one
token's head, or in a norm's weights, reaches nothing else, however many tokens the same lanes take after it."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_append import BF, F16, _cuda, _inputs, _turned, U  # noqa: F401

pytestmark = pytest.mark.gpu

N = 10000  # several times the tokens in work at once
SHAPES = [(32, 8, 72, 64, BF), (32, 8, 72, 0, F16), (7, 1, 40, 32, BF), (6, 2, 24, 16, F16), (12, 4, 120, 96, BF), (4, 2, 8, 0, BF)]


def run(hq, hk, d, rot, dt, seed, change, interleaved=False, eps=1e-5):
    g, q, k, v = _inputs(N, hq, hk, d, dt, seed)
    w = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2)]
    change(q, k, w)
    rope = pps.rope_table(500, rot) if rot else None
    pos = torch.randint(0, 500, (N,), generator=g, device="cuda", dtype=torch.int32)
    kc, vc = (torch.zeros(N // 16, 16, hk, d, dtype=dt, device="cuda") for _ in range(2))
    out = pps.kv_append(q, k, v, pos, torch.arange(N, device="cuda"), kc, vc, rope, *w, eps=eps, interleaved=interleaved)
    assert torch.equal(vc.view(N, hk, d), v)
    for got, x, weight in ((out, q, w[0]), (kc.view(N, hk, d), k, w[1])):
        want, size = _turned(x, weight, eps, rope, pos, interleaved)
        fine = torch.isfinite(want)
        assert bool((torch.isfinite(got) == fine).all()), f"{int((torch.isfinite(got) != fine).sum())} values"
        # one rounding of the result, fp32 arithmetic on the terms (a dozen roundings of 2^-24)
        err = (got.double() - want).abs()[fine]
        assert bool((err <= (U[dt] * want.abs() + 2.0 ** -19 * size + 2.0 ** -25)[fine]).all())
        yield fine


@pytest.mark.parametrize("hq,hk,d,rot,dt", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("x", [float("nan"), float("inf")])
def test_a_head_that_is_not_finite(hq, hk, d, rot, dt, interleaved, x):
    def change(q, k, w):
        q[0, 0, 1], q[1, hq - 1, d - 1], k[0, hk - 1, 2], k[17, 0, 0] = x, x, x, x
    fine_q, fine_k = run(hq, hk, d, rot, dt, d + rot, change, interleaved)
    if x != x:
        assert int((~fine_q).any(-1).sum()) == 2 and int((~fine_k).any(-1).sum()) == 2


@pytest.mark.parametrize("hq,hk,d,rot,dt", SHAPES)
def test_heads_of_zeros_without_eps(hq, hk, d, rot, dt):
    def change(q, k, w):
        q[0, 0], k[0, hk - 1] = 0.0, 0.0  # 0 / 0
    fine_q, fine_k = run(hq, hk, d, rot, dt, d + rot + 1, change, eps=0.0)
    assert not bool(fine_q[0, 0].any()) and int((~fine_q).any(-1).sum()) == 1
    assert not bool(fine_k[0, hk - 1].any()) and int((~fine_k).any(-1).sum()) == 1


@pytest.mark.parametrize("hq,hk,d,rot,dt", SHAPES)
def test_a_weight_that_is_not_finite(hq, hk, d, rot, dt):
    def change(q, k, w):
        w[0][d - 1], w[1][d - 2] = float("inf"), float("nan")  # channels behind the rotated ones
    fine_q, fine_k = run(hq, hk, d, rot, dt, d + rot + 2, change)
    assert not bool(fine_q[..., d - 1].any()) and bool(fine_q[..., :d - 1].all())
    assert not bool(fine_k[..., d - 2].any()) and bool(fine_k[..., :d - 2].all())
