"""pps_kv_append with the queries' own memory as its output, with several times the tokens that are in work at once."""
import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_append import BF, F16, _cuda, _inputs  # noqa: F401
from test_gpu_append_unread import N, SHAPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,d,rot,dt", SHAPES + [(32, 8, 128, 128, BF), (14, 2, 64, 32, F16), (20, 4, 80, 80, BF)])
def test_queries_in_place(hq, hk, d, rot, dt):
    g, q, k, v = _inputs(N, hq, hk, d, dt, d + rot + 3)
    w = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt)
    rope = pps.rope_table(500, rot) if rot else None
    pos = torch.randint(0, 500, (N,), generator=g, device="cuda", dtype=torch.int32)
    caches = [torch.zeros(N // 16, 16, hk, d, dtype=dt, device="cuda") for _ in range(4)]
    slot = torch.arange(N, device="cuda")
    want = pps.kv_append(q, k, v, pos, slot, *caches[:2], rope, w, w)
    got = pps.kv_append(q, k, v, pos, slot, *caches[2:], rope, w, w, out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want)
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
