"""pps_paged_attention at the longest sequences that 32-bit lengths can name: a table whose every entry is one page."""
import math

import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_attention import BF, F16, _cuda  # noqa: F401

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dt", [BF, F16])
@pytest.mark.parametrize("length", [2 ** 31 - 64, 2 ** 31 - 127, 2 ** 31 - 128, 2 ** 31 - 129])
def test_lengths_within_a_tile_of_2_31(length, dt):
    page, columns = 64, 2 ** 25 - 1
    kc = torch.randn(3, page, 1, 64, device="cuda").to(dt)
    vc = (torch.arange(64, device="cuda") % 3).to(dt).expand(3, page, 1, 64).contiguous()
    vc[2] = 1
    pages = torch.zeros(2, columns, **I32)
    pages[1] = 2
    q = torch.zeros(3, 2, 64, dtype=dt, device="cuda")  # all weights equal: sums are whole numbers below 2^24 per CTA
    status, lse = torch.zeros(1, **I32), torch.zeros(3, 2, device="cuda")
    out = pps.paged_attention(q, kc, vc, pages, torch.tensor([length, 70], **I32), torch.tensor([0, 1, 3], **I32), lse=lse,
                              status=status)
    longest = 2 ** 31 - 128  # beyond it lengths are cut
    assert int(status) == (pps.FLAG_INDEX if length > longest else 0)
    # the parts' sums are exact; 152 of them are added in fp32, twice 2^-24 each, and the result is rounded to 16 bits
    want = vc[0, 0].double().expand(2, 64)
    assert bool(((out[0].double() - want).abs() <= (2.0 ** -8 if dt is BF else 2.0 ** -11) * want).all())
    assert bool((lse[0].double() - math.log(min(length, longest))).abs().max() <= 2e-5 + 2.0 ** -22 * 22)
    assert bool((out[1:] == 1).all())
    assert bool((lse[1:].double() - torch.tensor([69.0, 70.0], device="cuda").log()[:, None]).abs().max() <= 1e-5)


def test_trees_behind_the_longest_prefix():
    page, columns = 64, 2 ** 25 - 1
    kc = torch.zeros(2, page, 1, 64, dtype=BF, device="cuda")
    vc = torch.ones(2, page, 1, 64, dtype=BF, device="cuda")
    pages = torch.zeros(1, columns, **I32)
    mask = torch.tensor([[1], [3]], **I32)
    status = torch.zeros(1, **I32)
    out = pps.paged_attention(torch.zeros(2, 1, 64, dtype=BF, device="cuda"), kc, vc, pages, torch.tensor([2 ** 31 - 64], **I32),
                              torch.tensor([0, 2], **I32), mask=mask, status=status)
    assert int(status) == pps.FLAG_INDEX and bool((out == 1).all())
