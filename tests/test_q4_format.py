"""The restatement of the cache in 4 bits against the formats' own definitions (no GPU)."""
import torch

from q4_format import held, values


def test_every_code_and_scale_stands_for_its_number():
    codes = torch.arange(256, dtype=torch.uint8)
    one = torch.tensor([0x38], dtype=torch.uint8)  # e4m3: 1
    v = values(codes.view(32, 1, 8), one.expand(32, 1, 4))
    table = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    table += [-x for x in table]
    assert v.flatten().tolist() == [float(table[n]) for c in range(256) for n in (c % 16, c // 16)]
    s = torch.arange(256, dtype=torch.uint8)
    got = values(torch.full((256, 1, 8), 0x22, dtype=torch.uint8), s.view(256, 1, 1))[:, 0, 0]
    want = s.view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_rounding_to_nearest_even_and_saturation():
    x = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -5, 0.2500001, 4.9999995, 0, 1, 2, 3], dtype=torch.float64)
    v, s = held(x.view(1, 1, 16))
    assert s.item() == 1
    assert v.flatten().tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -4, 0.5, 4, 0, 1, 2, 3]
    v, s = held((x * 1e6).view(1, 1, 16))  # beyond the scales
    assert s.item() == 448 and v.max().item() == 2688
    v, s = held((x / 6 * 6 * 2.0 ** -10.01).view(1, 1, 16))  # scale rounds to the smallest or to zero
    assert s.item() in (0.0, 2.0 ** -9)
    x[3] = float("inf")
    assert bool(torch.isnan(held(x.view(1, 1, 16))[0]).all())
