"""The cache in 4 bits, restated in 64 bits from its definition (test helper)."""
import torch


def held(x, unit=None):
    """[..., heads, d] in 64 bits -> the codes' magnitudes' scales and values: (value, scale) in units of `unit` [heads]; z is
    formed in 32 bits as the definition has it."""
    if unit is None:
        z = x.float()
    else:
        z = x.float() * (1.0 / unit.float())[:, None]
    z = z.unflatten(-1, (-1, 16)).double()
    want = (z.abs().amax(-1, keepdim=True).float() / 6).clamp(max=448.0).double()
    step = 2.0 ** (torch.frexp(want).exponent - 1).clamp(min=-6).double() / 8
    scale = torch.round(want / step) * step
    m = torch.where(scale > 0, z / scale, 0.0).clamp(-6, 6)
    step = torch.where(m.abs() < 2, 0.5, torch.where(m.abs() < 4, 1.0, 2.0))
    fine = torch.isfinite(z).all(-1, keepdim=True)
    value = torch.where(fine, torch.round(m / step) * step * scale, float("nan"))
    return value.flatten(-2), torch.where(fine, scale, float("nan"))[..., 0]


def values(codes, scales, unit=None):
    """The values in 64 bits that codes and scales [..., heads, bytes] stand for."""
    nib = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2).long()
    e, m = (nib % 8) // 2, (nib % 2).double()
    x = torch.where(e == 0, m / 2, 2.0 ** (e - 1).double() * (1 + m / 2)) * (1 - 2 * (nib // 8))
    b = scales[..., :codes.shape[-1] // 8].long()
    e, m = (b % 128) // 8, (b % 8).double()
    s = torch.where(e == 0, m / 512, 2.0 ** (e - 7).double() * (1 + m / 8)) * (1 - 2 * (b // 128))
    s = torch.where(b % 128 == 127, float("nan"), s)
    v = (x.unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)
    return v if unit is None else v * unit.double()[:, None]
