"""The four-bit cache of include/sla.h in plain torch, for its tests: rounding in 64 bits and the bytes of a plane."""
import numpy as np
import torch

SIGN, MAG = (15, 14, 7, 6), (0, 3, 8, 11)


def scales(a):
    """The smallest numbers of five significant bits, from 2^-40 on, with 7.5 s >= a; NaN from 2^40 on and where a is not finite."""
    table = torch.tensor([m * 2.0 ** e for e in range(-44, 36) for m in range(16, 32)] + [float("nan")], dtype=torch.float64, device=a.device)
    at = torch.searchsorted(7.5 * table[:-1], a.clamp(max=1e300))
    s = table[at.clamp(max=len(table) - 1)]
    return torch.where(torch.isfinite(a), s, float("nan"))


def quantise(x):
    """x [.., D] -> codes [.., D] (magnitudes with the sign of x: -0 is possible), scales [.., D / 32]."""
    g = x.double().unflatten(-1, (-1, 32))
    s = scales(g.abs().nan_to_num(nan=float("inf")).amax(-1))
    ok = ~torch.isnan(s)
    ratio = torch.where(ok[..., None], g.abs() / torch.where(ok, s, 1.0)[..., None], 0.0)
    whole = torch.floor(ratio)
    code = (whole + (ratio - whole >= 0.5)).clamp(max=7)
    code = torch.where(ok[..., None], torch.copysign(code, g), 0.0)
    return code.flatten(-2), s


def dequantise(codes, s):
    return (codes.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def held(x):
    return dequantise(*quantise(x))


def _unit_index(D, values):
    """For every dimension: 16-bit word of its row, and which of the four codes it is."""
    d = np.arange(D)
    n, g, c, i, h = D // 32, d // 32, d // 8 % 4, d // 2 % 4, d % 2
    return (2 * c + h) * n + g if values else 2 * (c * n + g) + h, i


def pack(codes, s, values):
    """[.., P, D], [.., P, D / 32] -> uint8 [.., plane]."""
    D = codes.shape[-1]
    unit, i = _unit_index(D, values)
    words = torch.zeros(*codes.shape[:-1], D // 4, dtype=torch.int64, device=codes.device)
    mag, neg = codes.abs().long(), torch.signbit(codes).long()
    for d in range(D):
        words[..., unit[d]] |= (mag[..., d] << MAG[i[d]]) | (neg[..., d] << SIGN[i[d]])
    rows = torch.stack([words & 255, words >> 8], -1).to(torch.uint8).flatten(-3)
    return torch.cat([rows, s.to(torch.bfloat16).contiguous().view(torch.uint8).flatten(-2)], -1)


def unpack(planes, P, D, values):
    """uint8 [.., plane] -> the values, fp64 [.., P, D]."""
    unit, i = _unit_index(D, values)
    b = planes[..., : P * D // 2].long().unflatten(-1, (P, D // 4, 2))
    words = b[..., 0] | b[..., 1] << 8
    s = planes[..., P * D // 2 :].contiguous().view(torch.bfloat16).double().unflatten(-1, (P, D // 32))
    u, sh_m, sh_s = (torch.as_tensor(a, device=planes.device) for a in (unit, np.array(MAG)[i], np.array(SIGN)[i]))
    w = words[..., u]
    code = (w >> sh_m & 7).double() * (1 - 2 * (w >> sh_s & 1)).double()
    return dequantise(code, s)
