"""Plain 64-bit form of microscaled 4-bit quantisation (blocks of 32, power-of-two scales, E2M1
values), from the definition."""
import math

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantise(x):
    """(codes, biased scale exponents) of a matrix of finite or non-finite values: every value
    is compared with the whole grid, and the nearest wins, the even code of two as near."""
    a = x.double().cpu().unflatten(1, (-1, 32))
    big = a.abs().amax(-1)
    fine = torch.isfinite(big)
    _, ex = torch.frexp(torch.where(fine & (big > 0), big, torch.ones_like(big)))
    e = torch.where(big > 0, (ex - 3).clamp(min=-127), torch.full_like(ex, -127))
    e = torch.where(fine, e, torch.zeros_like(e))
    u = torch.where(fine[..., None], a.abs() * torch.exp2(-e.double())[..., None],
                    torch.zeros_like(a))
    off = (u[..., None] - GRID).abs()
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])          # even codes first: they win ties
    code = order[off[..., order].argmin(-1)]
    code = code + 8 * (torch.signbit(a) & fine[..., None])
    return code.flatten(1), torch.where(fine, e + 127, torch.full_like(e, 255))


def values(code, exps):
    v = torch.cat([GRID, -GRID])[code].unflatten(1, (-1, 32))
    scale = torch.where(exps == 255, torch.full_like(exps, 0).double() + math.nan,
                        torch.exp2(exps.double() - 127))
    return (v * scale[..., None]).flatten(1)


def dequantised(x):
    return values(*quantise(x))
