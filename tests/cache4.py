"""Rotation and 4-bit codes from their definitions, in double on the CPU, for the tests of the calls that bring rows into a cache."""
import torch

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def rotate(x, rows, interleaved):
    """x [T, heads, D] turned by the table's rows [T, dim], as float32: products of two float32 numbers are exact in double, their sum is
    rounded there and the result once more, which is what the library does."""
    x, rows = x.double().cpu(), rows.double().cpu()[:, None]
    half = rows.shape[2] // 2
    cos, sin = rows[..., :half], rows[..., half:]
    y = x.clone()
    at = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]] = a * cos - b * sin
    y[..., at[1]] = b * cos + a * sin
    return y.float()


def quantise(x):
    """(codes uint8 [..., D], scales bfloat16 [...]) of float32 x: the nearest level, ties to the even code, decided in double, where the
    distances of a number of 24 bits from a level times a scale of 8 bits are exact."""
    x = x.double().cpu()
    largest = x.abs().amax(dim=-1)
    odd = ~torch.isfinite(x).all(dim=-1)
    scale = torch.minimum(largest / 6, torch.tensor(1.328125 * 2.0 ** 125, dtype=torch.float64)).float().to(torch.bfloat16)
    unit = scale.double()[..., None]
    level = torch.tensor(LEVELS, dtype=torch.float64)
    off = (x.abs()[..., None] - level * unit[..., None]).abs()
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])                  # of two that are equally near the even one
    codes = order[off[..., order].argmin(dim=-1)]
    codes = torch.where(unit == 0, 0, codes + 8 * (x < 0))
    codes[odd], scale[odd] = 0, float("nan")
    return codes.to(torch.uint8), scale


def packed(codes):
    """Two codes a byte, the first in its low half, 16 bytes for 32 codes."""
    pad = torch.zeros((*codes.shape[:-1], -(-codes.shape[-1] // 32) * 32), dtype=torch.uint8)
    pad[..., :codes.shape[-1]] = codes
    return pad[..., 0::2] | (pad[..., 1::2] << 4)


def unpacked(x, D):
    return torch.stack([x & 15, x >> 4], dim=-1).flatten(-2)[..., :D]


def values(codes, scale):
    """What codes and scales stand for, in double."""
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64)
    s = scale.double()[..., None]
    return torch.where(torch.isfinite(s), level[codes.long()] * s, torch.nan)
