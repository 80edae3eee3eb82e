"""Block-scaled rows in float64: what include/pvf.h says of their format, written element by element (CPU tensors)."""
import torch

E4M3, E2M1 = 0, 1
TOP = {E4M3: 448.0, E2M1: 6.0}
E2M1_VALUES = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def width(K):
    return (K + 127) // 128 * 128


def e4m3_table():
    """The 127 magnitudes by code."""
    v = []
    for c in range(127):
        e, m = c >> 3, c & 7
        v.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return torch.tensor(v, dtype=torch.float64)


def nearest(mag, table):
    """Code of the nearest magnitude, ties to the even code."""
    hi = torch.searchsorted(table, mag.contiguous()).clamp(max=len(table) - 1)
    lo = (hi - 1).clamp(min=0)
    d_lo, d_hi = mag - table[lo], table[hi] - mag
    take_lo = (d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0))
    return torch.where(take_lo, lo, hi)


def quantise(x, fmt):
    """(codes [M, Kp] one a byte, scale bytes [M, Kp / 32]) of float64 rows x [M, K]."""
    M, K = x.shape
    b = torch.zeros(M, width(K), dtype=torch.float64)
    b[:, :K] = x
    b = b.view(M, -1, 32)
    bad = ~torch.isfinite(b).all(2)
    amax = torch.where(bad[:, :, None], torch.zeros_like(b), b).abs().amax(2)
    byte = torch.zeros(amax.shape, dtype=torch.int64)
    for e in range(-127, 128):                                  # the smallest power with amax <= top 2^e
        byte += (amax > TOP[fmt] * 2.0 ** e).long()
    v = torch.where(bad[:, :, None], torch.zeros_like(b), b) / torch.pow(2.0, (byte - 127).double())[:, :, None]
    table = e4m3_table() if fmt == E4M3 else E2M1_VALUES[:8].clone()
    codes = nearest(v.abs(), table) + (torch.signbit(v).long() << (7 if fmt == E4M3 else 3))
    byte[bad] = 255
    return codes.view(M, -1), byte


def values(codes, byte, fmt):
    """float64 rows of codes (one an element) and scale bytes."""
    if fmt == E4M3:
        v = torch.cat([e4m3_table(), torch.tensor([float("nan")], dtype=torch.float64)])[codes & 127] * torch.where(codes >= 128, -1.0, 1.0)
    else:
        v = E2M1_VALUES[codes]
    s = torch.pow(2.0, (byte - 127).double())
    s[byte == 255] = float("nan")
    return v * s.repeat_interleave(32, 1)


def unpack(codes, scales, fmt):
    """(codes one an element, scale bytes [M, Kp / 32]) of device tensors as the library lays them out."""
    c = codes.view(torch.uint8).cpu().long()
    if fmt == E2M1:
        c = torch.stack((c & 15, c >> 4), 2).view(c.shape[0], -1)
    return c, scales.view(torch.uint8).cpu().long().transpose(0, 1).reshape(scales.shape[1], -1)


def pack(codes, byte, fmt, device="cuda"):
    """Device tensors of codes and scale bytes."""
    c = codes.to(torch.uint8)
    c = c.view(torch.float8_e4m3fn) if fmt == E4M3 else c[:, 0::2] | (c[:, 1::2] << 4)
    s = byte.to(torch.uint8).view(byte.shape[0], -1, 4).transpose(0, 1).contiguous().view(torch.float8_e8m0fnu)
    return c.contiguous().to(device), s.to(device)
