"""A plain model of the paged cache's 8- and 4-bit formats, in numpy and 64 bits,
from their definition."""
import numpy as np
import torch

from tests.gpu_util import DEV

CODES = {8: torch.float8_e4m3fn, 4: torch.float4_e2m1fn_x2}
LEAST = -100                                   # exponent of the smallest scale stored


def code_values(bits):
    """Value of each code: sign, exponent (bias 7 or 1), mantissa (3 bits or 1)."""
    mantissa, bias = (3, 7) if bits == 8 else (1, 1)
    c = np.arange(1 << bits)
    sign = np.where(c >> (bits - 1), -1.0, 1.0)
    c = c & ((1 << (bits - 1)) - 1)
    e, m = c >> mantissa, (c & ((1 << mantissa) - 1)) / (1 << mantissa)
    v = sign * np.where(e > 0, (1 + m) * 2.0 ** (e - bias), m * 2.0 ** (1 - bias))
    if bits == 8:
        v[[127, 255]] = np.nan
    return v


def values(codes, scales, bits):
    """Elements that codes [..., dim] and scale bytes [..., dim / 32] stand for."""
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return code_values(bits)[codes] * np.repeat(s, 32, axis=-1)


def quantise(x, bits, dtype):
    """Codes and scale bytes of rows x [..., dim] that are of `dtype`."""
    table = code_values(bits)[:127 if bits == 8 else 8]        # not negative, rising
    top = table[-1]
    fi = torch.finfo(dtype)
    last = 2.0 ** np.floor(np.log2(fi.max))                    # the type's last power of two
    edge = last * max(v / 2.0 ** np.floor(np.log2(v)) for v in table[1:])
    b = x.astype(np.float64).reshape(*x.shape[:-1], -1, 32)
    odd = ~np.isfinite(b).all(-1)
    a = np.minimum(np.where(odd[..., None], 0.0, np.abs(b)), edge)
    high = a.max(-1)
    e = np.full(high.shape, LEAST)
    some = high > 0
    e[some] = np.maximum(LEAST, np.ceil(np.log2(high[some] / top)))
    y = a / 2.0 ** e[..., None]
    high_code = np.clip(np.searchsorted(table, y), 0, len(table) - 1)   # the first not below y
    low_code = np.maximum(high_code - 1, 0)
    to_low, to_high = y - table[low_code], table[high_code] - y
    best = np.where((to_high < to_low) | ((to_high == to_low) & (high_code % 2 == 0)), high_code,
                    low_code)
    code = best | (np.signbit(b) & ~odd[..., None]).astype(np.int64) << (bits - 1)
    return code.reshape(x.shape), np.where(odd, 255, e + 127)


def pack(codes, bits):
    """Bytes of codes [..., dim]."""
    if bits == 8:
        return codes.astype(np.uint8)
    return (codes[..., ::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(b, bits):
    b = b.astype(np.int64)
    return b if bits == 8 else np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)


def to_device(b, layout, dtype):
    """Bytes [pages][page][heads][width] as a GPU tensor of `dtype`: the heads of a
    slot side by side ("slots"), the slots of a head ("heads"), or with room between."""
    x = torch.from_numpy(np.ascontiguousarray(b).view(np.uint8)).to(DEV)
    if layout == "heads":
        x = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    elif layout == "padded":
        pages, page, heads, width = x.shape
        room = width if width % 16 else 16
        full = torch.full((pages, page + 1, heads, width + room), 0x7f, dtype=torch.uint8, device=DEV)
        full[:, :page, :, :width] = x
        x = full[:, :page, :, :width]
    return x.view(dtype)


def to_host(t):
    return t.view(torch.uint8).cpu().numpy()
