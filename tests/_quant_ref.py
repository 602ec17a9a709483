"""Plain form of a cache held in 8 or 4 bits, in numpy: codes and scales from the format's definition, in 64 bits.

Codes are compared for equality.  8 bits: the quotient is an fp32 number by definition.  4 bits: x / scale, x of at most 24 significant
bits, scale of five: for whole n with |n| <= 7, (2 n + 1) scale has at most nine bits, so 2 x - (2 n + 1) scale, if it is not zero, is
at least the last bit of 2 x.  Near n + 1/2 that is a relative difference of more than 2^-24 of the quotient, and rounding it to fp32
moves it by at most 2^-24: it stays on its side, and what is rounded half to even from the fp32 quotient is the same as from the real one.
max / 7 rounded to five bits: likewise, a tie needs max = 7 t with t of six bits, and max - 7 t is zero or at least the last bit of max.
"""
import numpy as np
import torch

TINY = 2.0 ** -110


def group(d):
    return (np.arange(d) // 4) % (d // 32)


def quantize(x, bits):
    """x [..., d] fp32 or fp64 numpy -> (whole codes [..., d], scales [...] or [..., d / 32]) as float64."""
    x = np.asarray(x, np.float64)
    d = x.shape[-1]
    if bits == 8:
        top = np.abs(x).max(-1)
        top = np.where(np.isfinite(x).all(-1), np.where(top < TINY, 0.0, top), np.nan)
        scale = (top.astype(np.float32) / np.float32(127)).astype(np.float64)
        per = scale[..., None]
    else:
        g = group(d)
        top = np.stack([np.where(np.isfinite(x[..., g == j]).all(-1), np.abs(x[..., g == j]).max(-1), np.nan) for j in range(d // 32)], -1)
        top = np.where(top < TINY, 0.0, top)
        m, e = np.frexp(np.where(np.isnan(top), 0.0, top) / 7)
        scale = np.where(np.isnan(top), np.nan, np.ldexp(np.rint(m * 32), e - 5))
        per = scale[..., g]
    good = per > 0
    quotient = np.where(good, x, 0.0) / np.where(good, per, 1.0)
    if bits == 8:
        quotient = (np.where(good, x, 0.0).astype(np.float32) / np.where(good, per, 1.0).astype(np.float32)).astype(np.float64)
    return np.rint(quotient), scale


def pack(codes, bits):
    if bits == 8:
        return codes.astype(np.int8)
    u = (codes + 8).astype(np.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def values(cache):
    """A cache's rows (CPU tensors of codes and scales) as float64 tensors."""
    got = []
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        c, s = codes.cpu().numpy(), scale.double().cpu().numpy()
        if c.dtype == np.int8:
            got.append(torch.from_numpy(c.astype(np.float64) * s[..., None]))
            continue
        x = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1).astype(np.float64) - 8
        got.append(torch.from_numpy(x * s[..., group(x.shape[-1])]))
    return got
