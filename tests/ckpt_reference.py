"""The 8-bit checkpoint format from its definition, on integers and in 64 bits."""
import numpy as np
import torch


def held(x):
    """bf16 [..., d] -> int8 values, exponent bytes; runs with infinities or NaN get 255 (their values do not matter)."""
    bits = x.contiguous().view(torch.int16).numpy().view(np.uint16).astype(np.int64) & 0x7fff
    field = bits.reshape(*x.shape[:-1], -1, 32).max(-1) >> 7
    e = np.maximum(field, 7)
    y = x.double().numpy().reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore"):
        q = np.clip(np.rint(np.ldexp(y, (133 - e)[..., None])), -127, 127)     # np.rint: ties to even
    q = np.where((e == 255)[..., None], 0, q)
    return q.reshape(x.shape).astype(np.int8), e.astype(np.uint8)


def value(q, e):
    """What they stand for, fp64; NaN for runs marked 255."""
    y = np.ldexp(q.astype(np.float64).reshape(*e.shape, 32), (e.astype(np.int64) - 133)[..., None])
    return np.where((e == 255)[..., None], np.nan, y).reshape(q.shape)
