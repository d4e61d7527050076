"""Microscaled matrices for the tests: the oracle that quantises them, in numpy from the formats' tables, and what they stand for."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def e4m3_table():
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7.0), m / 8 * 2.0 ** -6)


TABLE = {4: E2M1, 8: e4m3_table()}


def filled(cols):
    return -(-cols // 128) * 128


def groups(cols):
    return -(-cols // 512)


def place(block):
    """where in [groups][rows][16] a block's scale stands: its group, its byte"""
    return block // 16, 4 * (block % 4) + block % 16 // 4


def quantise(x, bits):
    """x float64 [rows][cols] -> (elements uint8 [rows][row bytes], scales uint8 [groups][rows][16])"""
    rows, cols = x.shape
    wide = filled(cols)
    full = np.zeros((rows, wide))
    full[:, :cols] = x
    block = full.reshape(rows, -1, 32)
    table = TABLE[bits]
    top = np.abs(block).max(axis=2)                       # (a NaN comes through)
    fine = np.isfinite(top)
    e = np.full(top.shape, -127)
    t = np.where(fine, top, 0.0)
    for k in range(-126, 129):                            # the smallest exponent that fits
        e = np.where(t > table[-1] * 2.0 ** (k - 1), k, e)
    byte = np.where(fine, e + 127, 255).astype(np.uint8)
    scale = np.zeros((groups(cols), rows, 16), np.uint8)
    for b in range(-(-cols // 32)):
        g, at = place(b)
        scale[g, :, at] = byte[:, b]
    with np.errstate(invalid="ignore"):
        v = np.where(fine[:, :, None], block, 0.0) / 2.0 ** np.where(fine, e, 0)[:, :, None].astype(np.float64)
    a = np.abs(v).reshape(rows, wide)
    hi = np.searchsorted(table, a)                        # table[hi - 1] < a <= table[hi]
    lo = np.maximum(hi - 1, 0)
    hi = np.minimum(hi, len(table) - 1)
    down, up = a - table[lo], table[hi] - a
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code |= (np.signbit(v).reshape(rows, wide).astype(np.uint8)) << (bits - 1)
    code = np.where(np.repeat(fine, 32, axis=1), code, 0x7F if bits == 8 else 7).astype(np.uint8)
    if bits == 8:
        return code, scale
    return code[:, 0::2] | (code[:, 1::2] << 4), scale


def values(q, scale, cols, bits):
    """float64 [rows][cols]"""
    rows = q.shape[0]
    code = q if bits == 8 else np.stack((q & 15, q >> 4), axis=2).reshape(rows, -1)
    mag = code & (0x7F if bits == 8 else 7)
    table = np.append(TABLE[8], np.nan) if bits == 8 else TABLE[4]
    v = table[mag] * np.where(code >> (bits - 1), -1.0, 1.0)
    out = np.empty((rows, cols))
    for b in range(-(-cols // 32)):
        g, at = place(b)
        e = scale[g, :, at].astype(np.float64) - 127
        s = np.where(scale[g, :, at] == 255, np.nan, 2.0 ** e)
        out[:, 32 * b:32 * b + 32] = v[:, 32 * b:min(32 * b + 32, cols)] * s[:, None]
    return out


class GuardedBytes:
    """A contiguous uint8 tensor inside a larger one whose other bytes must not be written."""

    def __init__(self, shape, fill=0xA5):
        import torch
        n = int(np.prod(shape))
        self.fill, self.n = fill, n
        self.buf = torch.full((256 + n + 256,), fill, dtype=torch.uint8, device="cuda")
        self.view = self.buf[256:256 + n].view(shape)

    def intact(self):
        return bool((self.buf[:256] == self.fill).all()) and bool((self.buf[256 + self.n:] == self.fill).all())
