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


# ---- the product's kernels ------------------------------------------------------------------------
# Sizes that the plan sends to a tile (0: 256 x 256, 1: 128 x 128, 2: 64 x 128; 3: a pass over the weights for bands of 32 rows), for
# (element bits of x, results in fp32): "E2M1" any type, "E4M3" half precision, "E4M3 f32".  A name, its tile, in how many parts k
# is cut, rows, out_features, and in_features: numbers of tiles of 256 k values (or steps of 128) from one to nine, k that ends in
# each half of a tile and inside a step, edges in rows and columns.  test_mx_plan.py asks the plan itself.
LENGTHS = (1, 100, 129, 256, 300, 512, 600, 700, 800, 1000, 1100, 1300, 1536, 1700, 2000, 2300)
TILES = [
    ("E2M1", 0, 1, 3338, 3606, LENGTHS),
    ("E2M1", 1, 1, 4173, 402, (1700, 1800, 2100, 2400, 2600, 3000)),
    ("E2M1", 2, 1, 65, 2745, LENGTHS),
    ("E2M1", 2, 1, 498, 585, (100, 640, 900)),
    ("E4M3", 0, 1, 4724, 1668, LENGTHS),
    ("E4M3", 1, 1, 4173, 402, LENGTHS),
    ("E4M3", 2, 1, 65, 2745, LENGTHS),
    ("E4M3", 2, 1, 498, 585, (100, 640, 900)),
    ("E4M3 f32", 1, 1, 4173, 402, LENGTHS),
    ("E4M3 f32", 2, 1, 132, 3606, LENGTHS),
]
CUTS = [
    ("E2M1", 0, 3, 1929, 2263, (12930,)),
    ("E2M1", 1, 5, 1929, 295, (9231,)),
    ("E2M1", 2, 4, 1000, 257, (8192,)),
    ("E2M1", 2, 6, 1300, 200, (8000,)),
    ("E4M3", 0, 3, 1929, 2263, (9231,)),
    ("E4M3", 1, 3, 4097, 130, (8192,)),
    ("E4M3", 1, 5, 983, 734, (9231,)),
    ("E4M3", 2, 4, 33, 4097, (4096,)),
    ("E4M3", 2, 8, 65, 1537, (8100,)),
    ("E4M3 f32", 1, 5, 784, 734, (4702,)),
    ("E4M3 f32", 1, 4, 2047, 257, (4096,)),
    ("E4M3 f32", 2, 4, 300, 1300, (1700,)),
]
KINDS = {"E2M1": (4, ("f32", "f16", "bf16")), "E4M3": (8, ("f16", "bf16")), "E4M3 f32": (8, ("f32",))}
