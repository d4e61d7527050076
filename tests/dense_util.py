"""Plain 64-bit forms of the dense operators, their error bounds, and guarded buffers for the tests."""
from __future__ import annotations

import numpy as np

ACTS = ["none", "relu", "sigmoid", "silu", "gelu"]
# half a unit in the last place of a value in [1, 2), and the smallest subnormal's half
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
F32 = 2.0 ** -24
FN = 2.0 ** -19  # activation functions in fp32: a few roundings of values that stay below 8 in these tests, generously


def torch_type(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def code(name):
    from paper_2407_04272_amd import binding as b
    return {"f32": b.F32, "f16": b.F16, "bf16": b.BF16}[name]


def philox_words(c, k):
    """Philox4x32-10 of counters c (four uint64 arrays below 2^32) and key k (two integers)."""
    c = [np.asarray(v, np.uint64) for v in c]
    k = list(k)
    m, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> sh) ^ c[1] ^ np.uint64(k[0]), p1 & m, (p0 >> sh) ^ c[3] ^ np.uint64(k[1]), p0 & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def drop_factor(rows, cols, p, seed, offset, row0=0):
    """What drop() multiplies rows row0 .. row0 + rows - 1 by, float64 [rows][cols]."""
    t = int(np.floor(p * 65536 + 0.5))
    offset &= (1 << 64) - 1
    nb = -(-cols // 8)
    r, cb = np.meshgrid(np.arange(row0, row0 + rows), np.arange(nb), indexing="ij")
    z = np.zeros_like(r)
    w = philox_words([cb, r, z + (offset & 0xFFFFFFFF), z + (offset >> 32)], (seed & 0xFFFFFFFF, seed >> 32))
    half = np.empty((rows, nb, 8), np.uint32)
    for i in range(4):
        half[:, :, 2 * i] = w[i] & np.uint64(0xFFFF)
        half[:, :, 2 * i + 1] = w[i] >> np.uint64(16)
    keep = half.reshape(rows, nb * 8)[:, :cols] >= t
    return keep * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def act(name, z):
    """value and slope, float64 tensors"""
    import torch
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "sigmoid":
        q = torch.sigmoid(z)
        return q, q * (1 - q)
    if name == "silu":
        q = torch.sigmoid(z)
        return z * q, q * (1 + z * (1 - q))
    if name == "gelu":
        q = 0.5 * torch.erfc(-z / 2 ** 0.5)
        return z * q, q + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5
    return z, torch.ones_like(z)


def product(a, b, ea=None):
    """a b' in 64 bits and a bound on the error of an fp32 sum of its terms; ea: a's relative error"""
    v = a @ b.t()
    mag = a.abs() @ b.abs().t()
    return v, mag * ((a.shape[1] + 2) * F32 + (ea or 0.0))


def rounded(v, err, dtype):
    """bound on the error after rounding to the type"""
    return err * (1 + 2 * ROUND[dtype]) + ROUND[dtype] * v.abs() + TINY[dtype]


class Guarded:
    """A [rows][cols] view inside a larger buffer: leading dimension ld, `shift` elements behind a 16-byte boundary, filled
    with a value (NaN by default) that must not be read into results, nor be overwritten."""

    def __init__(self, rows, cols, dtype, ld=None, shift=0, fill=float("nan")):
        import torch
        self.ld = ld or cols
        self.fill = fill
        n = 64 + shift + max(rows, 1) * self.ld + 64
        self.buf = torch.full((n,), fill, dtype=torch_type(dtype), device="cuda")
        self.view = self.buf[64 + shift:64 + shift + max(rows, 1) * self.ld].view(max(rows, 1), self.ld)[:rows, :cols]

    def set(self, values):
        self.view.copy_(values)
        return self

    def intact(self):
        """nothing outside the view was written"""
        import torch
        copy = self.buf.clone()
        lo = self.view.storage_offset()
        rows, cols = self.view.shape
        if rows:
            copy[lo:lo + rows * self.ld].view(rows, self.ld)[:, :cols] = self.fill
        return bool(torch.isnan(copy).all()) if self.fill != self.fill else bool((copy == self.fill).all())


def assert_close(got, want, bound, what):
    import torch
    d = (got.double() - want).abs()
    bad = ~(d <= bound)
    if bool(bad.any()):
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])} for "
                             f"{float(want[i])}, bound {float(bound[i])}")
    assert not bool(torch.isnan(got).any()), what
