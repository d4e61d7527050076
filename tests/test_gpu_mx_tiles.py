"""The product of microscaled operands on each of its tiles, at sizes that take that tile (test_mx_plan.py asks the plan).

Most operands are hand-made: elements that stand for halves and whole numbers up to 6, scales of 1 and 2.  Products are whole numbers
of 2^-2 and of at most 144, so that sums of up to 12930 of them have fewer than 24 places: fp32 sums are exact in any order, E4M3
products lose nothing (a group's exponents lie less than 13 places apart), and a result is the exact one rounded once.  A fragment, a
scale or a tile of k values that is not the right one changes it."""
import pytest

from dense_util import ACTS, F32, FN, Guarded, act, assert_close, code, product, rounded, torch_type
from mx_util import CUTS, E2M1, KINDS, TILES, filled, groups, place

pytestmark = pytest.mark.gpu
# E4M3 times E2M1 with results of half precision: of eight products each loses less than 2^(E - 13), E the largest sum of two
# exponents; the largest is at least 2^(E - 1) (0.5 counts as 1 in E)
CUT = 7 * 2.0 ** -12
CODES = {4: [0, 1, 2, 3, 4, 5, 6, 7], 8: [0, 0x30, 0x38, 0x3C, 0x40, 0x44, 0x48, 0x4C]}     # of 0, 0.5, 1, 1.5, 2, 3, 4, 6


def _made(rows, cols, bits, seed, low=127, high=128):
    """A matrix in microscaled form, its filling as it has to be, and what it stands for (float64); all on the GPU."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def draw(n, shape):
        return torch.randint(0, n, shape, generator=g, device="cuda")

    wide, blocks = filled(cols), -(-cols // 32)
    which, sign = draw(8, (rows, wide)), draw(2, (rows, wide))
    which[:, cols:], sign[:, cols:] = 0, 0
    e = torch.tensor(CODES[bits], device="cuda")[which] | sign << (bits - 1)
    q = (e if bits == 8 else e[:, 0::2] | e[:, 1::2] << 4).to(torch.uint8)
    byte = low + draw(high - low + 1, (rows, blocks))
    return q.contiguous(), _placed(byte, rows, cols), _stands(which, sign, byte, cols)


def _placed(byte, rows, cols):
    """[rows][blocks] -> [groups][rows][16]"""
    import torch
    s = torch.zeros((groups(cols), rows, 16), dtype=torch.uint8, device="cuda")
    for k in range(byte.shape[1]):
        g, at = place(k)
        s[g, :, at] = byte[:, k].to(torch.uint8)
    return s


def _powers(byte, cols):
    """2^(byte - 127) for every column, from its bits (a power on the GPU may be off by a last place)"""
    import torch
    return (byte.long() + (1023 - 127) << 52).view(torch.float64).repeat_interleave(32, dim=1)[:, :cols]


def _stands(which, sign, byte, cols):
    import torch
    v = torch.tensor(E2M1, device="cuda")[which] * (1.0 - 2.0 * sign.double())
    return v[:, :cols] * _powers(byte, cols)


def _call(bits, dtype, xq, xs, wq, ws, n_in, bias=None, residual=None, act_name="none", y=None, ld=0):
    import torch
    from paper_2407_04272_amd import binding as b
    rows, n_out = xq.shape[0], wq.shape[0]
    cfg = b.make_mx_linear_config(code(dtype), bits, rows, n_in, n_out, act=ACTS.index(act_name), ld_y=ld, ld_res=ld if residual is not None and y is residual else 0)
    y = torch.full((rows, n_out), float("nan"), dtype=torch_type(dtype), device="cuda") if y is None else y
    work = torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    b.dlc_mx_linear_forward(cfg, xq, xs, wq, ws, bias, residual, y, work)
    return y


def _cases(table, lengths=None):
    return [pytest.param(kind, dtype, rows, n_in, n_out, id=f"{kind}-{dtype}-tile{tile}-cut{split}-{rows}x{n_in}-{n_out}".replace(" ", ""))
            for kind, tile, split, rows, n_out, ls in table for dtype in KINDS[kind][1] for n_in in (ls if lengths is None else lengths(ls))]


EVERY = pytest.mark.parametrize("kind,dtype,rows,n_in,n_out", _cases(TILES) + _cases(CUTS))
LONG = [t for t in TILES if t[3] != 498]
ONE_OF = _cases(LONG, lambda ls: [n for n in ls if n in (1300, 1800)]) + _cases(CUTS)
ONE = pytest.mark.parametrize("kind,dtype,rows,n_in,n_out", ONE_OF)


@EVERY
def test_whole_numbers(kind, dtype, rows, n_in, n_out):
    import torch
    bits = KINDS[kind][0]
    (xq, xs, x), (wq, ws, w) = _made(rows, n_in, bits, n_in), _made(n_out, n_in, 4, n_in + 1)
    y = Guarded(rows, n_out, dtype, ld=n_out + 3, shift=1)
    _call(bits, dtype, xq, xs, wq, ws, n_in, y=y.view, ld=n_out + 3)
    assert torch.equal(y.view, (x @ w.t()).to(torch_type(dtype))) and y.intact()


@ONE
def test_nan_blocks(kind, dtype, rows, n_in, n_out):
    """A block of x whose scale is NaN makes its row NaN, one of w its column, and nothing else: rows and columns at the borders of
    wavefronts and tiles and the last ones, blocks of the first group, the last block, which may have few elements."""
    import torch
    bits = KINDS[kind][0]
    (xq, xs, x), (wq, ws, w) = _made(rows, n_in, bits, 5), _made(n_out, n_in, 4, 6)
    last = (n_in - 1) // 32
    bad = []
    for s, n in ((xs, rows), (ws, n_out)):
        at = sorted({0, 15, 31, 64, 127, n // 2, n - 1} & set(range(n)))
        for i, row in enumerate(at):
            g, k = place([0, last, 7, last // 2, 13][i % 5])
            s[g, row, k] = 255
        bad.append(torch.tensor(at, device="cuda"))
    y = _call(bits, dtype, xq, xs, wq, ws, n_in)
    want = x @ w.t()
    want[bad[0]] = float("nan")
    want[:, bad[1]] = float("nan")
    want = want.to(torch_type(dtype))
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))


@ONE
def test_scales_from_end_to_end(kind, dtype, rows, n_in, n_out):
    """2^-127 against 2^127, and the other way round: the same whole numbers, times one power of two.  (E4M3 with results in fp32: from
    2^-112 on every element is one that counts.)"""
    import torch
    bits = KINDS[kind][0]
    (xq, xs, x), (wq, ws, w) = _made(rows, n_in, bits, 7, 127, 127), _made(n_out, n_in, 4, 8, 127, 127)
    one = x @ w.t()
    for a, c in ((15 if kind == "E4M3 f32" else 0, 250), (246, 4), (100, 150)):
        xa, wc = (torch.where(s > 0, torch.full_like(s, v), s) for s, v in ((xs, a), (ws, c)))
        y = _call(bits, dtype, xq, xa, wq, wc, n_in)
        assert torch.equal(y, (one * 2.0 ** (a + c - 254)).to(torch_type(dtype))), (a, c)


@ONE
def test_scales_far_apart(kind, dtype, rows, n_in, n_out):
    """Blocks of one row 2^24 apart.  Elements of a block are as they were: no product of a group of eight loses anything."""
    bits = KINDS[kind][0]
    (xq, xs, x), (wq, ws, w) = _made(rows, n_in, bits, 9, 103, 127), _made(n_out, n_in, 4, 10, 103, 127)
    v, e = product(x, w)
    assert_close(_call(bits, dtype, xq, xs, wq, ws, n_in), v, rounded(v, e, dtype), "far apart")


@pytest.mark.parametrize("kind,dtype,rows,n_in,n_out", [c for c in ONE_OF if c.values[0] != "E2M1"])
def test_elements_far_apart(kind, dtype, rows, n_in, n_out):
    """All codes of E4M3, subnormal ones among them: the half types lose what the scaled instruction cuts, fp32 nothing."""
    import torch
    (xq, xs, _), (wq, ws, w) = _made(rows, n_in, 8, 11), _made(n_out, n_in, 4, 12, 119, 120)
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    table = torch.cat([torch.arange(127, device="cuda"), torch.arange(128, 255, device="cuda")])
    q = table[torch.randint(0, 254, xq.shape, generator=g, device="cuda")].to(torch.uint8)
    q[:, n_in:] = 0
    byte = torch.stack([xs[place(k)[0], :, place(k)[1]] for k in range(-(-n_in // 32))], dim=1)
    x = q[:, :n_in].contiguous().view(torch.float8_e4m3fn).double() * _powers(byte, n_in)
    v, e = product(x, w)
    if dtype != "f32":
        e = e + CUT * (x.abs() @ w.abs().t())
    y = _call(8, dtype, q, xs, wq, ws, n_in)
    assert_close(y, v, rounded(v, e, dtype), "all codes")
    half = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    # (in the norm cut products of random signs are far below a rounding)
    assert float((y.double() - v).norm()) <= (half + 2.0 ** -12 * (dtype != "f32") + (n_in + 2) * F32) * float(v.norm())


@ONE
def test_epilogue(kind, dtype, rows, n_in, n_out):
    """Bias, every activation, a residual, in place too.  Scales are small, so that activations bend."""
    import torch
    bits, ty = KINDS[kind][0], torch_type(dtype)
    (xq, xs, x), (wq, ws, w) = _made(rows, n_in, bits, 14, 123, 124), _made(n_out, n_in, 4, 15, 122, 123)
    g = torch.Generator(device="cuda")
    g.manual_seed(16)
    bias, res = (torch.randn(s, generator=g, device="cuda").to(ty) for s in ((n_out,), (rows, n_out)))
    z = x @ w.t() + bias.double()       # (exact sums; the bias' addition is rounded in fp32)
    ez = z.abs() * F32
    for name in ACTS:
        v, _ = act(name, z)
        err = ez if name == "none" else 1.13 * ez + FN * (1 + v.abs())   # (slopes of these functions stay below 1.13)
        assert_close(_call(bits, dtype, xq, xs, wq, ws, n_in, bias, None, name), v, rounded(v, err, dtype), name)
        v = v + res.double()
        err = err + v.abs() * F32
        y = Guarded(rows, n_out, dtype, ld=n_out + 5, shift=1).set(res)
        _call(bits, dtype, xq, xs, wq, ws, n_in, bias, y.view, name, y.view, n_out + 5)
        assert_close(y.view, v, rounded(v, err, dtype), f"{name} in place")
        assert y.intact()
        other = _call(bits, dtype, xq, xs, wq, ws, n_in, bias, res, name)
        assert torch.equal(other, y.view)


@ONE
def test_the_same_every_time(kind, dtype, rows, n_in, n_out):
    """Calls on other data in between: nothing is left from one for the next, and sums do not depend on the run."""
    import torch
    bits = KINDS[kind][0]
    a = [_made(rows, n_in, bits, s)[:2] + _made(n_out, n_in, 4, s + 1)[:2] for s in (17, 19)]
    ys = [torch.empty((rows, n_out), dtype=torch_type(dtype), device="cuda") for _ in a]
    want = [_call(bits, dtype, *v, n_in).clone() for v in a]
    for _ in range(3):
        for v, y, c in zip(a, ys, want):
            y.fill_(float("nan"))
            _call(bits, dtype, *v, n_in, y=y)
        assert all(torch.equal(y, c) for y, c in zip(ys, want))
