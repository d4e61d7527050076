"""Microscaled form: quantisation and back bit for bit against the oracle, the product against 64 bits."""
import numpy as np
import pytest

from dense_util import ACTS, F32, FN, ROUND, Guarded, act, assert_close, code, product, rounded, torch_type
from mx_util import GuardedBytes, TABLE, quantise, values

pytestmark = pytest.mark.gpu
TYPES = ["f32", "f16", "bf16"]


def _matrix(rows, cols, dtype, seed, kind="normal"):
    """values of the type, as a float64 array and a tensor"""
    import torch
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, dtype=torch.float64)
    if kind == "wide":      # magnitudes from far below to far above one
        x = x * 2.0 ** torch.randint(-14, 14, (rows, cols), generator=g).double()
    t = x.to(torch_type(dtype))
    return t.double().numpy(), t.cuda()


def _quantised(x, bits, dtype, ld=None):
    from paper_2407_04272_amd import binding as b
    rows, cols = x.shape
    cfg = b.make_mx_config(code(dtype), bits, rows, cols, ld_x=ld or 0)
    q, s = GuardedBytes(b.dlc_mx_data_shape(cfg)), GuardedBytes(b.dlc_mx_scale_shape(cfg))
    b.dlc_mx_quantize(cfg, x, q.view, s.view)
    assert q.intact() and s.intact()
    return q.view, s.view


def _same(q, s, want_q, want_s, what):
    assert np.array_equal(s.cpu().numpy(), want_s), f"{what}: scales"
    assert np.array_equal(q.cpu().numpy(), want_q), f"{what}: elements"


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (17, 33), (5, 128), (16, 129), (15, 511), (33, 512), (2, 513), (70, 1664), (1, 4097)])
def test_quantise(rows, cols, dtype, bits):
    for kind in ("normal", "wide"):
        x, t = _matrix(rows, cols, dtype, rows * 7 + cols, kind)
        _same(*_quantised(t, bits, dtype), *quantise(x, bits), f"{kind} {rows}x{cols}")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_rows_apart(dtype, bits):
    for shift in (0, 1, 3):
        x, t = _matrix(9, 300, dtype, 5 + shift)
        v = Guarded(9, 300, dtype, ld=317, shift=shift).set(t)
        _same(*_quantised(v.view, bits, dtype, 317), *quantise(x, bits), f"shift {shift}")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_borders(dtype, bits):
    """Blocks whose largest magnitude is at, just below and just above the largest value times a power of two, ties between
    elements, zeros of both signs, the type's smallest and largest values, NaN and infinities."""
    import torch
    ty = torch_type(dtype)
    fin = torch.finfo(ty)
    top = 448.0 if bits == 8 else 6.0
    ulp = float(fin.eps)
    rows = []
    for e in (-10, -1, 0, 3, 6):
        for m in (top, top * (1 - ulp), top * (1 + ulp), top / 2, top * 0.75, top * 0.7500001, 1.0):
            rows.append([m * 2.0 ** e] + [m * 2.0 ** e * f for f in (0.5, -0.25, 1 / 3, -1 / 28, 0.01, 0.001, -1e-4)])
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] if bits == 4 else [17.0, 19.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 432.0, 208.0]
    rows.append([top] + [t for t in ties[:7]])
    rows.append([-top] + [-t for t in ties[-7:]])
    rows.append([0.0, -0.0, 0.0, -0.0, 0.0, 0.0, 0.0, -0.0])
    rows.append([fin.tiny, fin.smallest_normal / 2, -fin.tiny, fin.tiny * 3, 0.0, -0.0, fin.tiny, fin.tiny])
    rows.append([float(fin.smallest_normal) * ulp, 0, 0, 0, 0, 0, -float(fin.smallest_normal) * ulp, 0])
    rows.append([fin.max, -fin.max, fin.max / 2, 1.0, fin.tiny, 0, 0, 0])
    for bad in (float("nan"), float("inf"), -float("inf")):
        rows.append([1.0, 2.0, bad, 3.0, 0, 0, -1.0, 0])
    x = torch.zeros((len(rows), 96), dtype=torch.float64)
    for i, r in enumerate(rows):
        x[i, 40:48] = torch.tensor(r, dtype=torch.float64)    # (the second of three blocks)
        x[i, 3] = 1.0
    t = x.to(ty)
    q, s = _quantised(t.cuda(), bits, dtype)
    _same(q, s, *quantise(t.double().numpy(), bits), "borders")
    assert s[0, -1].cpu().tolist().count(255) == 1


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,ld", [(1, 1, 0), (19, 333, 0), (7, 1030, 1039)])
def test_back(rows, cols, ld, dtype, bits):
    """Any codes and scales: every element's value is exact in 64 bits and rounded once."""
    import torch
    from paper_2407_04272_amd import binding as b
    rng = np.random.default_rng(rows + cols)
    cfg = b.make_mx_config(code(dtype), bits, rows, cols, ld_y=ld)
    q = rng.integers(0, 256, b.dlc_mx_data_shape(cfg), dtype=np.uint8)
    s = rng.integers(127 - 20, 127 + 20, b.dlc_mx_scale_shape(cfg), dtype=np.uint8)
    if rows > 1:
        s[:, 1] = rng.integers(0, 256, s[:, 1].shape, dtype=np.uint8)      # far scales: subnormal, infinite, NaN
    y = Guarded(rows, cols, dtype, ld=ld or None)
    b.dlc_mx_dequantize(cfg, torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), y.view)
    with np.errstate(all="ignore"):
        want = torch.from_numpy(values(q, s, cols, bits))
    # (a value past fp32's range is an infinity on the way, as it is in the type)
    assert torch.equal(y.view.cpu().nan_to_num(nan=-7.0), want.to(torch_type(dtype)).nan_to_num(nan=-7.0))
    assert y.intact() or bool(torch.isnan(y.view).any())


def test_no_rows():
    import torch
    from paper_2407_04272_amd import binding as b
    cfg = b.make_mx_config(b.F32, b.MX_E2M1, 0, 40)
    q, s = (torch.empty(shape, dtype=torch.uint8, device="cuda") for shape in (b.dlc_mx_data_shape(cfg), b.dlc_mx_scale_shape(cfg)))
    x = torch.empty((0, 40), device="cuda")
    b.dlc_mx_quantize(cfg, x, q, s)
    b.dlc_mx_dequantize(cfg, q, s, x)
    w = torch.zeros((24, 64), dtype=torch.uint8, device="cuda")
    b.dlc_mx_linear_forward(b.make_mx_linear_config(b.F32, b.MX_E2M1, 0, 40, 24), q, s, w, torch.zeros((1, 24, 16), dtype=torch.uint8, device="cuda"),
                            None, None, torch.empty((0, 24), device="cuda"))


# ---- the product --------------------------------------------------------------------------------
# E4M3 times E2M1 with results of half precision: of eight products each loses less than 2^-13 of the largest one, which itself
# loses nothing
CUT = 7 * 2.0 ** -13


def _operand(rows, cols, bits, seed, spread=2.0):
    """a matrix in microscaled form (on the GPU) and what it stands for (float64, on the GPU)"""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-spread, spread + 1, (rows, cols)))
    q, s = quantise(x.astype(np.float32).astype(np.float64), bits)
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), torch.from_numpy(values(q, s, cols, bits)).cuda()


def _linear(rows, n_in, n_out, bits, dtype, act_name="none", bias=False, residual=False, ld=0, seed=1, inplace=False):
    import torch
    from paper_2407_04272_amd import binding as b
    xq, xs, x = _operand(rows, n_in, bits, seed)
    wq, ws, w = _operand(n_out, n_in, 4, seed + 1)
    ty = torch_type(dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    cfg = b.make_mx_linear_config(code(dtype), bits, rows, n_in, n_out, act=ACTS.index(act_name), ld_y=ld, ld_res=ld if inplace else 0)
    vb = torch.randn((n_out,), generator=g, device="cuda").to(ty) if bias else None
    vr = torch.randn((rows, n_out), generator=g, device="cuda").to(ty) if residual else None
    y = Guarded(rows, n_out, dtype, ld=ld or None, shift=1 if ld else 0)
    res = vr
    if inplace:
        y.set(vr)
        res = y.view
    work = torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    b.dlc_mx_linear_forward(cfg, xq, xs, wq, ws, vb, res, y.view, work)
    assert y.intact()
    z, ez = product(x, w)
    if bits == 8 and dtype != "f32":
        ez = ez + CUT * (x.abs() @ w.abs().t())
    if bias:
        z = z + vb.double()
        ez = ez + z.abs() * F32
    v, _ = act(act_name, z)
    # slopes of these functions stay below 1.13
    err = ez if act_name == "none" else 1.13 * ez + FN * (1 + v.abs())
    if residual:
        v = v + vr.double()
        err = err + v.abs() * F32
    what = f"{rows}x{n_in}->{n_out} {bits} {dtype} {act_name}"
    assert_close(y.view, v, rounded(v, err, dtype), what)
    # in the norm the cut products of random signs are far below a rounding
    if rows * n_out >= 1000:
        assert float((y.view.double() - v).norm()) <= (ROUND[dtype] + 2.0 ** -12 * (bits == 8 and dtype != "f32") + (n_in + 2) * F32) * float(v.norm()), what


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 1, 1), (1, 1664, 1024), (2, 33, 17), (7, 128, 16), (16, 8192, 96), (17, 129, 65), (31, 513, 40),
                                             (33, 640, 130), (64, 1024, 64), (65, 2049, 127), (130, 259, 513), (300, 512, 260), (777, 515, 1023)])
def test_product(rows, n_in, n_out, dtype, bits):
    _linear(rows, n_in, n_out, bits, dtype, seed=rows + n_in)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,n_in,n_out", [(512, 4096, 512), (1024, 1664, 1280), (257, 8192, 2048), (2048, 768, 2304)])
def test_large_product(rows, n_in, n_out, bits):
    _linear(rows, n_in, n_out, bits, "f32", seed=3)
    _linear(rows, n_in, n_out, bits, "bf16", "relu", bias=True, residual=True, seed=4)


@pytest.mark.parametrize("act_name", ACTS)
@pytest.mark.parametrize("rows", [1, 20, 100, 600])
def test_epilogue(rows, act_name):
    for dtype in TYPES:
        _linear(rows, 96, 200, 8, dtype, act_name, bias=True, residual=True, seed=9)
        _linear(rows, 96, 201, 4, dtype, act_name, bias=True, ld=219, seed=10)


@pytest.mark.parametrize("rows", [1, 40, 513])
def test_residual_in_place(rows):
    for dtype in TYPES:
        _linear(rows, 200, 72, 4, dtype, "relu", residual=True, ld=88, inplace=True)


def test_exact_sums():
    """Small whole numbers: every product and sum is exact in fp32, and so is the result, whatever the order."""
    import torch
    from paper_2407_04272_amd import binding as b
    rng = np.random.default_rng(2)
    for rows, n_in, n_out in ((5, 700, 90), (40, 3000, 70), (600, 1100, 600)):
        for bits in (4, 8):
            x = rng.choice([-2.0, -1.0, 0.0, 1.0, 2.0, 4.0], (rows, n_in))
            w = rng.choice([-1.0, 0.0, 1.0, 3.0], (n_out, n_in))
            (xq, xs), (wq, ws) = quantise(x, bits), quantise(w, 4)
            y = torch.empty((rows, n_out), device="cuda")
            cfg = b.make_mx_linear_config(b.F32, bits, rows, n_in, n_out)
            work = torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
            b.dlc_mx_linear_forward(cfg, *(torch.from_numpy(v).cuda() for v in (xq, xs, wq, ws)), None, None, y, work)
            assert np.array_equal(y.cpu().numpy(), (x @ w.T).astype(np.float32))


@pytest.mark.parametrize("rows", [1, 24, 200, 600])
def test_scales_far_apart_and_nan(rows):
    """Blocks of one row whose scales are far apart; a NaN block makes its row (of x) or column (of w) NaN and no other."""
    import torch
    from paper_2407_04272_amd import binding as b
    n_in, n_out = 1200, 48
    for bits in (4, 8):
        xq, xs, x = _operand(rows, n_in, bits, 21, spread=12)
        wq, ws, w = _operand(n_out, n_in, 4, 22, spread=12)
        if rows > 1:
            xs[1, 1, 5] = 255
        ws[0, 7, 9] = 255
        y = torch.empty((rows, n_out), device="cuda")
        cfg = b.make_mx_linear_config(b.F32, bits, rows, n_in, n_out)
        work = torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        b.dlc_mx_linear_forward(cfg, xq, xs, wq, ws, None, None, y, work)
        nan = torch.zeros_like(y, dtype=torch.bool)
        nan[:, 7] = True
        if rows > 1:
            nan[1] = True
        assert torch.equal(torch.isnan(y), nan)
        v, e = product(x, w)
        keep = ~nan
        assert_close(y[keep], v[keep], rounded(v, e, "f32")[keep], f"{rows} {bits}")


@pytest.mark.parametrize("rows", [3, 50, 300])
@pytest.mark.parametrize("bits", [4, 8])
def test_values_below_the_normal_range(rows, bits):
    """Scales down to 2^-127, whose elements are below fp32's normal numbers, times weights large enough that the results are
    not.  E4M3 with results in fp32 may take each value below 2^-126 for 0; nothing else is lost anywhere."""
    import torch
    from paper_2407_04272_amd import binding as b
    n_in, n_out = 600, 40
    rng = np.random.default_rng(31)
    x = rng.standard_normal((rows, n_in)) * np.exp2(rng.integers(-133, -118, (rows, n_in // 50)).repeat(50, axis=1).astype(float))
    w = rng.standard_normal((n_out, n_in)) * np.exp2(rng.integers(70, 90, (n_out, n_in)).astype(float))
    (xq, xs), (wq, ws) = quantise(x, bits), quantise(w, 4)
    assert (xs == 0).any()
    vx, vw = (torch.from_numpy(v).cuda() for v in (values(xq, xs, n_in, bits), values(wq, ws, n_in, 4)))
    for dtype in ("f32", "bf16"):
        y = torch.empty((rows, n_out), dtype=torch_type(dtype), device="cuda")
        cfg = b.make_mx_linear_config(code(dtype), bits, rows, n_in, n_out)
        work = torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        b.dlc_mx_linear_forward(cfg, *(torch.from_numpy(v).cuda() for v in (xq, xs, wq, ws)), None, None, y, work)
        v, e = product(vx, vw)
        if bits == 8 and dtype == "f32":
            e = e + torch.where(vx.abs() < 2.0 ** -126, vx.abs(), 0.0) @ vw.abs().t()
        elif bits == 8:
            e = e + CUT * (vx.abs() @ vw.abs().t())
        assert_close(y, v, rounded(v, e, dtype), f"{rows} {bits} {dtype}")


def test_scales_from_end_to_end():
    """Hand-made scales, 2^-127 against 2^127: the results are whole numbers of products of elements."""
    import torch
    from paper_2407_04272_amd import binding as b
    rows, n_in, n_out = 70, 256, 48
    rng = np.random.default_rng(32)
    for bits, lo in ((4, 0), (8, 15)):      # (E4M3: from 2^-112 on every element is a normal number)
        xq, xs = quantise(rng.choice([-2.0, -1.0, 0.0, 1.0, 2.0], (rows, n_in)), bits)
        wq, ws = quantise(rng.choice([-1.0, 0.0, 1.0, 3.0], (n_out, n_in)), 4)
        one = values(xq, np.full_like(xs, 127), n_in, bits) @ values(wq, np.full_like(ws, 127), n_in, 4).T
        for a, c in ((lo, 254 - lo), (254 - 8, 8), (100, 150)):
            y = torch.empty((rows, n_out), device="cuda")
            cfg = b.make_mx_linear_config(b.F32, bits, rows, n_in, n_out)
            work = torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
            if bits == 8 and a > 246:
                continue
            b.dlc_mx_linear_forward(cfg, torch.from_numpy(xq).cuda(), torch.full(xs.shape, a, dtype=torch.uint8, device="cuda"), torch.from_numpy(wq).cuda(),
                                    torch.full(ws.shape, c, dtype=torch.uint8, device="cuda"), None, None, y, work)
            assert np.array_equal(y.cpu().numpy().astype(np.float64), one * 2.0 ** (a + c - 254)), (bits, a, c)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(9, 7), (20, 9), (18, 23), (5, 35), (3, 95), (17, 121), (33, 519), (2, 1021)])
def test_quantise_rows_that_end_inside_an_eight(rows, cols, dtype, bits):
    """... a value that two lanes have must not count for the block of the second, a NaN neither"""
    x, t = _matrix(rows, cols, dtype, 51, "wide")
    for at in range(max(cols - 9, 0), cols):
        t = t.clone()
        t[at % rows, at] = float("nan") if at % 2 else 1000.0
        _same(*_quantised(t, bits, dtype), *quantise(t.double().cpu().numpy(), bits), f"{rows}x{cols} {bits} {dtype} {at}")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,ld", [(63, 8, 0), (64, 127, 0), (65, 128, 0), (130, 100, 0), (200, 5, 0), (300, 64, 71), (129, 33, 40), (4100, 128, 0)])
def test_narrow_rows(rows, cols, ld, dtype, bits):
    """At most 128 columns: several rows a wavefront, and all 16 bytes of a row's scales from a quarter of it."""
    x, t = _matrix(rows, cols, dtype, 61, "wide")
    if ld:
        t = Guarded(rows, cols, dtype, ld, 1).set(t).view
    _same(*_quantised(t, bits, dtype, ld), *quantise(x, bits), f"{rows}x{cols} {bits} {dtype}")
    test_back(rows, cols, ld, dtype, bits)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(33, 512, 16), (64, 2048, 300), (65, 129, 17), (96, 4100, 33), (127, 33, 1), (250, 700, 64), (1000, 640, 40), (5000, 300, 7)])
def test_bands_of_rows(rows, n_in, n_out, dtype, bits):
    """More than one band of 32 rows in a pass over the weights each, the last one not full."""
    _linear(rows, n_in, n_out, bits, dtype)
    _linear(rows, n_in, n_out, bits, dtype, "gelu", bias=True, residual=True, ld=n_out + 3)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,n_in,n_out", [(300, 2048, 2048), (300, 2000, 2040), (400, 1290, 1500), (200, 4000, 1100), (700, 768, 1030), (260, 513, 3000), (1100, 256, 1100)])
def test_tiles_of_every_length(rows, n_in, n_out, bits):
    """Numbers of tiles of k values from one to eight in middle tiles: whole turns through the loop, and every rest."""
    for dtype in ("bf16", "f32"):
        _linear(rows, n_in, n_out, bits, dtype, bias=True)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 40, 17), (1, 1100, 64), (2, 513, 5), (9, 130, 16), (16, 1000, 40)])
def test_few_rows_lose_nothing(rows, n_in, n_out, dtype):
    """Every block of 32 has +448 and -448 in different groups of eight, whose products (w 0.5 there) add up to nothing, and elements
    of at most 2^-4.  Products are whole numbers of 2^-10 and stay below 2^14 together (35 blocks of two 224 and 1100 of 0.375): fp32
    sums are exact in any order, and the result is rounded once."""
    import torch
    from paper_2407_04272_amd import binding as b
    rng = np.random.default_rng(rows + n_in)
    x = rng.choice(np.arange(25), (rows, n_in))                     # codes of 0 .. 2^-4
    x = TABLE[8][x] * rng.choice([-1.0, 1.0], (rows, n_in))
    w = rng.choice(TABLE[4], (n_out, n_in)) * rng.choice([-1.0, 1.0], (n_out, n_in))
    w[:, 31::32] = 6.0                                              # (its scale is 1 too)
    at = np.arange(3, n_in - 17, 32)
    x[:, at] = 448.0 * rng.choice([-1.0, 1.0], (rows, len(at)))
    x[:, at + 17] = -x[:, at]
    w[:, at] = w[:, at + 17] = 0.5
    (xq, xs), (wq, ws) = quantise(x, 8), quantise(w, 4)
    assert np.array_equal(values(xq, xs, n_in, 8), x) and np.array_equal(values(wq, ws, n_in, 4), w) and (np.abs(x) @ np.abs(w).T).max() < 2 ** 14
    cfg = b.make_mx_linear_config(code(dtype), b.MX_E4M3, rows, n_in, n_out)
    y = torch.empty((rows, n_out), dtype=torch_type(dtype), device="cuda")
    b.dlc_mx_linear_forward(cfg, *(torch.from_numpy(v).cuda() for v in (xq, xs, wq, ws)), None, None, y)
    assert torch.equal(y.cpu(), torch.from_numpy(x @ w.T).to(torch_type(dtype)))
