"""The norm with the residual's addition and its backward pass against 64 bits."""
import numpy as np
import pytest

from dense_util import F32, Guarded, assert_close, code, rounded, torch_type
from mx_util import GuardedBytes, quantise, values

pytestmark = pytest.mark.gpu
TYPES = ["f32", "f16", "bf16"]
EPS = 1e-5
SIZES = [(1, 1), (1, 1664), (2, 8), (3, 7), (37, 16), (33, 129), (5, 512), (9, 513), (64, 1000), (7, 2047), (6, 4096), (5, 5001),
         (4, 8192), (3, 8200), (2, 16385), (3, 32768), (2, 32777), (2, 70001)]


def _depth(cols):
    """roundings on the way of one square into a row's sum: a lane's own (8 a chunk, four chunks; long rows one chunk of 8192
    columns after the other), 6 across the lanes, 16 wavefronts"""
    return max(32, -(-cols // 8192) * 8) + 6 + 16 + 2


def _normal(rows, cols, dtype, seed, scale=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn((rows, cols) if cols else (rows,), generator=g, device="cuda") * scale).to(torch_type(dtype))


def _forward(s, w):
    """y and a bound on its error before the rounding, and r's relative error"""
    n = s.shape[1]
    r = ((s * s).mean(dim=1, keepdim=True) + EPS) ** -0.5
    er = (_depth(n) + 4) * F32 / 2 + 2 * F32
    y = s * r * (1 if w is None else w.double())
    return y, y.abs() * (er + 4 * F32), r, er


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype):
    import torch
    from paper_2407_04272_amd import binding as b
    x, res, w = _normal(rows, cols, dtype, 1), _normal(rows, cols, dtype, 2, 0.5), _normal(cols, 0, dtype, 3)
    for residual, weight in ((None, w), (res, w), (res, None)):
        cfg = b.make_norm_config(code(dtype), rows, cols, EPS)
        s, y = Guarded(rows, cols, dtype), Guarded(rows, cols, dtype)
        b.dlc_norm_forward(cfg, x, residual, weight, s.view, y.view)
        assert s.intact() and y.intact()
        v = x.double() if residual is None else x.double() + res.double()
        assert_close(s.view, v, rounded(v, v.abs() * F32, dtype), "sum")
        want, err, _, _ = _forward(v, weight)
        assert_close(y.view, want, rounded(want, err, dtype), "y")
        only = torch.empty_like(x)
        b.dlc_norm_forward(cfg, x, residual, weight, None, only)
        assert torch.equal(only, y.view)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_eight_bits(rows, cols, dtype):
    """What is quantised is y in fp32, which an f32 call stores: then bit for bit."""
    import torch
    from paper_2407_04272_amd import binding as b
    x, res, w = _normal(rows, cols, dtype, 4), _normal(rows, cols, dtype, 5), _normal(cols, 0, dtype, 6)
    cfg = b.make_norm_config(code(dtype), rows, cols, EPS)
    mx = b.make_mx_config(code(dtype), b.MX_E4M3, rows, cols)
    q, sc = GuardedBytes(b.dlc_mx_data_shape(mx)), GuardedBytes(b.dlc_mx_scale_shape(mx))
    y, s = torch.empty_like(x), torch.empty_like(x)
    b.dlc_norm_forward(cfg, x, res, w, s, y, q.view, sc.view)
    assert q.intact() and sc.intact()
    if dtype == "f32":
        want_q, want_s = quantise(y.double().cpu().numpy(), 8)
        assert np.array_equal(sc.view.cpu().numpy(), want_s) and np.array_equal(q.view.cpu().numpy(), want_q)
    want, err, _, _ = _forward(x.double() + res.double(), w)
    got = torch.from_numpy(values(q.view.cpu().numpy(), sc.view.cpu().numpy(), cols, 8)).cuda()
    # half a step of a normal element, or of a subnormal one: 2^-10 of a scale that is at most 1/224 of the block's largest
    wide = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device="cuda")
    wide[:, :cols] = want.abs() + err
    top = wide.view(rows, -1, 32).amax(dim=2).repeat_interleave(32, dim=1)[:, :cols]
    assert_close(got, want, 2.0 ** -4 * (want.abs() + err) + err + top / 224 * 2.0 ** -10, "8 bits")
    q2, s2 = torch.empty_like(q.view), torch.empty_like(sc.view)
    b.dlc_norm_forward(cfg, x, res, w, None, None, q2, s2)
    assert torch.equal(q2, q.view) and torch.equal(s2, sc.view)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 700, 9000])
def test_rows_apart_and_in_place(cols, dtype):
    import torch
    from paper_2407_04272_amd import binding as b
    rows, ld = 6, cols + 13
    x, res, w = _normal(rows, cols, dtype, 7), _normal(rows, cols, dtype, 8), _normal(cols, 0, dtype, 9)
    plain = b.make_norm_config(code(dtype), rows, cols, EPS)
    s0, y0 = torch.empty_like(x), torch.empty_like(x)
    b.dlc_norm_forward(plain, x, res, w, s0, y0)
    for shift in (0, 1):
        vx, vr = Guarded(rows, cols, dtype, ld, shift).set(x), Guarded(rows, cols, dtype, cols + 5, shift).set(res)
        vs, vy = Guarded(rows, cols, dtype, cols + 8), Guarded(rows, cols, dtype, cols + 3, 3)
        cfg = b.make_norm_config(code(dtype), rows, cols, EPS, ld_x=ld, ld_res=cols + 5, ld_sum=cols + 8, ld_y=cols + 3)
        b.dlc_norm_forward(cfg, vx.view, vr.view, w, vs.view, vy.view)
        assert torch.equal(vs.view, s0) and torch.equal(vy.view, y0) and vs.intact() and vy.intact()
        # the sum in place of the residual, of x; y in place of x
        same = b.make_norm_config(code(dtype), rows, cols, EPS, ld_x=ld, ld_res=cols + 5, ld_sum=cols + 5, ld_y=cols + 3)
        b.dlc_norm_forward(same, vx.view, vr.view, w, vr.view, vy.view)
        assert torch.equal(vr.view, s0) and torch.equal(vy.view, y0)
    a, y = x.clone(), torch.empty_like(x)
    b.dlc_norm_forward(plain, a, res, w, a, y)
    assert torch.equal(a, s0) and torch.equal(y, y0)
    a = x.clone()
    b.dlc_norm_forward(plain, a, res, w, s0, a)
    assert torch.equal(a, y0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES + [(3000, 40), (2999, 259), (1100, 1024)])
def test_backward(rows, cols, dtype):
    import torch
    from paper_2407_04272_amd import binding as b
    s, w = _normal(rows, cols, dtype, 11), _normal(cols, 0, dtype, 12)
    dy, ds = _normal(rows, cols, dtype, 13), _normal(rows, cols, dtype, 14)
    cfg = b.make_norm_config(code(dtype), rows, cols, EPS)
    work = torch.empty(b.dlc_norm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    sd, dyd, n = s.double(), dy.double(), cols
    depth = _depth(cols)
    for weight, along in ((w, ds), (w, None), (None, ds)):
        dx, dw = Guarded(rows, cols, dtype), Guarded(1, cols, dtype)
        b.dlc_norm_backward(cfg, s, weight, dy, along, dx.view, dw.view[0], work)
        assert dx.intact() and dw.intact()
        _, _, r, er = _forward(sd, w)
        g = dyd if weight is None else dyd * w.double()
        c = r * r * (g * sd).mean(dim=1, keepdim=True)
        ec = r * r * (g * sd).abs().sum(dim=1, keepdim=True) / n * (depth + 4) * F32 + c.abs() * (2 * er + 6 * F32)
        inner = g - sd * c
        want = r * inner + (0 if along is None else ds.double())
        err = r * (g.abs() * 2 * F32 + sd.abs() * ec + (sd * c).abs() * 2 * F32) + (r * inner).abs() * (er + 3 * F32) + want.abs() * F32
        assert_close(dx.view, want, rounded(want, err, dtype), "dx")
        t = dyd * sd * r
        wd = t.sum(dim=0)
        assert_close(dw.view[0], wd, rounded(wd, t.abs().sum(dim=0) * ((rows + 32) * F32 + er), dtype), "dweight")
        # each alone, and in place of dy
        d2, w2 = dy.clone(), torch.empty_like(w)
        b.dlc_norm_backward(cfg, s, weight, d2, along, d2, None, None)
        b.dlc_norm_backward(cfg, s, weight, dy, along, None, w2, work)
        assert torch.equal(d2, dx.view) and torch.equal(w2, dw.view[0])


def test_backward_rows_apart():
    import torch
    from paper_2407_04272_amd import binding as b
    rows, cols = 50, 300
    for dtype in TYPES:
        v = [_normal(rows, cols, dtype, 20 + i) for i in range(3)]
        w = _normal(cols, 0, dtype, 30)
        cfg = b.make_norm_config(code(dtype), rows, cols, EPS)
        work = torch.empty(b.dlc_norm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        dx, dw = torch.empty_like(v[0]), torch.empty_like(w)
        b.dlc_norm_backward(cfg, v[0], w, v[1], v[2], dx, dw, work)
        far = [Guarded(rows, cols, dtype, cols + 7 * (i + 1), i).set(t) for i, t in enumerate(v)]
        out, dw2 = Guarded(rows, cols, dtype, cols + 9, 1), torch.empty_like(w)
        cfg = b.make_norm_config(code(dtype), rows, cols, EPS, ld_sum=cols + 7, ld_dy=cols + 14, ld_ds=cols + 21, ld_dx=cols + 9)
        b.dlc_norm_backward(cfg, far[0].view, w, far[1].view, far[2].view, out.view, dw2, work)
        assert torch.equal(out.view, dx) and torch.equal(dw2, dw) and out.intact()


def test_backward_against_differences():
    """The definition's differences in 64 bits along random directions, steps of 1e-5: off by about 1e-9 of the terms; the
    call's fp32 gradients are asked for 1e-4 of the directions' norms."""
    import torch
    from paper_2407_04272_amd import binding as b
    rows, cols = 13, 200
    s, w, dy = _normal(rows, cols, "f32", 41), _normal(cols, 0, "f32", 42), _normal(rows, cols, "f32", 43)
    cfg = b.make_norm_config(b.F32, rows, cols, EPS)
    dx, dw = torch.empty_like(s), torch.empty_like(w)
    b.dlc_norm_backward(cfg, s, w, dy, None, dx, dw, torch.empty(b.dlc_norm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"))

    def value(a, c):
        return float((a / ((a * a).mean(dim=1, keepdim=True) + EPS).sqrt() * c * dy.double()).sum())

    h = 1e-5
    for i in range(5):
        u, v = _normal(rows, cols, "f32", 50 + i).double(), _normal(cols, 0, "f32", 60 + i).double()
        by_s = (value(s.double() + h * u, w.double()) - value(s.double() - h * u, w.double())) / (2 * h)
        by_w = (value(s.double(), w.double() + h * v) - value(s.double(), w.double() - h * v)) / (2 * h)
        assert abs(float((dx.double() * u).sum()) - by_s) <= 1e-4 * float(u.norm() * dx.double().norm())
        assert abs(float((dw.double() * v).sum()) - by_w) <= 1e-4 * float(v.norm() * dw.double().norm())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [24, 600, 3000, 40000])
def test_zeros_nan_and_far_values(cols, dtype):
    """A row of zeros is zeros (r = eps^-1/2), a NaN or an infinity spoils its own row only."""
    import torch
    from paper_2407_04272_amd import binding as b
    rows = 6
    x, w = _normal(rows, cols, dtype, 70), _normal(cols, 0, dtype, 71)
    x[1] = 0
    x[2, cols // 2] = float("nan")
    x[3, cols - 1] = float("inf")
    cfg, mx = b.make_norm_config(code(dtype), rows, cols, EPS), b.make_mx_config(code(dtype), b.MX_E4M3, rows, cols)
    y = torch.empty_like(x)
    q, sc = (torch.empty(shape, dtype=torch.uint8, device="cuda") for shape in (b.dlc_mx_data_shape(mx), b.dlc_mx_scale_shape(mx)))
    b.dlc_norm_forward(cfg, x, None, w, None, y, q, sc)
    assert bool((y[1] == 0).all()) and bool(torch.isnan(y[2]).all())
    assert bool(torch.isnan(y[3, -1])) and bool((y[3, :-1] == 0).all())
    v = values(q.cpu().numpy(), sc.cpu().numpy(), cols, 8)
    assert (v[1] == 0).all() and np.isnan(v[2]).all() and np.isnan(v[3, -1]) and (v[3, :(cols - 1) // 32 * 32] == 0).all()
    ok = [0, 4, 5]
    want, err, _, _ = _forward(x[ok].double(), w)
    assert_close(y[ok], want, rounded(want, err, dtype), "other rows")


def test_no_rows():
    import torch
    from paper_2407_04272_amd import binding as b
    for dtype in TYPES:
        e, w = torch.empty((0, 50), dtype=torch_type(dtype), device="cuda"), _normal(50, 0, dtype, 1)
        cfg = b.make_norm_config(code(dtype), 0, 50)
        b.dlc_norm_forward(cfg, e, e, w, e, e)
        dw = torch.full_like(w, 7.0)
        b.dlc_norm_backward(cfg, e, w, e, None, e, dw)
        assert bool((dw == 0).all())


# the last eight of a row starts in the lane before: behind every border between the teams' sizes, short rows of less than eight
ENDS = [(40, 5), (50, 9), (70, 15), (3, 127), (20, 131), (9, 519), (7, 1023), (5, 1025), (40, 2049), (4, 4097), (3, 8191), (3, 8193), (2, 12291), (2, 16383)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", ENDS)
def test_rows_that_end_inside_an_eight(rows, cols, dtype):
    test_forward(rows, cols, dtype)
    test_eight_bits(rows, cols, dtype)
    test_backward(rows, cols, dtype)
    test_rows_apart_and_in_place(cols, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [24, 600, 2000, 4099, 12288, 12289])
def test_many_rows_backward(cols, dtype):
    """More rows than work-groups: a team's sums for the weight's gradient go on from row to row."""
    test_backward(1100 if cols < 4000 else 600, cols, dtype)


@pytest.mark.parametrize("cols", [33, 1023, 12289])
def test_a_nan_stays_in_its_row(cols):
    """... of the columns that two lanes have, too, and of rows in 8 bits"""
    import torch
    from paper_2407_04272_amd import binding as b
    for at in (0, cols - 9, cols - 8, cols - 1):
        x, w = _normal(5, cols, "f32", 41), _normal(cols, 0, "f32", 42)
        x[2, at] = float("nan")
        cfg, mx = b.make_norm_config(b.F32, 5, cols, EPS), b.make_mx_config(b.F32, b.MX_E4M3, 5, cols)
        y, q, sc = torch.empty_like(x), GuardedBytes(b.dlc_mx_data_shape(mx)), GuardedBytes(b.dlc_mx_scale_shape(mx))
        b.dlc_norm_forward(cfg, x, None, w, None, y, q.view, sc.view)
        rows = [0, 1, 3, 4]
        assert bool(torch.isnan(y[2]).all()) and not bool(torch.isnan(y[rows]).any())
        want_q, want_s = quantise(y.double().cpu().numpy(), 8)
        assert np.array_equal(sc.view.cpu().numpy(), want_s) and np.array_equal(q.view.cpu().numpy(), want_q) and q.intact() and sc.intact()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(256, 16392), (257, 20000), (600, 16385), (700, 24583)])
def test_many_long_rows_backward(rows, cols, dtype):
    """Rows past 16384 columns, as many as there are work-groups and more: the weight's sums go on in memory from row to row."""
    test_backward(rows, cols, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(5, 5), (3000, 40), (1100, 131), (2999, 259), (1100, 1023), (1100, 2047), (700, 4099), (600, 6100), (600, 8191), (300, 12283),
                                       (300, 16383), (300, 16391)])
def test_backward_in_place(rows, cols, dtype):
    """dx in place of the gradient along s, of y's, and of both where they are one tensor; rows that end inside an eight, whose last
    columns two lanes load and store, and more rows than teams."""
    import torch
    from paper_2407_04272_amd import binding as b
    s, w, dy, ds = _normal(rows, cols, dtype, 81), _normal(cols, 0, dtype, 82), _normal(rows, cols, dtype, 83), _normal(rows, cols, dtype, 84)
    cfg = b.make_norm_config(code(dtype), rows, cols, EPS)
    work = torch.empty(b.dlc_norm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")

    def call(dy, ds, dx, cfg=cfg):
        dw = torch.empty_like(w)
        b.dlc_norm_backward(cfg, s, w, dy, ds, dx, dw, work)
        return dw

    dx, same = torch.empty_like(s), torch.empty_like(s)
    dw = call(dy, ds, dx)
    dw_same = call(dy, dy, same)
    for _ in range(3):
        a = ds.clone()
        assert torch.equal(call(dy, a, a), dw) and torch.equal(a, dx)
        a = dy.clone()
        assert torch.equal(call(a, ds, a), dw) and torch.equal(a, dx)
        a = dy.clone()
        assert torch.equal(call(a, a, a), dw_same) and torch.equal(a, same)
    far = Guarded(rows, cols, dtype, cols + 7, 1).set(ds)
    apart = b.make_norm_config(code(dtype), rows, cols, EPS, ld_ds=cols + 7, ld_dx=cols + 7)
    assert torch.equal(call(dy, far.view, far.view, apart), dw) and torch.equal(far.view, dx) and far.intact()
