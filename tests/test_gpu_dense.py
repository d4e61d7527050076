"""Linear layers, gated blocks and dropout against plain forms in 64 bits, through the C ABI.

Bounds: a sum of K terms in fp32 is off by at most about K 2^-24 of the sum of their magnitudes, in any order; an operand
rounded to the type adds its half unit in the last place of the same sum; activations have slopes below 1.13 and add a few
fp32 roundings; the result is rounded once."""
import numpy as np
import pytest

from dense_util import (ACTS, F32, FN, ROUND, Guarded, act, assert_close, code, drop_factor, philox_words, product, rounded,
                        torch_type)

TYPES = ["f32", "f16", "bf16"]
SEED, OFFSET = 0x9E3779B97F4A7C15, 0x123456789AB


def _inputs(rng_seed, dtype, **shapes):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(rng_seed)
    out = {}
    for name, (shape, scale) in shapes.items():
        out[name] = (torch.randn(shape, generator=g, device="cuda") * scale).to(torch_type(dtype))
    return out


def _lay(t, dtype, how):
    """the tensor in a buffer of its own: dense, on a 16-byte pitch with a gap, or odd"""
    rows, cols = t.shape if t.dim() == 2 else (1, t.shape[0])
    if how == "dense":
        g = Guarded(rows, cols, dtype)
    elif how == "pitch":
        g = Guarded(rows, cols, dtype, ld=(cols + 7) // 8 * 8 + 16)
    else:
        g = Guarded(rows, cols, dtype, ld=cols + 3, shift=1)
    g.set(t.view(rows, cols))
    return g


def _vec(g):
    return g.view[0]


def _factor(M, N, p, offset=OFFSET):
    import torch
    if p == 0:
        return torch.ones((M, N), dtype=torch.float64, device="cuda")
    return torch.from_numpy(drop_factor(M, N, p, SEED, offset)).cuda()


def _forward(op, dtype, M, K, N, name, bias, residual, save, p, how, seed=1):
    import torch
    from paper_2407_04272_amd import binding as b
    wide = 2 * N if op == "gated" else N
    t = _inputs(seed, dtype, x=((M, K), 1.0), w=((wide, K), K ** -0.5), bias=((wide,), 0.5), res=((M, N), 1.0))
    gx, gw, gb, gr = (_lay(t[k], dtype, how) for k in ("x", "w", "bias", "res"))
    gy, gp = _lay(t["res"], dtype, how), _lay(torch.zeros((M, wide), device="cuda"), dtype, how)
    cfg = b.make_dense_config(code(dtype), M, K, N, act=ACTS.index(name), dropout_p=p, seed=SEED, offset=OFFSET, ld_x=gx.ld,
                              ld_w=gw.ld, ld_y=gy.ld, ld_pre=gp.ld, ld_res=gr.ld)
    nb = (b.dlc_gated_workspace_bytes if op == "gated" else b.dlc_linear_workspace_bytes)(cfg)
    work = torch.full((nb + 64,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN in every type; guard bytes at the end
    args = (cfg, gx.view, gw.view, _vec(gb) if bias else None)
    if op == "gated":
        b.dlc_gated_forward(*args, gy.view, gp.view if save else None, work[:nb])
    else:
        b.dlc_linear_forward(*args, gr.view if residual else None, gy.view, gp.view if save else None, work[:nb])
    torch.cuda.synchronize()
    z, ez = product(t["x"].double(), t["w"].double())
    if bias:
        z, ez = z + t["bias"].double(), ez + F32 * (z.abs() + t["bias"].double().abs())
    what = f"{op} {dtype} {M} x {K} -> {N} {name} {how}"
    if save:
        assert_close(gp.view, z, rounded(z, ez, dtype), what + " pre")
    f = _factor(M, N, p)
    if op == "gated":
        g, u, eg, eu = z[:, :N], z[:, N:], ez[:, :N], ez[:, N:]
        v, _ = act(name, g)
        ev = 1.13 * eg + FN * (v.abs() + F32)
        y, ey = v * u * f, f * (ev * u.abs() + v.abs() * eu + ev * eu + 2 * F32 * (v * u).abs())
    else:
        v, _ = act(name, z)
        y, ey = v * f, f * (1.13 * ez + FN * (v.abs() + F32))
        if residual:
            r = t["res"].double()
            y, ey = y + r, ey + F32 * (y.abs() + r.abs())
    ey = ey + 2 * F32 * y.abs()
    assert_close(gy.view, y, rounded(y, ey, dtype), what + " y")
    assert gy.intact() and gp.intact(), what
    assert bool((work[nb:] == 0xFF).all()), what


def _backward(op, dtype, M, K, N, name, p, how, seed=2):
    import torch
    from paper_2407_04272_amd import binding as b
    wide = 2 * N if op == "gated" else N
    t = _inputs(seed, dtype, x=((M, K), 1.0), w=((wide, K), K ** -0.5), pre=((M, wide), 1.0), dy=((M, N), 1.0))
    gx, gw, gp, gd = (_lay(t[k], dtype, how) for k in ("x", "w", "pre", "dy"))
    zeros = torch.zeros
    gdx, gdw, gdb = (_lay(zeros(s, device="cuda"), dtype, how) for s in ((M, K), (wide, K), (1, wide)))
    cfg = b.make_dense_config(code(dtype), M, K, N, act=ACTS.index(name), dropout_p=p, seed=SEED, offset=OFFSET, ld_x=gx.ld,
                              ld_w=gw.ld, ld_pre=gp.ld, ld_dy=gd.ld, ld_dx=gdx.ld, ld_dw=gdw.ld)
    nb = (b.dlc_gated_workspace_bytes if op == "gated" else b.dlc_linear_workspace_bytes)(cfg, True)
    work = torch.full((nb + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    call = b.dlc_gated_backward if op == "gated" else b.dlc_linear_backward
    needs_pre = op == "gated" or name != "none"
    call(cfg, gx.view, gw.view, gp.view if needs_pre else None, gd.view, gdx.view, gdw.view, _vec(gdb), work[:nb])
    torch.cuda.synchronize()
    d = t["dy"].double() * _factor(M, N, p)
    pre = t["pre"].double()
    if op == "gated":
        v, s = act(name, pre[:, :N])
        dz = torch.cat((d * pre[:, N:] * s, d * v), 1)
        edz = torch.cat((d.abs() * pre[:, N:].abs(), d.abs()), 1) * FN + 4 * F32 * dz.abs()
    else:
        _, s = act(name, pre)
        dz = d * s
        edz = (d.abs() * FN if name not in ("none", "relu") else 0.0) + 2 * F32 * dz.abs()
    what = f"{op} backward {dtype} {M} x {K} -> {N} {name} {how}"
    x, w = t["x"].double(), t["w"].double()
    half = edz + ROUND[dtype] * dz.abs() + 2.0 ** -25   # dz rounded to the type (f16: subnormals too)
    v, e = product(dz, w.t())
    e = e + half @ w.abs()
    assert_close(gdx.view, v, rounded(v, e, dtype), what + " dx")
    v, e = product(dz.t(), x.t())
    e = e + half.t() @ x.abs()
    assert_close(gdw.view, v, rounded(v, e, dtype), what + " dw")
    v, e = dz.sum(0), edz.sum(0) + (M + 2) * F32 * dz.abs().sum(0)
    assert_close(_vec(gdb), v, rounded(v, e, dtype), what + " dbias")
    assert gdx.intact() and gdw.intact() and gdb.intact(), what
    assert bool((work[nb:] == 0xFF).all()), what


# rows, in, out: single tokens, the largest batch of the few-rows kernel and one past it, ragged and whole tiles, one
# column, one k, long sums that are cut, several tiles of every size
FORWARD = [(1, 1664, 1024), (3, 13, 1), (16, 520, 40), (17, 64, 128), (5, 1, 7), (32, 72, 24), (31, 1000, 130), (33, 64, 64), (40, 259, 129), (130, 72, 200),
           (777, 515, 103), (64, 8192, 64), (2048, 256, 1024), (300, 4096, 256), (1030, 200, 2000)]
BACKWARD = [(1, 64, 32), (2, 13, 1), (17, 100, 40), (1, 1, 1), (259, 37, 129), (1000, 264, 72), (4096, 64, 128),
            (2999, 259, 129), (2048, 1024, 512), (1025, 520, 1000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", FORWARD)
def test_linear_forward(dtype, shape):
    i = FORWARD.index(shape)
    for how in ("dense", "pitch", "odd"):
        _forward("linear", dtype, *shape, ACTS[i % 5], bias=True, residual=i % 2 == 0, save=True, p=0.3 if i % 3 == 0 else 0.0, how=how)
    _forward("linear", dtype, *shape, "relu", bias=False, residual=i % 2 == 1, save=False, p=0.5 if i % 3 else 0.0, how="dense")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", FORWARD)
def test_gated_forward(dtype, shape):
    i = FORWARD.index(shape)
    for how in ("dense", "pitch", "odd"):
        _forward("gated", dtype, *shape, ACTS[(i + 3) % 5], bias=i % 2 == 0, residual=False, save=i % 3 != 0,
                 p=0.3 if i % 4 == 0 else 0.0, how=how)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", BACKWARD)
def test_linear_backward(dtype, shape):
    i = BACKWARD.index(shape)
    for how in ("dense", "pitch", "odd"):
        _backward("linear", dtype, *shape, ACTS[i % 5], p=0.3 if i % 2 else 0.0, how=how)
    _backward("linear", dtype, *shape, "none", p=0.0, how="dense")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", BACKWARD)
def test_gated_backward(dtype, shape):
    i = BACKWARD.index(shape)
    for how in ("dense", "pitch", "odd"):
        _backward("gated", dtype, *shape, ACTS[(i + 2) % 5], p=0.3 if i % 2 else 0.0, how=how)


# the largest tiles in half precision, whole and ragged
FORWARD_LARGE = [("gated", (4096, 1024, 2048), "dense"), ("gated", (4090, 1030, 2050), "pitch"), ("linear", (8190, 1000, 4001), "odd")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op,shape,how", FORWARD_LARGE)
def test_large_forward(dtype, op, shape, how):
    _forward(op, dtype, *shape, "silu", bias=True, residual=op == "linear", save=True, p=0.0, how=how)


# both products in one launch on the largest tiles: nothing cut and the bias gradient in the same launch, the gradient of w
# cut; one launch after the other, the gradient of x cut
BACKWARD_LARGE = [("linear", (8200, 4100, 2056), "odd"), ("linear", (8192, 2048, 2048), "dense"), ("linear", (300, 4000, 2000), "pitch"),
                  ("gated", (1000, 2000, 4000), "dense"), ("gated", (2100, 700, 600), "odd")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op,shape,how", BACKWARD_LARGE)
def test_large_backward(dtype, op, shape, how):
    _backward(op, dtype, *shape, "relu" if op == "linear" else "silu", p=0.0, how=how)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", ["linear", "gated"])
def test_every_activation(dtype, op):
    for name in ACTS:
        _forward(op, dtype, 70, 96, 72, name, bias=True, residual=op == "linear", save=True, p=0.25, how="dense")
        _backward(op, dtype, 70, 96, 72, name, p=0.25, how="dense")


# ---- dropout ------------------------------------------------------------------------------------
def test_philox_known_answers():
    """The generator's published known answers (counter, key -> output)."""
    m = 0xFFFFFFFF
    for c, k, want in [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                       ((m, m, m, m), (m, m), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                       ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
                        (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(int(v[0]) for v in philox_words([np.array([v]) for v in c], k)) == want


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 8), (256, 16), (37, 259), (5, 20000), (1024, 1024)])
def test_dropout(dtype, shape):
    import torch
    from paper_2407_04272_amd import binding as b
    rows, cols = shape
    for how in ("dense", "pitch", "odd"):
        for p in (0.0, 1e-5, 0.1, 0.5, 1.0):
            for residual in (False, True):
                t = _inputs(7, dtype, x=(shape, 1.0), res=(shape, 1.0))
                gx, gr = _lay(t["x"], dtype, how), _lay(t["res"], dtype, how)
                gy = _lay(t["x"] * 0, dtype, how)
                cfg = b.make_dropout_config(code(dtype), rows, cols, p, seed=SEED, offset=OFFSET, ld_x=gx.ld, ld_res=gr.ld, ld_y=gy.ld)
                b.dlc_dropout(cfg, gx.view, gr.view if residual else None, gy.view)
                # one fp32 product, one fp32 sum, one rounding: every bit is fixed
                f = torch.from_numpy(drop_factor(rows, cols, p, SEED, OFFSET)).cuda().float()
                want = t["x"].float() * f
                want = torch.where(f == 0, torch.zeros_like(want), want)
                if residual:
                    want = want + t["res"].float()
                assert torch.equal(gy.view, want.to(torch_type(dtype))), (dtype, shape, how, p, residual)
                assert gy.intact()
    # in place, and the gradient is the same call
    y = t["x"].clone()
    cfg = b.make_dropout_config(code(dtype), rows, cols, 0.5, seed=SEED, offset=OFFSET)
    b.dlc_dropout(cfg, y, None, y)
    f = torch.from_numpy(drop_factor(rows, cols, 0.5, SEED, OFFSET)).cuda().float()
    assert torch.equal(y, (t["x"].float() * f).to(torch_type(dtype)))


@pytest.mark.gpu
def test_a_dropped_element_is_zero_whatever_it_holds():
    import torch
    from paper_2407_04272_amd import binding as b
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = torch.empty_like(x)
    b.dlc_dropout(b.make_dropout_config(b.F32, 64, 64, 0.5, seed=3), x, None, y)
    keep = torch.from_numpy(drop_factor(64, 64, 0.5, 3, 0)).cuda() > 0
    assert bool((y[~keep] == 0).all()) and bool(torch.isnan(y[1::2][keep[1::2]]).all()) and bool(torch.isinf(y[::2][keep[::2]]).all())
    share = float(keep.double().mean())
    assert abs(share - 0.5) < 5 * 0.5 / 64   # five standard deviations of 4096 fair bits


@pytest.mark.gpu
def test_what_is_not_finite_stays_where_it_belongs():
    """A row or column that is not finite spoils its own results only; a closed relu passes no gradient."""
    import torch
    from paper_2407_04272_amd import binding as b
    for M in (5, 200):
        t = _inputs(5, "bf16", x=((M, 96), 1.0), w=((72, 96), 0.1), dy=((M, 72), 1.0))
        x, w = t["x"].clone(), t["w"].clone()
        x[2, 3], w[70, 5] = float("nan"), float("inf")
        cfg = b.make_dense_config(b.BF16, M, 96, 72, act=b.ACT_RELU)
        work = torch.empty(max(1, b.dlc_linear_workspace_bytes(cfg), b.dlc_linear_workspace_bytes(cfg, True)), dtype=torch.uint8, device="cuda")
        y, pre = torch.empty((M, 72), dtype=torch.bfloat16, device="cuda"), torch.empty((M, 72), dtype=torch.bfloat16, device="cuda")
        b.dlc_linear_forward(cfg, x, w, None, None, y, pre, work)
        ok = torch.ones((M, 72), dtype=torch.bool, device="cuda")
        ok[2], ok[:, 70] = False, False
        assert bool(torch.isnan(y[2]).all()) and bool(torch.isfinite(y[ok]).all()) and not bool(torch.isfinite(pre[:, 70]).any())
        pre = -torch.ones_like(pre)
        pre[0, 0] = 1.0
        dy = torch.full_like(y, float("inf"))
        dy[0, 0] = 2.0
        dx, dw, db = torch.empty_like(t["x"]), torch.empty_like(t["w"]), torch.empty(72, dtype=torch.bfloat16, device="cuda")
        b.dlc_linear_backward(cfg, t["x"], t["w"], pre, dy, dx, dw, db, work)
        assert float(db[0]) == 2.0 and bool((db[1:] == 0).all()) and bool((dx[1:] == 0).all()) and bool((dw[1:] == 0).all())
        assert torch.equal(dx[0], 2 * t["w"][0]) and torch.equal(dw[0], 2 * t["x"][0])


# ---- sizes and calls ----------------------------------------------------------------------------
@pytest.mark.gpu
def test_no_rows():
    import torch
    from paper_2407_04272_amd import binding as b
    for op in ("linear", "gated"):
        wide = 24 if op == "gated" else 12
        e = torch.empty
        x, y, pre = e((0, 20), device="cuda"), e((0, 12), device="cuda"), e((0, wide), device="cuda")
        w, dw, db = torch.ones((wide, 20), device="cuda"), torch.ones((wide, 20), device="cuda"), torch.ones(wide, device="cuda")
        cfg = b.make_dense_config(b.F32, 0, 20, 12, act=b.ACT_SILU)
        if op == "gated":
            b.dlc_gated_forward(cfg, x, w, None, y, pre)
            b.dlc_gated_backward(cfg, x, w, pre, y, x, dw, db)
        else:
            b.dlc_linear_forward(cfg, x, w, None, None, y, pre)
            b.dlc_linear_backward(cfg, x, w, pre, y, x, dw, db)
        assert bool((dw == 0).all()) and bool((db == 0).all())
    b.dlc_dropout(b.make_dropout_config(b.F32, 0, 12, 0.5), y, None, y)


@pytest.mark.gpu
def test_outputs_that_are_not_wanted():
    """Each gradient alone equals the one of the whole call, bit for bit, and so does a second call."""
    import torch
    from paper_2407_04272_amd import binding as b
    for name, p in (("none", 0.0), ("silu", 0.2)):
        t = _inputs(9, "f16", x=((500, 264), 1.0), w=((136, 264), 0.1), pre=((500, 136), 1.0), dy=((500, 136), 1.0))
        cfg = b.make_dense_config(b.F16, 500, 264, 136, act=ACTS.index(name), dropout_p=p, seed=1)
        work = torch.empty(b.dlc_linear_workspace_bytes(cfg, True), dtype=torch.uint8, device="cuda")
        e = lambda *s: torch.empty(s, dtype=torch.float16, device="cuda")
        outs = [[e(500, 264), e(136, 264), e(136)] for _ in range(5)]
        for k, o in enumerate(outs):
            work.fill_(0xFF)
            a = [v if k < 2 or i == k - 2 else None for i, v in enumerate(o)]
            b.dlc_linear_backward(cfg, t["x"], t["w"], t["pre"], t["dy"], *a, work)
        for i in range(3):
            assert torch.equal(outs[0][i], outs[1][i]) and torch.equal(outs[0][i], outs[2 + i][i]), (name, i)


@pytest.mark.gpu
def test_residual_in_place():
    import torch
    from paper_2407_04272_amd import binding as b
    for M in (4, 300):
        t = _inputs(11, "bf16", x=((M, 512), 1.0), w=((100, 512), 0.1), res=((M, 100), 1.0))
        cfg = b.make_dense_config(b.BF16, M, 512, 100, act=b.ACT_RELU)
        work = torch.empty(max(1, b.dlc_linear_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
        y = torch.empty_like(t["res"])
        b.dlc_linear_forward(cfg, t["x"], t["w"], None, t["res"], y, None, work)
        b.dlc_linear_forward(cfg, t["x"], t["w"], None, t["res"], t["res"], None, work)
        assert torch.equal(y, t["res"])


@pytest.mark.gpu
def test_gradients_against_differences():
    """f32: the directional derivative of sum(y c) against a central difference of forward calls.  With step h the
    difference is off by h^2 times the third derivative along the direction, here below 2 sum|c| (d z)^3, and by the sums'
    roundings, K 2^-24 of their magnitudes over h."""
    import torch
    from paper_2407_04272_amd import binding as b
    M, K, N, h = 33, 48, 40, 2.0 ** -6
    for op in ("linear", "gated"):
        for name in ("sigmoid", "silu", "gelu"):
            wide = 2 * N if op == "gated" else N
            t = _inputs(13, "f32", x=((M, K), 1.0), w=((wide, K), K ** -0.5), bias=((wide,), 0.2), c=((M, N), 1.0),
                        ex=((M, K), 1.0), ew=((wide, K), K ** -0.5), eb=((wide,), 0.2))
            cfg = b.make_dense_config(b.F32, M, K, N, act=ACTS.index(name), dropout_p=0.25, seed=5, offset=6)
            y, pre = torch.empty((M, N), device="cuda"), torch.empty((M, wide), device="cuda")
            size = b.dlc_gated_workspace_bytes if op == "gated" else b.dlc_linear_workspace_bytes
            work = torch.empty(max(size(cfg), size(cfg, True)), dtype=torch.uint8, device="cuda")

            def value(x, w, bias):
                if op == "gated":
                    b.dlc_gated_forward(cfg, x, w, bias, y, pre, work)
                else:
                    b.dlc_linear_forward(cfg, x, w, bias, None, y, pre, work)
                return float((y.double() * t["c"].double()).sum())

            grads = [torch.empty_like(t[k]) for k in ("x", "w", "bias")]
            value(t["x"], t["w"], t["bias"])
            (b.dlc_gated_backward if op == "gated" else b.dlc_linear_backward)(cfg, t["x"], t["w"], pre, t["c"], *grads, work)
            for i, (k, ek) in enumerate((("x", "ex"), ("w", "ew"), ("bias", "eb"))):
                at = lambda s: [t[j] + s * h * t[ek] if j == k else t[j] for j in ("x", "w", "bias")]
                diff = (value(*at(1.0)) - value(*at(-1.0))) / (2 * h)
                along = float((grads[i].double() * t[ek].double()).sum())
                e = [t[j].double() if j != k else t[ek].double() for j in ("x", "w")]
                dz = e[0] @ e[1].t() if k != "bias" else t["eb"].double().expand(M, wide)
                zmag = t["x"].double().abs() @ t["w"].double().abs().t() + 1.0
                if op == "gated":
                    gu = t["x"].double() @ t["w"].double().t() + t["bias"].double()
                    third = (dz[:, :N].abs() ** 3 * (gu[:, N:].abs() + 1) + dz[:, :N].abs() ** 2 * dz[:, N:].abs() * 3) * 4 / 3
                    mag = zmag[:, :N] * zmag[:, N:]
                else:
                    third, mag = dz.abs() ** 3 * 4 / 3, zmag
                c = t["c"].double().abs()
                tol = h * h * float((c * third).sum()) + (K + 8) * F32 * float((c * mag).sum()) * (1 + 1 / h)
                assert abs(diff - along) <= tol, (op, name, k, diff, along, tol)


@pytest.mark.gpu
def test_under_graph_capture():
    """A training step's calls in a HIP graph, the dropout counter on the GPU: every replay against the eager result."""
    import torch
    from paper_2407_04272_amd import binding as b
    M, K, N = 200, 264, 136
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    t = _inputs(17, "bf16", x=((M, K), 1.0), w=((N, K), 0.06), w2=((2 * N, N), 0.08), bias=((N,), 0.1), dy=((M, N), 1.0))
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    c1 = b.make_dense_config(b.BF16, M, K, N, act=b.ACT_RELU, dropout_p=0.25, seed=1, offset=100, d_offset=count)
    c2 = b.make_dense_config(b.BF16, M, N, N, act=b.ACT_SILU, dropout_p=0.25, seed=2, offset=100, d_offset=count)
    c3 = b.make_dropout_config(b.BF16, M, N, 0.25, seed=3, offset=100, d_offset=count)
    work = torch.empty(max(b.dlc_linear_workspace_bytes(c1), b.dlc_linear_workspace_bytes(c1, True),
                           b.dlc_gated_workspace_bytes(c2), b.dlc_gated_workspace_bytes(c2, True)), dtype=torch.uint8, device="cuda")
    y, pre, y2, pre2, y3 = e(M, N), e(M, N), e(M, N), e(M, 2 * N), e(M, N)
    d3, dh, dw2, dx, dw, db = e(M, N), e(M, N), e(2 * N, N), e(M, K), e(N, K), e(N)

    def step():
        b.dlc_linear_forward(c1, t["x"], t["w"], t["bias"], None, y, pre, work)
        b.dlc_gated_forward(c2, y, t["w2"], None, y2, pre2, work)
        b.dlc_dropout(c3, y2, y, y3)
        b.dlc_dropout(c3, t["dy"], None, d3)
        b.dlc_gated_backward(c2, y, t["w2"], pre2, d3, dh, dw2, None, work)
        b.dlc_linear_backward(c1, t["x"], t["w"], pre, dh, dx, dw, db, work)

    outs = (y, pre, y2, pre2, y3, d3, dh, dw2, dx, dw, db)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    seen = []
    for k in range(4):
        count.fill_(k if k < 3 else 0)
        t["x"].copy_(_inputs(20 + k % 3, "bf16", x=((M, K), 1.0))["x"])
        step()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (o, wv) in enumerate(zip(outs, want)):
            assert torch.equal(o, wv), (k, i)
        seen.append(d3.clone())
    assert not torch.equal(seen[0], seen[1]) and torch.equal(seen[0], seen[3])
    f = torch.from_numpy(drop_factor(M, N, 0.25, 3, 102)).cuda().float()
    assert torch.equal(seen[2], (t["dy"].float() * f).bfloat16())


@pytest.mark.gpu
def test_on_another_stream():
    import torch
    from paper_2407_04272_amd import binding as b
    t = _inputs(19, "f16", x=((600, 256), 1.0), w=((256, 256), 0.06))
    cfg = b.make_dense_config(b.F16, 600, 256, 256)
    work = torch.empty(max(1, b.dlc_linear_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
    y, y2 = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    b.dlc_linear_forward(cfg, t["x"], t["w"], None, None, y, None, work)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.dlc_linear_forward(cfg, t["x"], t["w"], None, None, y2, None, work, stream=side)
    side.synchronize()
    assert torch.equal(y, y2)


@pytest.mark.gpu
def test_pointers_off_the_boundary():
    """Rows whose length and pitch are fine behind pointers that are not: the flag makes room for copies, without it the
    call says that there is too little; the results are those of the same rows elsewhere."""
    import torch
    from paper_2407_04272_amd import binding as b
    for M, back in ((300, False), (300, True), (5, False)):
        t = _inputs(29, "bf16", x=((M, 128), 1.0), w=((72, 128), 0.1), dy=((M, 72), 1.0))
        off = {k: Guarded(*t[k].shape, "bf16", shift=3).set(t[k]) for k in ("x", "w")}
        outs = []
        for x, w, flags in ((t["x"], t["w"], 0), (off["x"].view, off["w"].view, b.DENSE_OFF_BOUNDARY), (off["x"].view, t["w"], b.DENSE_OFF_BOUNDARY)):
            cfg = b.make_dense_config(b.BF16, M, 128, 72, flags=flags)
            work = torch.full((max(16, b.dlc_linear_workspace_bytes(cfg, back)),), 0xFF, dtype=torch.uint8, device="cuda")
            y, dx, dw = torch.zeros_like(t["dy"]), torch.zeros_like(t["x"]), torch.zeros_like(t["w"])
            if back:
                b.dlc_linear_backward(cfg, x, w, None, t["dy"], dx, dw, None, work)
            else:
                b.dlc_linear_forward(cfg, x, w, None, None, y, None, work)
            outs.append((y, dx, dw))
        for o in outs[1:]:
            assert all(torch.equal(a, c) for a, c in zip(outs[0], o))
        cfg = b.make_dense_config(b.BF16, M, 128, 72)
        work = torch.empty(b.dlc_linear_workspace_bytes(cfg, back), dtype=torch.uint8, device="cuda")
        if back or M > 16:
            with pytest.raises(b.DlcError) as err:
                if back:
                    b.dlc_linear_backward(cfg, off["x"].view, off["w"].view, None, t["dy"], dx, dw, None, work)
                else:
                    b.dlc_linear_forward(cfg, off["x"].view, off["w"].view, None, None, y, None, work)
            assert err.value.status == b.ECAPACITY


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Operands of more than 2^32 bytes: rows past that point, forward and backward."""
    import torch
    from paper_2407_04272_amd import binding as b
    M, K, N = 2_300_003, 1024, 8
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    for r in range(0, M, 1 << 18):
        x[r:r + (1 << 18)].normal_()
    t = _inputs(23, "bf16", w=((N, K), K ** -0.5))
    dy = torch.randn((M, N), device="cuda").bfloat16()
    cfg = b.make_dense_config(b.BF16, M, K, N)
    work = torch.empty(max(1, b.dlc_linear_workspace_bytes(cfg), b.dlc_linear_workspace_bytes(cfg, True)), dtype=torch.uint8, device="cuda")
    y, dx, dw = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(t["w"])
    b.dlc_linear_forward(cfg, x, t["w"], None, None, y, None, work)
    b.dlc_linear_backward(cfg, x, t["w"], None, dy, dx, dw, None, work)
    want, mag = torch.zeros((N, K), dtype=torch.float64, device="cuda"), torch.zeros((N, K), dtype=torch.float64, device="cuda")
    for r in range(0, M, 1 << 18):
        s = slice(r, min(M, r + (1 << 18)))
        v, e = product(x[s].double(), t["w"].double())
        assert_close(y[s], v, rounded(v, e, "bf16"), f"y from row {r}")
        v, e = product(dy[s].double(), t["w"].double().t())
        assert_close(dx[s], v, rounded(v, e, "bf16"), f"dx from row {r}")
        want += dy[s].double().t() @ x[s].double()
        mag += dy[s].double().abs().t() @ x[s].double().abs()
    # (in any order the sum's error is below its terms' count times 2^-24 of their magnitudes; cut into stretches and
    # added tile by tile it stays far below that, 64 times is asked for)
    assert_close(dw, want, rounded(want, mag * (M / 64 * F32), "bf16"), "dw")


@pytest.mark.gpu
def test_dropout_past_32_bits():
    import torch
    from paper_2407_04272_amd import binding as b
    ld, cols = 2 ** 31 + 24, 100
    buf = torch.empty(2 * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, cols), (ld, 1))
    x.normal_()
    y = torch.empty((3, cols), dtype=torch.bfloat16, device="cuda")
    b.dlc_dropout(b.make_dropout_config(b.BF16, 3, cols, 0.5, seed=9, ld_x=ld), x, None, y)
    f = torch.from_numpy(drop_factor(3, cols, 0.5, 9, 0)).cuda().float()
    assert torch.equal(y, (x.float() * f).bfloat16())


# ---- refusals -----------------------------------------------------------------------------------
def test_invalid_geometry_has_no_workspace():
    from paper_2407_04272_amd import binding as b
    mk = b.make_dense_config
    assert b.dlc_linear_workspace_bytes(mk(b.F32, 512, 64, 64), True) > 0
    for bad in (mk(3, 512, 64, 64), mk(-1, 512, 64, 64), mk(b.F32, -1, 64, 64), mk(b.F32, 512, 0, 64), mk(b.F32, 512, 64, 0),
                mk(b.F32, 512, 64, 64, act=5), mk(b.F32, 512, 64, 64, act=-1), mk(b.F32, 512, 64, 64, dropout_p=1.5),
                mk(b.F32, 512, 64, 64, dropout_p=-0.1), mk(b.F32, 512, 64, 64, dropout_p=float("nan")), mk(b.F32, 512, 64, 64, flags=2),
                mk(b.F32, 512, 64, 64, ld_x=63), mk(b.F32, 512, 64, 64, ld_dw=-1), mk(b.F32, (1 << 30) + 1, 64, 64),
                mk(b.F32, 512, (1 << 20) + 1, 64), mk(b.F32, 512, 64, (1 << 20) + 1), mk(b.F32, 512, 64, 64, ld_w=1 << 40),
                mk(b.F32, 1 << 30, 1 << 20, 64)):
        assert b.dlc_linear_workspace_bytes(bad, True) == 0 and b.dlc_gated_workspace_bytes(bad, True) == 0
        assert b.dlc_linear_workspace_bytes(bad) == 0 and b.dlc_gated_workspace_bytes(bad) == 0
    assert b.dlc_gated_workspace_bytes(mk(b.F32, 512, 64, 64, ld_pre=127), True) == 0
    assert b.dlc_gated_workspace_bytes(mk(b.F32, 512, 64, (1 << 19) + 1), True) == 0
    assert b.dlc_gated_workspace_bytes(mk(b.F32, 512, 64, 1 << 19), True) > 0
    assert b.dlc_linear_workspace_bytes(mk(b.F32, 512, 64, 64, ld_pre=127), True) > 0


@pytest.mark.gpu
def test_refusals():
    import ctypes as C
    import torch
    from paper_2407_04272_amd import binding as b
    M, K, N = 100, 64, 48
    e = lambda *s: torch.ones(s, dtype=torch.float16, device="cuda")
    x, w, bias, y, pre = e(M, K), e(N, K), e(N), e(M, N), e(M, N)
    cfg = b.make_dense_config(b.F16, M, K, N, act=b.ACT_RELU)
    need = b.dlc_linear_workspace_bytes(cfg, True)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")

    def refused(status, f, *a):
        with pytest.raises(b.DlcError) as err:
            f(*a)
        assert err.value.status == status, err.value

    f, g = b.dlc_linear_forward, b.dlc_linear_backward
    refused(b.EINVAL, f, cfg, None, w, bias, None, y, None, work)
    refused(b.EINVAL, f, cfg, x, None, bias, None, y, None, work)
    refused(b.EINVAL, f, cfg, x, w, bias, None, None, None, work)
    refused(b.EINVAL, f, cfg, x.float(), w, bias, None, y, None, work)
    refused(b.EINVAL, f, cfg, x[:, :-1], w, bias, None, y, None, work)
    refused(b.EINVAL, f, cfg, e(M, 2 * K)[:, ::2], w, bias, None, y, None, work)
    refused(b.EINVAL, f, cfg, e(M, K + 8)[:, :K], w, bias, None, y, None, work)      # the configuration says dense rows
    refused(b.EINVAL, f, cfg, x.cpu(), w, bias, None, y, None, work)
    refused(b.EINVAL, f, cfg, x, w, e(N + 1), None, y, None, work)
    refused(b.EINVAL, g, cfg, x, w, None, y, x, w, bias, work)                       # relu needs what forward saved
    refused(b.EINVAL, g, cfg, x, w, pre, None, x, w, bias, work)
    refused(b.EINVAL, g, cfg, x, w, pre, y, x, w, bias, None)
    refused(b.ECAPACITY, g, cfg, x, w, pre, y, x, w, bias, work[:need - 1])
    refused(b.EINVAL, b.dlc_gated_backward, cfg, x, e(2 * N, K), None, y, x, e(2 * N, K), None, work)
    bad = b.make_dense_config(b.F16, M, K, N, act=9)
    refused(b.EINVAL, f, bad, x, w, bias, None, y, None, work)
    refused(b.EINVAL, f, b.make_dense_config(7, M, K, N), x, w, bias, None, y, None, work)
    refused(b.EINVAL, b.dlc_dropout, b.make_dropout_config(b.F16, M, N, 1.01), y, None, pre)
    refused(b.EINVAL, b.dlc_dropout, b.make_dropout_config(b.F16, M, N, 0.5), None, None, pre)
    refused(b.EINVAL, b.dlc_dropout, b.make_dropout_config(b.F16, M, N, 0.5, ld_x=N - 1), y, None, pre)
    # the C entry points themselves: misaligned pointers, no configuration
    L, n = b.lib(), C.c_void_p(None)
    p = lambda t, off=0: C.c_void_p(t.data_ptr() + off)
    assert L.dlc_linear_forward(C.byref(cfg), p(x, 1), p(w), n, n, p(y), n, p(work), need, n) == b.EINVAL
    assert L.dlc_linear_forward(None, p(x), p(w), n, n, p(y), n, p(work), need, n) == b.EINVAL
    assert L.dlc_linear_backward(C.byref(cfg), p(x), p(w), p(pre), p(y), p(x), p(w), n, p(work, 8), need, n) == b.EINVAL
    assert L.dlc_gated_forward(None, p(x), p(w), n, p(y), n, p(work), need, n) == b.EINVAL
    assert L.dlc_dropout(None, p(y), n, p(pre), n) == b.EINVAL
    drop = b.make_dropout_config(b.F16, M, N, 0.5)
    drop.reserved = 1
    assert L.dlc_dropout(C.byref(drop), p(y), n, p(pre), n) == b.EINVAL
    torch.cuda.synchronize()
