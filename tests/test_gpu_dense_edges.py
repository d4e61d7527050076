"""Dense operators where numbers run out: infinities and NaN in what a backward call reads, saturated units.

Rule of the backward pass: a product with a factor of 0 (a dropped element, a dy of 0, a slope of 0) is 0 whatever the other
factor holds, and values and slopes at infinite pre-activations are their limits."""
import pytest

from dense_util import ACTS, F32, FN, ROUND, act, assert_close, code, drop_factor, product, rounded, torch_type

pytestmark = pytest.mark.gpu
TYPES = ["f32", "f16", "bf16"]
SEED, OFFSET = 0x1234567890ABCDEF, 77


def _normal(gen, dtype, *shape, scale=1.0):
    import torch
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(torch_type(dtype))


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _call_backward(op, dtype, name, p, x, w, pre, dy):
    import torch
    from paper_2407_04272_amd import binding as b
    (M, K), N = x.shape, dy.shape[1]
    cfg = b.make_dense_config(code(dtype), M, K, N, act=ACTS.index(name), dropout_p=p, seed=SEED, offset=OFFSET)
    size, call = ((b.dlc_gated_workspace_bytes, b.dlc_gated_backward) if op == "gated" else
                  (b.dlc_linear_workspace_bytes, b.dlc_linear_backward))
    work = torch.full((size(cfg, True),), 0xFF, dtype=torch.uint8, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(w.shape[0], dtype=w.dtype, device="cuda")
    call(cfg, x, w, pre, dy, dx, dw, db, work)
    return dx, dw, db


def _check_grads(dtype, what, got, x, w, dz, edz):
    """dz in 64 bits with the bound edz on what the call may make of it: see tests/test_gpu_dense.py"""
    dx, dw, db = got
    x, w, M = x.double(), w.double(), x.shape[0]
    half = edz + ROUND[dtype] * dz.abs() + 2.0 ** -25
    v, e = product(dz, w.t())
    assert_close(dx, v, rounded(v, e + half @ w.abs(), dtype), what + " dx")
    v, e = product(dz.t(), x.t())
    assert_close(dw, v, rounded(v, e + half.t() @ x.abs(), dtype), what + " dw")
    v, e = dz.sum(0), edz.sum(0) + (M + 2) * F32 * dz.abs().sum(0)
    assert_close(db, v, rounded(v, e, dtype), what + " dbias")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ACTS)
def test_linear_gradients_of_infinite_pre_activations(dtype, name):
    """Every activation's slope has a finite limit at both ends, so the gradients are finite; NaN stands where it is dropped
    or where dy is 0."""
    import torch
    inf, nan = float("inf"), float("nan")
    M, K, N = 70, 96, 72
    for p in (0.0, 0.5):
        g = _gen(31)
        x, w, dy = _normal(g, dtype, M, K), _normal(g, dtype, N, K, scale=K ** -0.5), _normal(g, dtype, M, N)
        pre = _normal(g, dtype, M, N)
        pick = torch.rand((M, N), generator=g, device="cuda")
        pre[pick < 0.1] = inf
        pre[pick > 0.9] = -inf
        dy[(pick > 0.4) & (pick < 0.5)] = 0.0
        f = torch.from_numpy(drop_factor(M, N, p, SEED, OFFSET)).cuda() if p else torch.ones((M, N), dtype=torch.float64, device="cuda")
        off = (f == 0) | (dy == 0)
        if name != "none":
            pre[off & (pick < 0.6)] = nan
        dy[(f == 0) & (pick > 0.6)] = nan     # dropped: whatever it holds
        if name == "relu":
            dy[(pick > 0.9)] = inf            # behind a closed unit
        z = torch.nan_to_num(pre.double(), nan=0.0, posinf=1e4, neginf=-1e4)   # (the slopes' limits)
        d = torch.where(f == 0, torch.zeros_like(f), dy.double() * f)
        s = act(name, z)[1]
        dz = torch.where((d == 0) | (s == 0), torch.zeros_like(d), d * s)
        edz = (torch.where(torch.isfinite(d), d.abs(), torch.zeros_like(d)) * FN if name not in ("none", "relu") else 0.0) + 2 * F32 * dz.abs()
        _check_grads(dtype, f"linear {dtype} {name} {p}", _call_backward("linear", dtype, name, p, x, w, pre, dy), x, w, dz, edz)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ACTS)
def test_gated_gradients_of_infinite_pre_activations(dtype, name):
    """Infinities where the other factors are 0: dropped, dy = 0, or the gate's limits."""
    import torch
    inf, nan = float("inf"), float("nan")
    M, K, N = 70, 96, 72
    for p in (0.0, 0.5):
        g = _gen(37)
        x, w, dy = _normal(g, dtype, M, K), _normal(g, dtype, 2 * N, K, scale=K ** -0.5), _normal(g, dtype, M, N)
        pre = _normal(g, dtype, M, 2 * N)
        gate, up = pre[:, :N], pre[:, N:]
        pick = torch.rand((M, N), generator=g, device="cuda")
        dy[(pick > 0.4) & (pick < 0.5)] = 0.0
        f = torch.from_numpy(drop_factor(M, N, p, SEED, OFFSET)).cuda() if p else torch.ones((M, N), dtype=torch.float64, device="cuda")
        off = (f == 0) | (dy == 0)
        dy[(f == 0) & (pick > 0.6)] = nan
        if name != "none":                    # the value's and the slope's limit are 0 (sigmoid: at both ends the slope's)
            gate[pick < 0.15] = -inf
            up[pick < 0.05] = inf
            up[(pick >= 0.05) & (pick < 0.1)] = -inf
        if name == "sigmoid":
            gate[pick > 0.9] = inf
            up[pick > 0.95] = inf
        if name == "relu":                    # a closed gate stops what comes from behind, too
            gate[(pick > 0.2) & (pick < 0.25)] = -1.0
            up[(pick > 0.2) & (pick < 0.25)] = inf
            dy[(pick > 0.22) & (pick < 0.25)] = inf
        gate[off & (pick > 0.3)] = inf
        up[off & (pick > 0.35)] = -inf
        gate[off & (pick > 0.45) & (pick < 0.7)] = nan
        up[off & (pick > 0.65) & (pick < 0.8)] = nan
        z = torch.nan_to_num(gate.double(), nan=0.0, posinf=1e4, neginf=-1e4)
        u = up.double()
        d = torch.where(f == 0, torch.zeros_like(f), dy.double() * f)
        v, s = act(name, z)

        def times(*a):
            r = a[0]
            for q in a[1:]:
                r = torch.where((r == 0) | (q == 0), torch.zeros_like(r), r * q)
            return r

        dz = torch.cat((times(d, s, u), times(d, v)), 1)
        assert bool(torch.isfinite(dz).all())
        mag = torch.cat((times(d.abs(), (s != 0).double(), u.abs()), times(d.abs(), (v != 0).double())), 1)
        edz = mag * FN + 4 * F32 * dz.abs()
        _check_grads(dtype, f"gated {dtype} {name} {p}", _call_backward("gated", dtype, name, p, x, w, pre, dy), x, w, dz, edz)


@pytest.mark.parametrize("op", ["linear", "gated"])
@pytest.mark.parametrize("name", ["relu", "sigmoid", "silu", "gelu"])
def test_sums_past_the_largest_f16(op, name):
    """|z| > 65504 is saved as an infinity; the layer's output and gradients are those of z all the same."""
    import torch
    from paper_2407_04272_amd import binding as b
    M, K, N = 40, 16, 24
    wide = 2 * N if op == "gated" else N
    g = _gen(41)
    x, w = _normal(g, "f16", M, K), _normal(g, "f16", wide, K, scale=0.25)
    x[:, 0] = 300.0
    w[:, 0] = 0.0
    w[0:3, 0] = -250.0            # z about -75000 in three (gate) columns
    if op == "linear":
        w[3:5, 0] = 200.0         # and 60000, finite, in two
    dy = _normal(g, "f16", M, N)
    cfg = b.make_dense_config(b.F16, M, K, N, act=ACTS.index(name))
    fwd, size = ((b.dlc_gated_forward, b.dlc_gated_workspace_bytes) if op == "gated" else (b.dlc_linear_forward, b.dlc_linear_workspace_bytes))
    work = torch.empty(max(16, size(cfg)), dtype=torch.uint8, device="cuda")
    y, pre = torch.empty((M, N), dtype=torch.float16, device="cuda"), torch.empty((M, wide), dtype=torch.float16, device="cuda")
    fwd(cfg, x, w, None, *(() if op == "gated" else (None,)), y, pre, work)
    assert bool(torch.isinf(pre[:, :3]).all()) and bool((y[:, :3] == 0).all())
    z = pre.double().clamp(min=-1e4)        # (every slope and value is at its limit there)
    d = dy.double()
    if op == "gated":
        v, s = act(name, z[:, :N])
        dz = torch.cat((d * z[:, N:] * s, d * v), 1)
        edz = torch.cat((d.abs() * z[:, N:].abs(), d.abs()), 1) * FN + 4 * F32 * dz.abs()
    else:
        dz = d * act(name, z)[1]
        edz = (d.abs() * FN if name != "relu" else 0.0) + 2 * F32 * dz.abs()
    got = _call_backward(op, "f16", name, 0.0, x, w, pre, dy)
    assert all(bool(torch.isfinite(t[:3] if t.dim() == 1 else t).all()) for t in got[1:])
    _check_grads("f16", f"{op} {name}", got, x, w, dz, edz)


def test_what_is_kept_shows():
    """Only a factor of 0 hides what is not finite."""
    import torch
    inf, nan = float("inf"), float("nan")
    g = _gen(43)
    x, w = _normal(g, "f32", 20, 16), _normal(g, "f32", 16, 16)
    pre, dy = torch.ones((20, 16), device="cuda"), torch.ones((20, 8), device="cuda")
    pre[3, 8 + 2] = inf       # u of column 2
    pre[5, 4] = nan           # the gate of column 4
    dy[7, 6] = -inf
    dx, dw, db = _call_backward("gated", "f32", "silu", 0.0, x, w, pre, dy)
    bad = ~torch.isfinite(db)
    assert bad.nonzero().flatten().tolist() == [2, 4, 6, 8 + 4, 8 + 6] and float(db[2]) == inf and bool(torch.isnan(db[4]))
    assert (~torch.isfinite(dx)).any(1).nonzero().flatten().tolist() == [3, 5, 7]
    pre = torch.ones((20, 16), device="cuda")
    pre[5, 4] = nan
    dy = torch.ones((20, 16), device="cuda")
    dy[7, 6] = -inf
    db = _call_backward("linear", "f32", "gelu", 0.0, x, w, pre, dy)[2]
    assert (~torch.isfinite(db)).nonzero().flatten().tolist() == [4, 6] and float(db[6]) == -inf


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("op", ["linear", "gated"])
def test_slope_of_a_saturated_sigmoid(op, dtype):
    """The slope e / (1 + e)^2, e = exp(-|z|), is even and keeps its digits far out.  Relative bound: the exponential's argument
    is off by 2 units of 2^-24 of |z| log2 e (44 at most), the exponential and the reciprocal by 2 units each (the latter counts
    twice), three products and a sum by one: 2 * 44 + 2 + 4 + 5 < 128.  One row, so that the bias gradient is dz itself."""
    import torch
    N = 1 << 13
    lin = torch.linspace(0, 30, N // 2, device="cuda")
    z = torch.cat((lin, -lin))[None].to(torch_type(dtype))
    g = _gen(47)
    dy = (_normal(g, dtype, 1, N, scale=0.1).float().abs() + 1).to(torch_type(dtype)) * 256
    if op == "gated":
        up = torch.full((1, N), 1.0, dtype=z.dtype, device="cuda")
        z2 = torch.cat((z, up), 1)
    x = torch.ones((1, 8), dtype=z.dtype, device="cuda")
    w = torch.zeros((2 * N if op == "gated" else N, 8), dtype=z.dtype, device="cuda")
    dx, dw, db = _call_backward(op, dtype, "sigmoid", 0.0, x, w, z2 if op == "gated" else z, dy)
    e = torch.exp(-z[0].double().abs())
    dz = dy[0].double() * e / (1 + e) ** 2
    err = 128 * F32 * dz
    assert_close(db[:N], dz, rounded(dz, err, dtype), f"{op} {dtype} dbias")
    # (dw holds dz rounded to the type, times one)
    assert_close(dw[:N, 0], dz, rounded(dz, err + rounded(dz, err, dtype), dtype), f"{op} {dtype} dw")
    if op == "gated":
        q = torch.sigmoid(z[0].double())
        v = dy[0].double() * q
        assert_close(db[N:], v, rounded(v, 128 * F32 * v, dtype), f"{op} {dtype} dbias of u")


def test_a_saturated_sigmoid_is_not_closed():
    """Its slope at 20 is 2e-9, not 0: what is not finite in dy shows."""
    import torch
    z, dy = torch.full((1, 8), 20.0, device="cuda"), torch.full((1, 8), float("inf"), device="cuda")
    z[0, 4:] *= -1
    x, w = torch.ones((1, 8), device="cuda"), torch.ones((8, 8), device="cuda")
    assert bool(torch.isinf(_call_backward("linear", "f32", "sigmoid", 0.0, x, w, z, dy)[2]).all())


def _values(dtype):
    """Pre-activations from tiny to past where every exponential overflows"""
    import torch
    v = torch.cat((torch.linspace(0, 40, 2001, dtype=torch.float64), torch.logspace(1.5, 4.5, 200, dtype=torch.float64),
                   torch.tensor([65504.0]), torch.logspace(-7, 0, 100, dtype=torch.float64)))
    if dtype != "f16":
        v = torch.cat((v, torch.logspace(5, 38, 200, dtype=torch.float64)))
    v = torch.cat((v, -v)).to(torch_type(dtype))
    return v[torch.isfinite(v)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("rows", [1, 40])
def test_activations_far_out(name, dtype, rows):
    """y = act(z) for one z a column (x is 1 in one place, w holds z there): relative to the value, where that can be asked
    for.  The exponential's argument is off by a unit of 2^-24 of itself or two, which is 2 |z| units of the result (gelu:
    z^2 / 2 is the argument, rounded four times, the quotient's argument once, and erfc's fit is off by 3 units); a few
    roundings more.  A value that a normal fp32 number does not hold may be 0; its factor z comes after."""
    import torch
    from paper_2407_04272_amd import binding as b
    v = _values(dtype)
    N = v.numel()
    x = torch.zeros((rows, 16), dtype=v.dtype, device="cuda")
    x[:, 3] = 1.0
    w = torch.zeros((N, 16), dtype=v.dtype, device="cuda")
    w[:, 3] = v.cuda()
    y, pre = torch.empty((rows, N), dtype=v.dtype, device="cuda"), torch.empty((rows, N), dtype=v.dtype, device="cuda")
    cfg = b.make_dense_config(code(dtype), rows, 16, N, act=ACTS.index(name))
    work = torch.empty(max(16, b.dlc_linear_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
    b.dlc_linear_forward(cfg, x, w, None, None, y, pre, work)
    z = v.double().cuda()
    assert torch.equal(pre, v.cuda().expand(rows, N))
    if name in ("none", "relu"):
        assert torch.equal(y, (v.clamp(min=0) if name == "relu" else v).cuda().expand(rows, N))
        return
    want = act(name, z)[0]
    units = 16 + (4 * z * z if name == "gelu" else 4 * z.abs())
    units = torch.where(z > 0, torch.full_like(z, 16.0), units)       # (1 - something small, or 0.5 and more)
    err = units.clamp(max=2.0 ** 24) * F32 * want.abs() + 2.0 ** -126 * z.abs().clamp(min=1)
    assert_close(y, want.expand(rows, N), rounded(want, err, dtype).expand(rows, N), f"{name} {dtype}")


@pytest.mark.parametrize("dtype", TYPES)
def test_activations_at_infinity(dtype):
    import torch
    from paper_2407_04272_amd import binding as b
    inf = float("inf")
    x = torch.ones((1, 8), dtype=torch_type(dtype), device="cuda")
    w = torch.zeros((4, 8), dtype=torch_type(dtype), device="cuda")
    w[0, 0], w[1, 0], w[2, 0], w[3, 0] = inf, -inf, float("nan"), 1.0
    for name, high, low in (("none", inf, -inf), ("relu", inf, 0.0), ("sigmoid", 1.0, 0.0), ("silu", inf, None), ("gelu", inf, None)):
        y = torch.empty((1, 4), dtype=x.dtype, device="cuda")
        b.dlc_linear_forward(b.make_dense_config(code(dtype), 1, 8, 4, act=ACTS.index(name)), x, w, None, None, y)
        assert float(y[0, 0]) == high and bool(torch.isnan(y[0, 2])) and bool(torch.isfinite(y[0, 3])), name
        if low is not None:
            assert float(y[0, 1]) == low, name
