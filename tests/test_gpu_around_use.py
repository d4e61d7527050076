"""The norm, microscaled operands and clipping as programs use them: one after the other, on other streams, in graphs that are
replayed, two at once, on matrices past 2^32 bytes."""
import os
import sys

import numpy as np
import pytest

from dense_util import F32, assert_close
from mx_util import values

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import served_tower
    return served_tower


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_the_example_runs(dtype):
    losses, same = _example().run(steps=3, dtype=dtype, tables=4, batch=256, dim=16, report=lambda s: None)
    assert len(losses) == 3 and all(np.isfinite(losses)) and 0.0 <= same <= 1.0


def test_gradients_of_a_step():
    """f32 against the same tower in 64 bits: six layers of sums of up to 300 terms, each off by about 300 2^-24 of its terms'
    magnitudes, some twenty times the sums: 1e-3 relative at worst, 1e-4 is asked for in the norm.  Then the clipped ones."""
    import torch
    rows, features, hidden, wide = 300, 64, 48, 96
    t = _example().Tower(rows, features, hidden, wide, seed=3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    for p in t.bias + t.g:
        p += 0.1 * torch.randn(p.shape, generator=gen, device="cuda")
    x, d = torch.randn((rows, features), generator=gen, device="cuda"), torch.randn((rows, 1), generator=gen, device="cuda")
    logit, dx = t.forward(x).clone(), t.backward(x, d).clone()
    w, bias, g = ([v.double().requires_grad_() for v in p] for p in (t.w, t.bias, t.g))
    xd = x.double().requires_grad_()

    def norm(v, gain):
        return v / ((v * v).mean(dim=1, keepdim=True) + 1e-5).sqrt() * gain

    h = xd @ w[0].t() + bias[0]
    a = torch.nn.functional.silu(norm(h, g[0]) @ w[1].t() + bias[1])
    want = norm(a @ w[2].t() + bias[2] + h, g[1]) @ w[3].t() + bias[3]
    want.backward(d.double())

    def close(v, c, what):
        assert float((v.double() - c).norm()) <= 1e-4 * float(c.norm()), what

    close(logit, want.detach(), "logit")
    close(dx, xd.grad, "dx")
    all_grads = [p.grad for p in w + bias + g]
    for i, (v, c) in enumerate(zip(t.gradients.tensors, all_grads)):
        close(v, c, i)
    n = float(torch.stack([c.norm() for c in all_grads]).norm())
    before = [v.clone() for v in t.gradients.tensors]
    t.update(0.0, n / 3)
    assert abs(float(t.length) - n) <= 1e-4 * n
    for v, old in zip(t.gradients.tensors, before):
        assert_close(v, old.double() / 3, old.double().abs() * 1e-4, "clipped")


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_norm_into_a_product(rows):
    """What the norm writes in 8 bits is what the product multiplies: its result against 64 bits of the same bytes."""
    import torch
    from paper_2407_04272_amd import binding as b
    cols, n = 700, 130
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    x, w = torch.randn((rows, cols), generator=g, device="cuda"), torch.randn((n, cols), generator=g, device="cuda")
    gain = torch.rand((cols,), generator=g, device="cuda") + 0.5
    xc, wc = b.make_mx_config(b.F32, b.MX_E4M3, rows, cols), b.make_mx_config(b.F32, b.MX_E2M1, n, cols)
    (xq, xs), (wq, ws) = ([torch.empty(s, dtype=torch.uint8, device="cuda") for s in (b.dlc_mx_data_shape(c), b.dlc_mx_scale_shape(c))] for c in (xc, wc))
    b.dlc_norm_forward(b.make_norm_config(b.F32, rows, cols), x, None, gain, None, None, xq, xs)
    b.dlc_mx_quantize(wc, w, wq, ws)
    cfg = b.make_mx_linear_config(b.F32, b.MX_E4M3, rows, cols, n)
    y, work = torch.empty((rows, n), device="cuda"), torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    b.dlc_mx_linear_forward(cfg, xq, xs, wq, ws, None, None, y, work)
    xv, wv = values(xq.cpu().numpy(), xs.cpu().numpy(), cols, 8), values(wq.cpu().numpy(), ws.cpu().numpy(), cols, 4)
    want, mag = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    assert (np.abs(y.double().cpu().numpy() - want) <= mag * (cols + 2) * F32 + np.abs(want) * F32).all()


class Calls:
    """Every operator once, on inputs that can be changed; out() is what they made."""

    def __init__(self, rows=70, cols=300, n=90, seed=1):
        import torch
        from paper_2407_04272_amd import binding as b
        self.b, self.gen = b, torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        e = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        self.x, self.res, self.dy, self.w, self.gain = e(rows, cols), e(rows, cols), e(rows, cols), e(n, cols), e(cols)
        self.sum, self.y, self.dx, self.dgain, self.z = e(rows, cols), e(rows, cols), e(rows, cols), e(cols), e(rows, n)
        self.norm = b.make_norm_config(b.BF16, rows, cols)
        self.xc, self.wc = b.make_mx_config(b.BF16, b.MX_E4M3, rows, cols), b.make_mx_config(b.BF16, b.MX_E2M1, n, cols)
        self.xq, self.wq = ([e(*s, dtype=torch.uint8) for s in (b.dlc_mx_data_shape(c), b.dlc_mx_scale_shape(c))] for c in (self.xc, self.wc))
        self.lin = b.make_mx_linear_config(b.BF16, b.MX_E4M3, rows, cols, n)
        self.grads = [e(50, 40), e(33, dtype=torch.float32), e(12345, dtype=torch.float16)]
        self.out_grads = [torch.zeros_like(g) for g in self.grads]
        self.list, self.out_list = b.GradientList(self.grads), b.GradientList(self.out_grads)
        self.total, self.length = e(1, dtype=torch.float64), e(1, dtype=torch.float32)
        need = max(b.dlc_norm_workspace_bytes(self.norm), b.dlc_mx_linear_workspace_bytes(self.lin), b.dlc_gradient_workspace_bytes(self.list))
        self.work = e(need, dtype=torch.uint8)
        self.change()

    def change(self):
        import torch
        for t in (self.x, self.res, self.dy, self.w, self.gain, *self.grads):
            t.copy_(torch.randn(t.shape, generator=self.gen, device="cuda"))

    def run(self, stream=None):
        b = self.b
        b.dlc_norm_forward(self.norm, self.x, self.res, self.gain, self.sum, self.y, *self.xq, stream=stream)
        b.dlc_mx_quantize(self.wc, self.w, *self.wq, stream=stream)
        b.dlc_mx_linear_forward(self.lin, *self.xq, *self.wq, None, None, self.z, self.work, stream=stream)
        b.dlc_norm_backward(self.norm, self.sum, self.gain, self.dy, self.y, self.dx, self.dgain, self.work, stream=stream)
        b.dlc_gradient_norm(self.list, self.total, self.work, stream=stream)
        b.dlc_gradient_clip(self.list, self.total, 3.0, self.length, self.out_list, stream=stream)

    def out(self):
        return [t.clone() for t in (self.sum, self.y, self.dx, self.dgain, self.z, *self.xq, *self.wq, self.total, self.length, *self.out_grads)]

    def clear(self):
        for t in (self.sum, self.y, self.dx, self.dgain, self.z, *self.xq, *self.wq, self.total, self.length, *self.out_grads):
            t.zero_()


def _equal(a, c):
    import torch
    assert all(torch.equal(x, y) for x, y in zip(a, c))


def test_another_stream():
    import torch
    c = Calls()
    c.run()
    want = c.out()
    c.clear()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    side.synchronize()
    _equal(c.out(), want)


@pytest.mark.parametrize("rows", [9, 70, 400])
def test_graph(rows):
    """Replayed with other inputs, with eager work and synchronisation between."""
    import torch
    c, eager = Calls(rows=rows), Calls(rows=rows)
    c.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for i in range(4):
        c.change()
        for a, v in zip((eager.x, eager.res, eager.dy, eager.w, eager.gain, *eager.grads), (c.x, c.res, c.dy, c.w, c.gain, *c.grads)):
            a.copy_(v)
        c.clear()
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        eager.run()
        torch.cuda.synchronize()
        _equal(c.out(), eager.out())


def test_two_at_once():
    """Two streams, each with buffers and a workspace of its own."""
    import torch
    calls = [Calls(rows=500, cols=1000, n=600, seed=s) for s in (1, 2)]
    want = []
    for c in calls:
        c.run()
        want.append(c.out())
        c.clear()
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(calls, streams):
            c.run(stream=s)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        _equal(c.out(), w)


def test_the_same_result_every_time():
    c = Calls(rows=900, cols=2100, n=300)
    c.run()
    want = c.out()
    for _ in range(3):
        c.clear()
        c.run()
        _equal(c.out(), want)


# ---- past 2^32 bytes -----------------------------------------------------------------------------
def test_far_rows():
    """Norm, quantisation and a product of a matrix of 4.6 GB: its last rows are as those rows alone."""
    import torch
    from paper_2407_04272_amd import binding as b
    rows, cols, n, last = 1_120_000, 2048, 16, 40
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_()
    gain = torch.rand((cols,), device="cuda").bfloat16()

    def chain(v):
        m = v.shape[0]
        mx = b.make_mx_config(b.BF16, b.MX_E4M3, m, cols)
        q, s = (torch.empty(shape, dtype=torch.uint8, device="cuda") for shape in (b.dlc_mx_data_shape(mx), b.dlc_mx_scale_shape(mx)))
        y, back = torch.empty_like(v), torch.empty_like(v)
        b.dlc_norm_forward(b.make_norm_config(b.BF16, m, cols), v, None, gain, None, y, q, s)
        b.dlc_mx_dequantize(mx, q, s, back)
        return y, q, s, back

    whole, part = chain(x), chain(x[-last:].contiguous())
    for i, (a, c) in enumerate(zip(whole, part)):
        assert torch.equal(a[:, -last:] if i == 2 else a[-last:], c)
    w = torch.empty((n, cols), dtype=torch.bfloat16, device="cuda").normal_()
    wc = b.make_mx_config(b.BF16, b.MX_E2M1, n, cols)
    wq, ws = (torch.empty(shape, dtype=torch.uint8, device="cuda") for shape in (b.dlc_mx_data_shape(wc), b.dlc_mx_scale_shape(wc)))
    b.dlc_mx_quantize(wc, w, wq, ws)
    far = 2_200_000                     # rows of 8-bit elements past 2^32 bytes, and scales of several groups
    q = torch.randint(0, 120, (far, cols), dtype=torch.uint8, device="cuda")
    s = torch.randint(120, 130, (4, far, 16), dtype=torch.uint8, device="cuda")
    outs = []
    for qq, sc in ((q, s), (q[-last:].contiguous(), s[:, -last:].contiguous())):
        cfg = b.make_mx_linear_config(b.F16, b.MX_E4M3, qq.shape[0], cols, n)
        y, work = torch.empty((qq.shape[0], n), dtype=torch.float16, device="cuda"), torch.empty(b.dlc_mx_linear_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        b.dlc_mx_linear_forward(cfg, qq, sc, wq, ws, None, None, y, work)
        outs.append(y[-last:])
    # (another tile adds up in another order)
    assert torch.allclose(outs[0].double(), outs[1].double(), rtol=2 ** -9, atol=2 ** -9 * float(outs[1].abs().max()))


def test_a_large_gradient():
    """2.2e9 half-precision elements in one tensor: powers of two, so that the sum is exact."""
    import torch
    from paper_2407_04272_amd import binding as b
    n = 2_200_000_000
    g = torch.full((n,), 0.25, dtype=torch.float16, device="cuda")
    g[-1] = 4.0
    lst = b.GradientList([g])
    total, length = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    b.dlc_gradient_norm(lst, total, torch.empty(b.dlc_gradient_workspace_bytes(lst), dtype=torch.uint8, device="cuda"))
    assert float(total) == (n - 1) / 16 + 16
    b.dlc_gradient_clip(lst, total, float(total) ** 0.5 / 2, length)
    assert abs(float(length) - float(total) ** 0.5) <= 2 * F32 * float(length)
    assert bool((g[:-1] == 0.125).all()) and float(g[-1]) == 2.0
