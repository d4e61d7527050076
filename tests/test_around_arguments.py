"""What the norm, the microscaled operators and gradient clipping refuse, in the binding and at the C entry, before anything is
launched.  No GPU: tensors are stand-ins that say where they are, and every call that passes the checks has nothing to do."""
import ctypes as C

import pytest

from test_dense_arguments import Stream, Stub, _refused

INF, NAN = float("inf"), float("nan")


def _b():
    from paper_2407_04272_amd import binding as b
    return b


class At(Stub):
    """... at an address, with strides."""

    def __init__(self, dtype, *shape, ptr=4096, strides=None, **k):
        super().__init__(dtype, *shape, **k)
        self._ptr, self._strides = ptr, strides

    def data_ptr(self):
        return self._ptr

    def stride(self, i=None):
        if self._strides:
            return self._strides if i is None else self._strides[i]
        return super().stride(i) if i is not None else None


# ---- the norm -----------------------------------------------------------------------------------
def _norm_calls(device, stream, **elsewhere):
    import torch
    b = _b()
    ty, N = torch.float16, 40

    def at(name, *shape):
        return Stub(torch.uint8 if name in ("q", "scale", "work") else ty, *shape, device=elsewhere.get(name, device))

    cfg = b.make_norm_config(b.F16, 0, N)
    m = {n: at(n, 0, N) for n in ("x", "residual", "sum", "y", "s", "dy", "ds", "dx")}
    return {"forward": lambda: b.dlc_norm_forward(cfg, m["x"], m["residual"], at("weight", N), m["sum"], m["y"], at("q", 0, 128), at("scale", 1, 0, 16), stream=stream),
            "backward": lambda: b.dlc_norm_backward(cfg, m["s"], at("weight", N), m["dy"], m["ds"], m["dx"], None, at("work", 64), stream=stream)}


def _mx_calls(device, stream, **elsewhere):
    import torch
    b = _b()
    ty, K, N = torch.bfloat16, 40, 24

    def at(name, *shape):
        return Stub(ty if name in ("x", "y", "bias", "residual") else torch.uint8, *shape, device=elsewhere.get(name, device))

    cfg, lin = b.make_mx_config(b.BF16, b.MX_E2M1, 0, K), b.make_mx_linear_config(b.BF16, b.MX_E4M3, 0, K, N)
    return {"quantize": lambda: b.dlc_mx_quantize(cfg, at("x", 0, K), at("q", 0, 64), at("scale", 1, 0, 16), stream=stream),
            "dequantize": lambda: b.dlc_mx_dequantize(cfg, at("q", 0, 64), at("scale", 1, 0, 16), at("y", 0, K), stream=stream),
            "linear": lambda: b.dlc_mx_linear_forward(lin, at("xq", 0, 128), at("xs", 1, 0, 16), at("wq", N, 64), at("ws", 1, N, 16), at("bias", N),
                                                      at("residual", 0, N), at("y", 0, N), at("work", 64), stream=stream)}


TAKES = [(_norm_calls, "forward", ["x", "residual", "weight", "sum", "y", "q", "scale"]), (_norm_calls, "backward", ["s", "weight", "dy", "ds", "dx", "work"]),
         (_mx_calls, "quantize", ["x", "q", "scale"]), (_mx_calls, "dequantize", ["q", "scale", "y"]),
         (_mx_calls, "linear", ["xq", "xs", "wq", "ws", "bias", "residual", "y", "work"])]


@pytest.mark.parametrize("calls,entry,takes", TAKES, ids=[t[1] for t in TAKES])
def test_tensors_of_another_gpu(calls, entry, takes):
    for device in (0, 1):
        calls(device, Stream(device))[entry]()
        _refused(calls(device, Stream(1 - device))[entry])
        for name in takes:
            _refused(calls(device, Stream(device), **{name: 1 - device})[entry])
            _refused(calls(device, Stream(device), **{name: -1})[entry])


def test_shapes_and_types():
    import torch
    b = _b()
    f, u, S = torch.float32, torch.uint8, Stream()
    norm, x, w = b.make_norm_config(b.F32, 3, 40), Stub(f, 3, 40), Stub(f, 40)
    q, sc = Stub(u, 3, 128), Stub(u, 1, 3, 16)
    for bad in (Stub(f, 3, 41), Stub(f, 2, 40), Stub(torch.float16, 3, 40)):
        _refused(b.dlc_norm_forward, norm, bad, None, w, None, x, stream=S)
        _refused(b.dlc_norm_forward, norm, x, bad, w, None, x, stream=S)
        _refused(b.dlc_norm_backward, norm, x, w, bad, None, x, None, stream=S)
    for bq, bs in ((Stub(u, 3, 40), sc), (q, Stub(u, 3, 16)), (q, Stub(u, 3, 1, 16)), (Stub(f, 3, 128), sc), (q, None), (None, sc),
                   (Stub(u, 3, 128, contiguous=False), sc)):
        _refused(b.dlc_norm_forward, norm, x, None, w, None, None, bq, bs, stream=S)
    _refused(b.dlc_norm_forward, norm, x, None, Stub(f, 41), None, x, stream=S)
    _refused(b.dlc_norm_forward, norm, x, None, w, None, None, stream=S)          # nothing to write
    mx = b.make_mx_config(b.F32, b.MX_E2M1, 3, 40)
    for bad in (Stub(u, 3, 128), Stub(u, 3, 20), Stub(u, 2, 64)):
        _refused(b.dlc_mx_quantize, mx, x, bad, sc, stream=S)
        _refused(b.dlc_mx_dequantize, mx, bad, sc, x, stream=S)


# ---- the C entries ------------------------------------------------------------------------------
def _c(name, *a):
    return getattr(_b().lib(), name)(*a)


def test_norm_configurations():
    b = _b()

    def call(cfg, x=4096, res=None, w=4096, s=None, y=8192, q=None, sc=None):
        return _c("dlc_norm_forward", C.byref(cfg), x, res, w, s, y, q, sc, None)

    mk = b.make_norm_config
    assert call(mk(b.F32, 0, 8)) == b.OK and b.dlc_norm_workspace_bytes(mk(b.F32, 5, 8)) > 0
    for bad in [mk(3, 0, 8), mk(b.F32, -1, 8), mk(b.F32, (1 << 30) + 1, 8), mk(b.F32, 0, 0), mk(b.F32, 0, (1 << 20) + 1), mk(b.F32, 0, 8, eps=0.0),
                mk(b.F32, 0, 8, eps=-1.0), mk(b.F32, 0, 8, eps=NAN), mk(b.F32, 0, 8, eps=INF), mk(b.F32, 0, 8, eps=1e-39),
                mk(b.F32, 0, 8, ld_x=7), mk(b.F32, 0, 8, ld_dx=-1), mk(b.F32, 1 << 30, 8, ld_y=1 << 40)]:
        assert call(bad) == b.EINVAL and b.dlc_norm_workspace_bytes(bad) == 0
    three = mk(b.F16, 3, 8)
    for kw in [dict(x=None), dict(x=4097), dict(w=4097), dict(y=None), dict(y=8193), dict(q=4096), dict(sc=4096), dict(q=4104, sc=4096), dict(q=4096, sc=4104),
               dict(s=4096, y=4096), dict(res=8192, y=8192)]:
        assert call(three, **kw) == b.EINVAL, kw
    apart = mk(b.F16, 3, 8, ld_x=9, ld_res=9)
    assert call(apart, s=4096) == b.EINVAL and call(apart, y=4096) == b.EINVAL and call(apart, res=2048, s=2048) == b.EINVAL

    def back(cfg, s=4096, w=4096, dy=8192, ds=None, dx=16384, dw=None, work=None, size=0):
        return _c("dlc_norm_backward", C.byref(cfg), s, w, dy, ds, dx, dw, work, size, None)

    assert back(mk(b.F16, 0, 8)) == b.OK and back(three, dx=None) == b.OK
    for kw in [dict(s=None), dict(dy=None), dict(dx=4096), dict(dy=8193), dict(dw=4097), dict(dw=4096), dict(dw=4096, work=4104, size=1 << 20)]:
        assert back(three, **kw) == b.EINVAL, kw
    assert back(three, dw=4096, work=65536, size=b.dlc_norm_workspace_bytes(three) - 1) == b.ECAPACITY
    assert back(mk(b.F16, 3, 8, ld_dx=9), dx=8192) == b.EINVAL and back(mk(b.F16, 3, 8, ld_dx=9), ds=2048, dx=2048) == b.EINVAL


def test_mx_configurations():
    b = _b()
    mk, lin = b.make_mx_config, b.make_mx_linear_config
    data, scale = (lambda c: _c("dlc_mx_data_bytes", C.byref(c))), (lambda c: _c("dlc_mx_scale_bytes", C.byref(c)))
    for rows, cols in ((1, 1), (3, 128), (3, 129), (7, 512), (5, 513), (2, 1 << 20)):
        for elem in (b.MX_E2M1, b.MX_E4M3):
            c = mk(b.F32, elem, rows, cols)
            for bytes_, shape in ((data(c), b.dlc_mx_data_shape(c)), (scale(c), b.dlc_mx_scale_shape(c))):
                n = 1
                for v in shape:
                    n *= v
                assert bytes_ == n
            assert data(c) == rows * -(-cols // 128) * 128 * elem // 8 and scale(c) == rows * -(-cols // 512) * 16

    def quant(cfg, x=4096, q=8192, sc=16384, entry="dlc_mx_quantize"):
        return _c(entry, C.byref(cfg), *((q, sc, x) if "deq" in entry else (x, q, sc)), None)

    assert quant(mk(b.F16, b.MX_E2M1, 0, 8)) == b.OK and quant(mk(b.F16, b.MX_E4M3, 0, 8), entry="dlc_mx_dequantize") == b.OK
    for bad in [mk(3, 4, 0, 8), mk(b.F32, 0, 0, 8), mk(b.F32, 6, 0, 8), mk(b.F32, 4, -1, 8), mk(b.F32, 4, 0, 0), mk(b.F32, 4, 0, (1 << 20) + 1),
                mk(b.F32, 4, (1 << 30) + 1, 8), mk(b.F32, 4, 0, 8, ld_x=7), mk(b.F32, 4, 0, 8, ld_y=7)]:
        assert quant(bad) == b.EINVAL and data(bad) == 0 and scale(bad) == 0
    for kw in [dict(x=None), dict(x=4097), dict(q=None), dict(q=8200), dict(sc=None), dict(sc=16392)]:
        for entry in ("dlc_mx_quantize", "dlc_mx_dequantize"):
            assert quant(mk(b.F16, 4, 2, 8), entry=entry, **kw) == b.EINVAL, kw

    def call(cfg, xq=4096, xs=8192, wq=16384, ws=32768, bias=None, res=None, y=65536, work=None, size=0):
        return _c("dlc_mx_linear_forward", C.byref(cfg), xq, xs, wq, ws, bias, res, y, work, size, None)

    assert call(lin(b.F16, 4, 0, 8, 8)) == b.OK
    for bad in [lin(3, 4, 0, 8, 8), lin(b.F16, 5, 0, 8, 8), lin(b.F16, 4, -1, 8, 8), lin(b.F16, 4, 0, 0, 8), lin(b.F16, 4, 0, 8, 0), lin(b.F16, 4, 0, 8, 8, act=5),
                lin(b.F16, 4, 0, (1 << 20) + 1, 8), lin(b.F16, 4, 0, 8, (1 << 20) + 1), lin(b.F16, 4, 0, 8, 8, ld_y=7), lin(b.F16, 4, 0, 8, 8, ld_res=7),
                lin(b.F16, 4, 1 << 30, 8, 2000)]:
        assert call(bad) == b.EINVAL and b.dlc_mx_linear_workspace_bytes(bad) == 0
    two = lin(b.F16, 8, 2, 8, 8)
    for kw in [dict(xq=None), dict(xs=None), dict(wq=None), dict(ws=None), dict(y=None), dict(xq=4104), dict(xs=4104), dict(wq=4104), dict(ws=4104),
               dict(bias=4097), dict(res=4097), dict(y=4097), dict(work=4104)]:
        assert call(two, **kw) == b.EINVAL, kw
    assert call(lin(b.F16, 8, 2, 8, 8, ld_y=9), res=65536) == b.EINVAL


# ---- gradients ----------------------------------------------------------------------------------
def _entry(p=4096, rows=2, cols=8, ld=0, dtype=0, reserved=0):
    return _b().Tensor(p, rows, cols, ld, dtype, reserved)


def _entries(*e):
    return (_b().Tensor * len(e))(*e)


def test_gradient_lists_at_the_entry():
    b = _b()

    def norm(lst, count=None, total=4096, work=8192, size=1 << 20):
        return _c("dlc_gradient_norm", lst, len(lst) if count is None else count, total, work, size, None)

    def clip(lst, out=None, total=4096, limit=1.0, n=None, count=None):
        return _c("dlc_gradient_clip", lst, len(lst) if count is None else count, total, limit, n, lst if out is None else out, None)

    none = _entries(_entry(None, 0, 8), _entry(None, 5, 0))
    assert clip(none) == b.OK and clip(_entries()) == b.OK
    assert _c("dlc_gradient_workspace_bytes", none, 2) == 0 and _c("dlc_gradient_workspace_bytes", _entries(_entry()), 1) == 8
    for bad in [_entry(None), _entry(4097), _entry(4098), _entry(dtype=3), _entry(rows=-1), _entry(cols=-1), _entry(ld=7), _entry(reserved=1), _entry(4097, dtype=1)]:
        e = _entries(_entry(), bad)
        assert norm(e) == b.EINVAL and clip(e) == b.EINVAL and _c("dlc_gradient_workspace_bytes", e, 2) == 0
    for far in [_entry(rows=1 << 21, cols=1 << 20), _entry(rows=1 << 31, cols=1 << 33), _entry(rows=1 << 30, cols=8, ld=1 << 40)]:
        assert norm(_entries(far)) == b.ELIMIT and clip(_entries(far)) == b.ELIMIT
    many = _entries(*[_entry(rows=1 << 20, cols=1 << 20) for _ in range(17)])
    assert norm(many) == b.ELIMIT and _c("dlc_gradient_workspace_bytes", many, 16) > 0
    one = _entries(_entry())
    assert norm(one, total=None) == b.EINVAL and norm(one, total=4100) == b.EINVAL and norm(one, work=None) == b.EINVAL and norm(one, work=8200) == b.EINVAL
    assert norm(one, size=7) == b.ECAPACITY and norm(one, count=-1) == b.EINVAL and norm(None, count=1) == b.EINVAL
    for kw in [dict(total=None), dict(total=4100), dict(limit=-1.0), dict(limit=NAN), dict(n=4097), dict(out=_entries(_entry(rows=3))),
               dict(out=_entries(_entry(cols=9))), dict(out=_entries(_entry(dtype=1))), dict(out=_entries(_entry(ld=9)))]:
        assert clip(one, **kw) == b.EINVAL, kw


def test_gradient_lists_of_the_binding():
    import torch
    b = _b()
    f = torch.float32
    lst = b.GradientList([At(f, 3, 5), At(torch.bfloat16, 7, ptr=8192), At(f, 4, 6, ptr=16384, strides=(9, 1), contiguous=False),
                          At(f, 5, ptr=32768, strides=(3,), contiguous=False), At(f, 2, 3, 4, ptr=65536), At(f, 0, ptr=0)])
    got = [(e.rows, e.cols, e.ld, e.dtype) for e in lst.entries]
    assert got[0] in ((3, 5, 5, b.F32), (3, 5, 0, b.F32)) and got[2:] == [(4, 6, 9, b.F32), (5, 1, 3, b.F32), (1, 24, 0, b.F32), (1, 0, 0, b.F32)]
    assert got[1][3] == b.BF16 and lst.device == 0 and len(lst) == 6
    for bad in ([At(torch.float64, 3)], [At(torch.int32, 3)], [At(f, 3, device=-1)], [At(f, 3), At(f, 4, device=1)], [At(f, 3), At(f, 3)],
                [At(f, 4, 6, strides=(1, 4), contiguous=False)], [At(f, 4, 6, strides=(0, 1), contiguous=False)], [At(f, 5, strides=(0,), contiguous=False)],
                [At(f, 2, 3, 4, strides=(24, 8, 1), contiguous=False)]):
        _refused(b.GradientList, bad)
    total, n = Stub(torch.float64, 1), Stub(f, 1)
    one, other = b.GradientList([At(f, 0)]), b.GradientList([At(f, 0, device=1)])
    b.dlc_gradient_clip(b.GradientList([]), total, 1.0, stream=Stream())
    b.dlc_gradient_clip(one, total, 1.0, stream=Stream())
    b.dlc_gradient_clip(other, Stub(torch.float64, 1, device=1), 1.0, stream=Stream(1))
    _refused(b.dlc_gradient_clip, other, total, 1.0, stream=Stream())
    for bad in (Stub(f, 1), Stub(torch.float64, 0), Stub(torch.float64, 1, device=1), Stub(torch.float64, 1, device=-1)):
        _refused(b.dlc_gradient_clip, one, bad, 1.0, stream=Stream())
        _refused(b.dlc_gradient_norm, one, bad, stream=Stream())
    for bad in (Stub(torch.float64, 1), Stub(f, 0), Stub(f, 1, device=1)):
        _refused(b.dlc_gradient_clip, one, total, 1.0, bad, stream=Stream())
    _refused(b.dlc_gradient_clip, one, total, 1.0, None, b.GradientList([At(f, 0), At(f, 0)]), stream=Stream())
    _refused(b.dlc_gradient_clip, one, total, 1.0, None, b.GradientList([At(torch.float16, 0)]), stream=Stream())
    _refused(b.dlc_gradient_norm, one, total, Stub(torch.uint8, 64, device=1), stream=Stream())


def test_gradients_that_overlap():
    """Memory that two entries share would be counted twice, and clipped by two work-groups at once."""
    import torch
    b = _b()
    f, total = torch.float32, Stub(torch.float64, 1)
    _refused(b.GradientList, [At(f, 10, ptr=4096), At(f, 10, ptr=4096 + 36)])
    _refused(b.GradientList, [At(f, 10, ptr=4096 + 36), At(f, 2, 5, ptr=4096)])
    _refused(b.GradientList, [At(f, 100, ptr=4096), At(f, 1, ptr=8192), At(f, 3, ptr=4096 + 40)])
    _refused(b.GradientList, [At(f, 100, ptr=4096), At(torch.float16, 2, ptr=4096 + 4), At(f, 1, ptr=4096 + 200)])

    def rows(ptr):
        return At(f, 4, 2, ptr=ptr, strides=(4, 1), contiguous=False)

    # side by side, and rows between rows
    lst = b.GradientList([At(f, 10, ptr=4096), At(f, 10, ptr=4096 + 40), rows(8192), rows(8200)])
    for p, q in ((4096 + 40, 4096), (4096 + 4, 65536), (65536, 4096 + 36), (65536, 4096)):
        _refused(b.dlc_gradient_clip, lst, total, 1.0, None, b.GradientList([At(f, 10, ptr=p), At(f, 10, ptr=q), rows(1 << 20), rows((1 << 20) + 8)]), stream=Stream())
    _refused(b.dlc_gradient_clip, lst, total, 1.0, None, b.GradientList([At(f, 10, ptr=65536), At(f, 10, ptr=65536 + 40), rows(8200), rows(1 << 20)]), stream=Stream())
    # some of the outputs may be the gradients themselves
    for p, q in ((4096, 65536), (65536, 4096 + 40), (4096, 4096 + 40), (65536, 65536 + 40)):
        b._check_apart(lst, b.GradientList([At(f, 10, ptr=p), At(f, 10, ptr=q), rows(8192), rows(1 << 20)]))


# ---- one configuration, several threads -----------------------------------------------------------
def _linear_tensors(M, K, N):
    import torch
    u = torch.uint8
    return [Stub(u, M, -(-K // 128) * 128), Stub(u, -(-K // 512), M, 16), Stub(u, N, -(-K // 128) * 64), Stub(u, -(-K // 512), N, 16), None, None,
            Stub(torch.float32, M, N)]


def test_a_call_in_the_middle_of_another():
    """What a call keeps on its configuration is complete whenever another thread may read it: here the other's whole call stands
    behind every single attribute that the first one sets."""
    b = _b()
    inner = []

    class Watched(b.MxLinearConfig):
        def __setattr__(self, name, value):
            super().__setattr__(name, value)
            if name not in fields and not inner:
                inner.append(name)
                b.dlc_mx_linear_forward(self, *_linear_tensors(0, self.in_features, self.out_features), stream=Stream())

    fields = {f for f, _ in b.MxLinearConfig._fields_}
    cfg = Watched(b.F32, b.ACT_NONE, b.MX_E4M3, 0, 0, 40, 24, 0, 0)
    for K, N in ((40, 24), (700, 24), (700, 30)):
        cfg.in_features, cfg.out_features = K, N
        del inner[:]
        b.dlc_mx_linear_forward(cfg, *_linear_tensors(0, K, N), stream=Stream())
        _refused(b.dlc_mx_linear_forward, cfg, *_linear_tensors(0, K + 512, N), stream=Stream())
        _refused(b.dlc_mx_linear_forward, cfg, *_linear_tensors(0, K, N + 1), stream=Stream())


def test_threads_that_share_a_configuration():
    import sys
    import threading
    b = _b()
    b.lib()
    wrong, was = [], sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        for _ in range(300):
            cfg, start = b.make_mx_linear_config(b.F32, b.MX_E4M3, 0, 40, 24), threading.Barrier(6)

            def call():
                start.wait()
                try:
                    b.dlc_mx_linear_forward(cfg, *_linear_tensors(0, 40, 24), stream=Stream())
                except Exception as e:
                    wrong.append(e)

            threads = [threading.Thread(target=call) for _ in range(6)]
            for t in threads:
                t.start()
            for t in threads:
                t.join()
    finally:
        sys.setswitchinterval(was)
    assert not wrong, wrong[0]
