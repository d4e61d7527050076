"""What the binding of the dense operators refuses before anything is launched.  No GPU: the tensors are stand-ins that say
where they are, and every call that passes the checks has no rows."""
import pytest


class Stub:
    """As much of a tensor on a GPU as the binding asks for."""

    def __init__(self, dtype, *shape, device=0, contiguous=True):
        import torch
        self.dtype, self.shape = dtype, torch.Size(shape)
        self.device = torch.device("cuda", device) if device >= 0 else torch.device("cpu")
        self.is_cuda = device >= 0
        self._contiguous = contiguous

    def get_device(self):
        return self.device.index if self.is_cuda else -1

    def is_contiguous(self):
        return self._contiguous

    def numel(self):
        n = 1
        for v in self.shape:
            n *= v
        return n

    def element_size(self):
        return self.dtype.itemsize

    def stride(self, i):
        return 1 if i == len(self.shape) - 1 else self.shape[-1]

    def data_ptr(self):
        return 4096


class Stream:
    def __init__(self, device=0):
        self.device_index, self.cuda_stream = device, 0


def _refused(f, *a, **k):
    from paper_2407_04272_amd import binding as b
    with pytest.raises(b.DlcError) as err:
        f(*a, **k)
    assert err.value.status == b.EINVAL, err.value


def test_the_counter_of_a_replayed_graph():
    """d_offset is read by kernels: one whole 64-bit word on a GPU, or nothing."""
    import torch
    from paper_2407_04272_amd import binding as b
    made = [lambda t: b.make_dense_config(b.F32, 8, 8, 8, dropout_p=0.5, d_offset=t),
            lambda t: b.make_dropout_config(b.F32, 8, 8, 0.5, d_offset=t)]
    for make in made:
        _refused(make, torch.zeros(1, dtype=torch.int64))                 # host memory
        _refused(make, Stub(torch.int32, 1))
        _refused(make, Stub(torch.float64, 1))
        _refused(make, Stub(torch.int64, 0))
        assert make(None).d_offset is None
        for dtype in (torch.int64, torch.uint64):
            t = Stub(dtype, 1)
            assert make(t).d_offset == t.data_ptr()


def _calls(device, stream, **elsewhere):
    """Every entry point with no rows, its tensors on `device` but for the named ones"""
    import torch
    from paper_2407_04272_amd import binding as b
    ty, K, N = torch.float16, 16, 8

    def at(name, *shape):
        return Stub(torch.uint8 if name == "work" else ty, *shape, device=elsewhere.get(name, device))

    cfg = b.make_dense_config(b.F16, 0, K, N, act=b.ACT_SILU)
    drop = b.make_dropout_config(b.F16, 0, N, 0.5)
    x, res, y, dy, dx, work = (at("x", 0, K), at("residual", 0, N), at("y", 0, N), at("dy", 0, N), at("dx", 0, K), at("work", 64))
    w, bias, pre, dw, db = (lambda n: at("w", n, K)), (lambda n: at("bias", n)), (lambda n: at("pre", 0, n)), (lambda n: at("dw", n, K)), (lambda n: at("dbias", n))
    return {"linear_forward": lambda: b.dlc_linear_forward(cfg, x, w(N), bias(N), res, y, pre(N), work, stream=stream),
            "gated_forward": lambda: b.dlc_gated_forward(cfg, x, w(2 * N), bias(2 * N), y, pre(2 * N), work, stream=stream),
            "linear_backward": lambda: b.dlc_linear_backward(cfg, x, w(N), pre(N), dy, dx, None, None, work, stream=stream),
            "gated_backward": lambda: b.dlc_gated_backward(cfg, x, w(2 * N), pre(2 * N), dy, dx, None, None, work, stream=stream),
            "dropout": lambda: b.dlc_dropout(drop, at("x", 0, N), res, y, stream=stream)}


TAKES = {"linear_forward": ["x", "w", "bias", "residual", "y", "pre", "work"], "gated_forward": ["x", "w", "bias", "y", "pre", "work"],
         "linear_backward": ["x", "w", "pre", "dy", "dx", "work"], "gated_backward": ["x", "w", "pre", "dy", "dx", "work"],
         "dropout": ["x", "residual", "y"]}


@pytest.mark.parametrize("entry", sorted(TAKES))
def test_tensors_of_another_gpu(entry):
    """A call goes to the GPU of its stream, and every tensor has to be there."""
    for device in (0, 1):
        _calls(device, Stream(device))[entry]()
        _refused(_calls(device, Stream(1 - device))[entry])
        for name in TAKES[entry]:
            _refused(_calls(device, Stream(device), **{name: 1 - device})[entry])
            _refused(_calls(device, Stream(device), **{name: -1})[entry])


def test_a_gradient_on_another_gpu():
    import torch
    from paper_2407_04272_amd import binding as b
    ty, K, N = torch.float16, 16, 8
    ok = [Stub(ty, N, K), Stub(ty, N)]
    cfg = b.make_dense_config(b.F16, 5, K, N)
    x, w, dy, work = Stub(ty, 5, K), Stub(ty, N, K), Stub(ty, 5, N), Stub(torch.uint8, 1 << 20)
    for dw, db in ((Stub(ty, N, K, device=1), ok[1]), (ok[0], Stub(ty, N, device=1))):
        _refused(b.dlc_linear_backward, cfg, x, w, None, dy, None, dw, db, work, stream=Stream())


def test_a_counter_on_another_gpu():
    import torch
    from paper_2407_04272_amd import binding as b
    for device in (0, 1):
        t = Stub(torch.int64, 1, device=device)
        y, cfg = Stub(torch.float32, 0, 8), b.make_dropout_config(b.F32, 0, 8, 0.5, d_offset=t)
        x, w, dense = Stub(torch.float32, 0, 4), Stub(torch.float32, 8, 4), b.make_dense_config(b.F32, 0, 4, 8, dropout_p=0.5, d_offset=t)
        calls = [lambda: b.dlc_dropout(cfg, y, None, y, stream=Stream()), lambda: b.dlc_linear_forward(dense, x, w, None, None, y, stream=Stream()),
                 lambda: b.dlc_linear_backward(dense, x, w, None, y, x, None, None, stream=Stream())]
        for call in calls:
            if device:
                _refused(call)
            else:
                call()


def test_results_that_no_launch_covers():
    from paper_2407_04272_amd import binding as b
    mk, size = b.make_dense_config, b.dlc_linear_workspace_bytes
    assert size(mk(b.F32, 1 << 30, 4, 128), True) > 0 and size(mk(b.F32, 1 << 30, 4, 129), True) == 0
    assert size(mk(b.F16, 1 << 30, 4, 768), True) > 0 and size(mk(b.F16, 1 << 30, 4, 769), True) == 0
    assert size(mk(b.F16, 64, 1 << 20, 1 << 20), True) == 0


def test_few_rows_on_boundaries_need_no_workspace():
    """Up to 32 rows, operands whose rows are on 16-byte boundaries: one pass over the weights, which has no partial sums."""
    from paper_2407_04272_amd import binding as b
    mk = b.make_dense_config
    for size in (b.dlc_linear_workspace_bytes, b.dlc_gated_workspace_bytes):
        for rows in (1, 16, 17, 32):
            assert size(mk(b.BF16, rows, 4096, 512)) == 0 and size(mk(b.F32, rows, 4096, 512, ld_x=4100, ld_w=4104)) == 0
            assert (size(mk(b.BF16, rows, 4096, 512, flags=b.DENSE_OFF_BOUNDARY)) > 0) == (rows > 16)
            assert (size(mk(b.BF16, rows, 4095, 512)) > 0) == (rows > 16) and (size(mk(b.BF16, rows, 4096, 512, ld_w=4099)) > 0) == (rows > 16)
        assert size(mk(b.BF16, 33, 4096, 512)) > 0
