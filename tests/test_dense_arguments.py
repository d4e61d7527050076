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
