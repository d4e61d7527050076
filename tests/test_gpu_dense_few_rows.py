"""17 to 32 rows: a pass over the weights without a workspace, or tiles with one where operands are off 16-byte boundaries."""
import pytest

from dense_util import Guarded, assert_close, code, product, rounded, torch_type

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [17, 32])
def test_without_a_workspace_and_off_boundaries(M, dtype):
    import torch
    from paper_2407_04272_amd import binding as b
    K, N = 4096, 72
    g = torch.Generator(device="cuda")
    g.manual_seed(59)
    x = torch.randn((M, K), generator=g, device="cuda").to(torch_type(dtype))
    w = (torch.randn((N, K), generator=g, device="cuda") * K ** -0.5).to(torch_type(dtype))
    want, e = product(x.double(), w.double())
    bound = rounded(want, e, dtype)
    y = torch.empty((M, N), dtype=x.dtype, device="cuda")
    b.dlc_linear_forward(b.make_dense_config(code(dtype), M, K, N), x, w, None, None, y)
    assert_close(y, want, bound, "no workspace")
    # pointers off the boundary: with the flag there is room for copies and partial sums; without it a call with too little says
    # so, and one with a larger layer's workspace goes through
    off = [Guarded(*t.shape, dtype, shift=1).set(t).view for t in (x, w)]
    for xo, wo in (off, (off[0], w), (x, off[1])):
        cfg = b.make_dense_config(code(dtype), M, K, N, flags=b.DENSE_OFF_BOUNDARY)
        need = b.dlc_linear_workspace_bytes(cfg)
        work = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        y.zero_()
        b.dlc_linear_forward(cfg, xo, wo, None, None, y, None, work[:need])
        assert_close(y, want, bound, "off boundaries")
        assert bool((work[need:] == 0xFF).all())
        y.fill_(3.0)
        for small in (None, work[:16]):
            with pytest.raises(b.DlcError) as err:
                b.dlc_linear_forward(b.make_dense_config(code(dtype), M, K, N), xo, wo, None, None, y, None, small)
            assert err.value.status == b.ECAPACITY
        assert bool((y == 3.0).all())
        b.dlc_linear_forward(b.make_dense_config(code(dtype), M, K, N), xo, wo, None, None, y, None, work)
        assert_close(y, want, bound, "off boundaries, no flag")
