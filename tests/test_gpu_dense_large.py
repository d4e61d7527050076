"""Dense operators at the largest sizes that a card holds."""
import pytest

from dense_util import product, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_back():
    import torch
    yield
    torch.cuda.empty_cache()


def test_as_many_rows_as_there_may_be():
    """2^30 rows, one output: the result has more blocks of 64 rows than a launch has work-groups of 256 threads."""
    import torch
    from paper_2407_04272_amd import binding as b
    M, K = 1 << 30, 4
    step = 1 << 26
    x = torch.empty((M, K), device="cuda")
    for r in range(0, M, step):
        x[r:r + step].normal_()
    w = torch.randn((1, K), device="cuda")
    y = torch.empty((M, 1), device="cuda")
    cfg = b.make_dense_config(b.F32, M, K, 1)
    work = torch.empty(max(b.dlc_linear_workspace_bytes(cfg), b.dlc_linear_workspace_bytes(cfg, True)), dtype=torch.uint8, device="cuda")
    b.dlc_linear_forward(cfg, x, w, None, None, y, None, work)
    for r in range(0, M, step):
        v, e = product(x[r:r + step].double(), w.double())
        bad = ~((y[r:r + step].double() - v).abs() <= rounded(v, e, "f32"))
        assert not bool(bad.any()), r
    # the gradient of x: one product an element, rounded once
    dx = torch.empty_like(x)
    b.dlc_linear_backward(cfg, x, w, None, y, dx, None, None, work)
    for r in range(0, M, step):
        assert torch.equal(dx[r:r + step], y[r:r + step] * w), r


def test_no_rows_behind_many_weights():
    """No rows and 2^35 weights: their gradient is 0, and more than a launch's threads write it."""
    import torch
    from paper_2407_04272_amd import binding as b
    N, K = 1 << 15, 1 << 20
    dw = torch.empty((N, K), dtype=torch.float16, device="cuda")
    dw.fill_(1.0)
    db = torch.ones(N, dtype=torch.float16, device="cuda")
    x, dy = torch.empty((0, K), dtype=torch.float16, device="cuda"), torch.empty((0, N), dtype=torch.float16, device="cuda")
    b.dlc_linear_backward(b.make_dense_config(b.F16, 0, K, N), x, None, None, dy, None, dw, db)
    assert bool((db == 0).all())
    for r in range(0, N, 1 << 10):
        assert not bool(dw[r:r + (1 << 10)].any()), r
