"""The gradients' norm and clipping against 64 bits."""
import math

import numpy as np
import pytest

from dense_util import F32, Guarded, assert_close, code, rounded, torch_type

pytestmark = pytest.mark.gpu
TYPES = ["f32", "f16", "bf16"]


def _tensors(shapes, types, seed=1, scale=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(torch.randn(s, generator=g, device="cuda") * scale).to(torch_type(types[i % len(types)])) for i, s in enumerate(shapes)]


def _norm(tensors, lst=None, stream=None):
    import torch
    from paper_2407_04272_amd import binding as b
    lst = lst or b.GradientList(tensors)
    total = torch.full((1,), -1.0, dtype=torch.float64, device="cuda")
    work = torch.empty(b.dlc_gradient_workspace_bytes(lst), dtype=torch.uint8, device="cuda")
    b.dlc_gradient_norm(lst, total, work, stream=stream)
    return lst, total


def _exact(tensors):
    return math.fsum(float((t.double() ** 2).sum()) for t in tensors)


def _check(tensors, max_norm, out=None):
    """clipped tensors are the originals times the factor, rounded once"""
    import torch
    from paper_2407_04272_amd import binding as b
    names = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}
    before = [t.clone() for t in tensors]
    lst, total = _norm(tensors)
    want = _exact(tensors)
    count = sum(t.numel() for t in tensors)
    assert abs(float(total) - want) <= want * (count + 64) * 2.0 ** -53
    n = torch.empty(1, device="cuda")
    b.dlc_gradient_clip(lst, total, max_norm, n, b.GradientList(out) if out else None)
    assert abs(float(n) - math.sqrt(want)) <= 2 * F32 * math.sqrt(want)
    f = max_norm / math.sqrt(want) if math.sqrt(want) > max_norm else 1.0
    for t, o in zip(before, out or tensors):
        if t.numel():
            v = t.double() * f
            assert_close(o, v, rounded(v, v.abs() * 2 * F32, names[t.dtype]), f"{tuple(t.shape)} {t.dtype}")
    if out:
        assert all(torch.equal(a, t) for a, t in zip(before, tensors))


SETS = {"one": [(1,)], "bias": [(7,)], "empty among": [(3, 5), (0,), (4, 0), (9,)], "layers": [(64, 33), (64,), (1, 64), (1,), (129, 257), (129,)],
        "large": [(2048, 1500), (2048,), (300000,)], "many": [(i % 13 + 1, i % 7 + 1) for i in range(200)], "border": [(32768,), (32769,), (65536,), (32767,)]}


@pytest.mark.parametrize("which", sorted(SETS))
@pytest.mark.parametrize("dtype", TYPES + ["mixed"])
def test_clip(which, dtype):
    types = TYPES if dtype == "mixed" else [dtype]
    for factor in (0.3, 2.0):
        t = _tensors(SETS[which], types, seed=len(which))
        limit = factor * math.sqrt(_exact(t))
        _check(t, limit)
        t = _tensors(SETS[which], types, seed=len(which))
        import torch
        _check(t, limit, [torch.full_like(v, 99.0) for v in t])


def test_rows_apart():
    import torch
    for dtype in TYPES:
        base = _tensors([(40, 70), (33, 9), (5,)], [dtype], 3)
        for ld, shift in ((70, 0), (83, 1)):
            g = [Guarded(40, 70, dtype, ld, shift).set(base[0]), Guarded(33, 9, dtype, 16, shift).set(base[1])]
            _check([g[0].view, g[1].view, base[2].clone()], 0.5)
            assert g[0].intact() and g[1].intact()
            g = [Guarded(40, 70, dtype, ld, shift).set(base[0]), Guarded(33, 9, dtype, 16, shift).set(base[1])]
            o = [Guarded(40, 70, dtype, 71, 3), Guarded(33, 9, dtype)]
            _check([g[0].view, g[1].view], 0.5, [o[0].view, o[1].view])
            assert o[0].intact() and o[1].intact()
        column = torch.randn((50, 4), device="cuda").to(torch_type(dtype))
        keep = column.clone()
        _check([column[:, 1], column[:, 2:3]], 0.1)
        assert torch.equal(column[:, 0], keep[:, 0]) and torch.equal(column[:, 3], keep[:, 3])
        three = torch.randn((4, 5, 6), device="cuda").to(torch_type(dtype))
        _check([three], 0.1)


def test_far_values():
    """Squares far outside fp32's range, and far below: the sum is 64-bit."""
    import torch
    big, small = torch.full((1000,), 1e30, device="cuda"), torch.full((1000,), 1e-30, device="cuda")
    _check([big.clone()], 1.0)
    _check([small.clone()], 1e-35)
    _check([small.clone(), big.clone()], 1.0)


def test_norms_that_are_not_finite():
    import torch
    from paper_2407_04272_amd import binding as b
    for bad in (float("inf"), -float("inf"), float("nan")):
        t = _tensors([(100,), (30, 30)], TYPES)
        t[1][3, 4] = bad
        before = [v.clone() for v in t]
        lst, total = _norm(t)
        n = torch.zeros(1, device="cuda")
        b.dlc_gradient_clip(lst, total, 0.5, n)
        assert math.isnan(float(n)) if math.isnan(bad) else float(n) == float("inf")
        assert all(torch.equal(a.nan_to_num(nan=5.0), v.nan_to_num(nan=5.0)) for a, v in zip(before, t))


def test_limits():
    import torch
    from paper_2407_04272_amd import binding as b
    t = _tensors([(100,)], ["f32"])
    before = t[0].clone()
    lst, total = _norm(t)
    b.dlc_gradient_clip(lst, total, float("inf"))
    assert torch.equal(t[0], before)
    b.dlc_gradient_clip(lst, total, 0.0)
    assert bool((t[0] == 0).all())
    lst, total = _norm(t)                     # all zeros: a norm of zero is within every limit
    b.dlc_gradient_clip(lst, total, 0.0)
    assert float(total) == 0.0 and bool((t[0] == 0).all())


def test_nothing_to_do():
    import torch
    from paper_2407_04272_amd import binding as b
    for t in ([], [torch.empty(0, device="cuda")]):
        lst, total = _norm(t)
        n = torch.full((1,), 7.0, device="cuda")
        b.dlc_gradient_clip(lst, total, 1.0, n)
        assert float(total) == 0.0 and float(n) == 0.0


def test_sums_do_not_depend_on_the_run():
    import torch
    t = _tensors([(1000, 1000), (77,), (123457,)], TYPES)
    first = [float(_norm(t)[1]) for _ in range(5)]
    assert len(set(first)) == 1


def test_parts_on_several_gpus_add_up():
    """The calls are apart so that sums can be added between them: two halves of a list clipped by their common norm."""
    import torch
    from paper_2407_04272_amd import binding as b
    a, c = _tensors([(50, 50), (9,)], ["f32"], 1), _tensors([(31, 31)], ["f32"], 2)
    want = _exact(a + c)
    (la, sa), (lc, sc) = _norm(a), _norm(c)
    both = sa + sc
    before = [v.clone() for v in a + c]
    b.dlc_gradient_clip(la, both, 0.7)
    b.dlc_gradient_clip(lc, both, 0.7)
    for v, t in zip(before, a + c):
        assert_close(t, v.double() * (0.7 / math.sqrt(want)), v.double().abs() * (0.7 / math.sqrt(want)) * 4 * F32, "part")


@pytest.mark.parametrize("sizes", [[(32768,)], [(32767,), (1,)], [(32768,), (1,)], [(512, 1)] * 64, [(512, 1)] * 65, [(8, 3), (0,), (100, 7), (20000,)], [(17,)] * 9])
def test_lists_that_one_work_group_adds_up(sizes):
    """... and the next larger ones"""
    for dtype in TYPES:
        _check(_tensors(sizes, [dtype], 71), 0.25)
        t = _tensors(sizes, [dtype], 72)
        assert len({float(_norm(t)[1]) for _ in range(3)}) == 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length,limit", [(3e31, 1e-9), (1e35, 1e-7), (1e20, 1e-25), (5e-20, 1e-44), (2.0, 1.5)])
def test_factors_far_below_one(length, limit, dtype):
    """Factors below fp32's normal range, with results that are not: off by the rounding of the result alone (what f loses in 64
    bits is far below; bf16 rounds a second time, from fp32)."""
    import torch
    t = _tensors([(1000,), (37, 5)], [dtype])
    t = [(v.double() * (length / 40.0)).to(v.dtype) for v in t]
    before = [v.clone() for v in t]
    from paper_2407_04272_amd import binding as b
    lst, total = _norm(t)
    b.dlc_gradient_clip(lst, total, limit)
    f = min(1.0, limit / math.sqrt(_exact(before)))
    for old, new in zip(before, t):
        v = old.double() * f
        assert_close(new, v, rounded(v, v.abs() * F32 + 2.0 ** -149 if dtype != "f32" else v.abs() * 2.0 ** -50, dtype), f"{length} {limit} {dtype}")


@pytest.mark.parametrize("where", ["in place", "elsewhere", "nothing to clip"])
def test_a_finite_norm_past_the_range_of_floats(where):
    """The gradients are clipped, and the norm that is stored says so: it is finite.  An infinite one says that they were not."""
    import torch
    from paper_2407_04272_amd import binding as b
    big = float(torch.finfo(torch.float32).max)
    t = [torch.full((100,), big, device="cuda"), torch.full((7, 9), -big / 2, dtype=torch.bfloat16, device="cuda")]
    before = [v.clone() for v in t]
    lst, total = _norm(t)
    n, exact = torch.zeros(1, device="cuda"), math.sqrt(_exact(before))
    assert exact > big
    if where == "nothing to clip":
        b.dlc_gradient_clip(b.GradientList([]), total, 1.0, n)
        assert float(n) == big
        return
    out = [torch.zeros_like(v) for v in t] if where == "elsewhere" else t
    b.dlc_gradient_clip(lst, total, 1.0, n, b.GradientList(out) if where == "elsewhere" else None)
    assert float(n) == big
    for old, new, name in zip(before, out, ("f32", "bf16")):
        v = old.double() / exact
        assert_close(new, v, rounded(v, v.abs() * F32, name), name)
    total.fill_(float("inf"))
    b.dlc_gradient_clip(lst, total, 1.0, n)
    assert float(n) == float("inf")
