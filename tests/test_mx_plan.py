"""Which kernel the product of microscaled operands takes: the sizes that the GPU tests use for each of them, asked of the plan's own
source, which is host code.  A change of the measured costs that moves a size to another kernel fails here."""
import ctypes as C
import os
import subprocess

import pytest

from mx_util import CUTS, KINDS, TILES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """#include "dlc_mx_plan.h"
extern "C" void plan(int64_t m, int64_t k, int64_t n, int e4m3, int fp32, int64_t* out) {
    const dlc::MxPlan p = dlc::mx_plan(m, k, n, e4m3 != 0, fp32 != 0);
    const int64_t v[] = {p.tile, p.split, p.kper, (int64_t)p.bytes};
    for (int i = 0; i < 4; ++i) out[i] = v[i];
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    folder = tmp_path_factory.mktemp("plan")
    src, lib = folder / "plan.cpp", folder / "plan.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2407_04272_amd", "csrc"),
                    "-o", str(lib), str(src)], check=True)
    f = C.CDLL(str(lib)).plan
    f.argtypes = [C.c_int64] * 3 + [C.c_int] * 2 + [C.POINTER(C.c_int64)]

    def ask(rows, n_in, n_out, bits, fp32):
        out = (C.c_int64 * 4)()
        f(rows, n_in, n_out, int(bits == 8), int(fp32), out)
        return tuple(out)
    return ask


def _fp32(kind):
    """results in fp32: the plan tells them apart for E4M3 rows only"""
    return (False,) if kind == "E4M3" else (True,) if kind == "E4M3 f32" else (False, True)


@pytest.mark.parametrize("kind,tile,split,rows,n_out,lengths", TILES + CUTS, ids=lambda v: str(v).replace(" ", "") if not isinstance(v, tuple) else "")
def test_sizes_take_the_tile_that_they_stand_for(plan, kind, tile, split, rows, n_out, lengths):
    for n_in in lengths:
        for fp32 in _fp32(kind):
            assert plan(rows, n_in, n_out, KINDS[kind][0], fp32)[:2] == (tile, split), n_in


def test_every_tile_is_there_and_every_length(plan):
    for cases, cut in ((TILES, False), (CUTS, True)):
        assert {(k, t) for k, t, *_ in cases} == {("E2M1", 0), ("E2M1", 1), ("E2M1", 2), ("E4M3", 0), ("E4M3", 1), ("E4M3", 2), ("E4M3 f32", 1), ("E4M3 f32", 2)}
        assert all((split > 1) == cut for _, _, split, *_ in cases)
    for kind, tile in {(k, t) for k, t, *_ in TILES}:
        lengths = [n for k, t, _, _, _, ls in TILES if (k, t) == (kind, tile) for n in ls]
        assert {-(-n // 256) % 4 for n in lengths} == {0, 1, 2, 3}                          # the loop's turns of four tiles, and every rest
        assert {-(-n // 128) % 4 for n in lengths} == {0, 1, 2, 3}
        assert any(n % 128 for n in lengths) and any(0 < n % 256 <= 128 for n in lengths) and any(n % 256 > 128 for n in lengths)


def test_few_rows_and_the_parts_of_a_cut(plan):
    for rows in (1, 16):
        for n_in, n_out in ((1, 1), (8192, 2048), (1 << 20, 1 << 20)):
            for bits in (4, 8):
                assert plan(rows, n_in, n_out, bits, False)[:2] == (3, 1)
    for kind, _, split, rows, n_out, lengths in CUTS:
        for n_in in lengths:
            _, parts, kper, size = plan(rows, n_in, n_out, KINDS[kind][0], _fp32(kind)[0])
            assert kper % 512 == 0 and (parts - 1) * kper < n_in <= parts * kper and size == parts * rows * -(-n_out // 8) * 8 * 4
