"""Which kernel a product takes, from the rule's own header compiled for the host: the shapes that the GPU tests run reach every kernel there is."""
import ctypes
import os
import shutil
import subprocess

import pytest

import product_shapes as shapes
from paper_1708_04801_amd import build

KINDS = ["rows", "tile128", "tile256", "fast256"]
F32, BF16 = 1, 0


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("plan")
    source, lib = str(at / "plan.cc"), str(at / "plan.so")
    with open(source, "w") as f:
        f.write('#include "block_plan.h"\nextern "C" void plan(int64_t m, int64_t n, int64_t blocks, int f32, int wide_rows, int sums, int *o)\n{\n'
                "    const auto p = wpsgd::plan_matmul(m, n, blocks, f32 != 0, wide_rows != 0, sums != 0);\n    const auto r = wpsgd::rows_shape(m, n);\n"
                "    const int v[] = {(int)p.kind, p.parts, p.each, r.mt, r.nt, (int)r.turned};\n    for (int i = 0; i < 6; ++i) o[i] = v[i];\n}\n")
    subprocess.run([cxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + build.CSRC, source, "-o", lib], check=True)
    f = ctypes.CDLL(lib).plan
    f.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 3 + [ctypes.c_void_p]

    def call(m, n, k, f32, wide=False, sums=False):
        o = (ctypes.c_int * 6)()
        f(m, n, -(-k // 128), f32, wide, sums, o)
        return dict(kind=KINDS[o[0]], parts=o[1], each=o[2], sixteens=(o[3], o[4]), turned=bool(o[5]))
    return call


def test_few_rows(plan):
    for m, n, k, sixteens in shapes.ROWS:
        for f32 in (F32, BF16):
            p = plan(m, n, k, f32)
            assert p["kind"] == "rows" and p["sixteens"] == sixteens and p["turned"] == (m > n), (m, n, k)
    assert {s[3] for s in shapes.ROWS} == {(1, 1), (2, 1), (2, 2), (4, 1), (4, 2)}
    assert all({plan(m, n, k, F32)["turned"] for m, n, k, s in shapes.ROWS if s[1] == nt} == {True, False} for nt in (1, 2))


def test_tiles_of_128(plan):
    for m, n, k, parts in shapes.TILES_128:
        for f32 in (F32, BF16):
            p = plan(m, n, k, f32)
            assert p["kind"] == "tile128" and p["parts"] == parts, (m, n, k, p)


def test_tiles_of_256(plan):
    for m, n, k in shapes.TILES_256:
        assert plan(m, n, k, F32)["kind"] == "tile256", (m, n, k)
    for m, n, k in shapes.FAST_256:
        assert plan(m, n, k, BF16)["kind"] == "fast256", (m, n, k)
    # every remainder of the blocks by the loops' own steps, and remainders of rows by 256, 32 and 8
    assert {-(-k // 128) % 4 for _, _, k in shapes.FAST_256} == {-(-k // 128) % 4 for _, _, k in shapes.TILES_256} == {0, 1, 2, 3}
    assert min(-(-k // 128) for _, _, k in shapes.FAST_256) == 2


def test_parts_cover_the_sum(plan):
    for m in (65, 128, 300, 1000):
        for blocks in list(range(1, 70)) + [511, 512, 513, 4000]:
            for f32 in (F32, BF16):
                p = plan(m, m, blocks * 128, f32)
                if p["kind"] == "tile128":
                    assert (p["parts"] - 1) * p["each"] < blocks <= p["parts"] * p["each"] and (p["parts"] == 1 or p["each"] % 4 == 0)


def test_wide_rows_go_where_addresses_are_64_bits(plan):
    assert plan(5000, 5000, 4096, F32, wide=True)["kind"] == plan(5000, 5000, 4096, BF16, wide=True)["kind"] == "rows"


def test_sums_asked_for(plan):
    for m, n, k in shapes.FAST_256:
        assert plan(m, n, k, BF16, sums=True)["kind"] in ("tile128", "tile256")
    for m, n, k in shapes.SUMS_256:
        assert plan(m, n, k, BF16, sums=True)["kind"] == "tile256"
    for m, n, k in shapes.TILES_256:
        assert plan(m, n, k, F32, sums=True) == plan(m, n, k, F32) and plan(m, n, k, BF16, sums=True)["kind"] == "tile256"
