"""Host checks of the rules that choose a W8A8 product's kernel (CPU): the
plain C++ functions that the launcher uses, compiled with the host compiler."""
import ctypes as C
import os
import subprocess

import pytest

from tests import test_gpu_w8a8 as gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_28803_amd", "csrc")

SOURCE = r"""
#include "gemm_rules.h"
extern "C" int tiling(int64_t M, int64_t N, int64_t K) { return oq::w8_tiling(M, N, K); }
extern "C" bool few(int64_t M, int64_t N) { return oq::w8_few_rows(M, N); }
extern "C" int64_t split(int64_t M, int64_t N, int64_t K, bool* columns) {
  const oq::W8Split s = oq::w8_split(M, N, K);
  *columns = s.columns;
  return s.at;
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("w8rules")
    src, so = d / "rules.cpp", d / "rules.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.tiling.argtypes = [C.c_int64] * 3
    lib.few.argtypes, lib.few.restype = [C.c_int64] * 2, C.c_bool
    lib.split.argtypes, lib.split.restype = [C.c_int64] * 3 + [C.POINTER(C.c_bool)], C.c_int64
    return lib


# (M, N, K, us with each tiling, in one launch), measured on an MI355X in graphs of many calls that
# rotate through more weights than the caches hold.
TIMES = [
    (128, 4096, 4096, [46.08, 24.05, 21.80, 14.14, 11.71]), (256, 8192, 8192, [102.64, 62.86, 56.68, 40.39, 42.03]),
    (512, 2048, 4096, [46.40, 24.15, 22.00, 14.45, 12.14]), (816, 2560, 2048, [27.91, 15.15, 14.89, 13.95, 18.44]),
    (816, 2048, 16384, [169.78, 108.02, 98.28, 59.51, 61.62]), (816, 32768, 2048, [74.48, 79.04, 95.71, 101.48, 145.19]),
    (1024, 1536, 6144, [65.96, 34.17, 30.63, 22.70, 26.23]), (1024, 6144, 1536, [24.57, 17.29, 17.84, 20.50, 28.51]),
    (1024, 4608, 1536, [23.90, 15.66, 16.29, 17.38, 24.14]), (2000, 6144, 1536, [27.01, 27.38, 30.36, 36.02, 52.95]),
    (4000, 4096, 4096, [67.44, 79.33, 99.04, 111.19, 139.84]), (4080, 2048, 16384, [193.31, 139.70, 210.63, 219.95, 251.65]),
    (4080, 4096, 1024, [25.18, 26.71, 30.58, 35.63, 57.78]), (4096, 8192, 8192, [234.16, 284.64, 362.83, 438.06, 527.64]),
    (16384, 4096, 4096, [248.35, 300.68, 356.44, 432.72, 545.00]),
    (16384, 8192, 8192, [920.31, 1113.19, 1329.90, 1664.30, 2025.95]), (1100, 32768, 128, [32.22, 26.01, 29.30, 33.81, 89.10]),
    (6000, 6000, 4096, [165.42, 163.20, 193.91, 236.56, 299.71]), (5000, 3000, 2048, [36.98, 40.50, 46.55, 54.56, 77.50]),
    (2100, 32768, 2048, [165.38, 174.93, 210.48, 251.58, 362.17]), (9000, 5000, 1024, [67.75, 70.17, 76.88, 95.13, 152.35]),
    (65, 16384, 4096, [51.39, 34.88, 31.38, 23.73, 25.82]), (300, 2048, 8192, [83.49, 42.48, 38.08, 23.20, 18.03]),
    (2048, 2048, 2048, [28.70, 17.07, 16.39, 19.19, 24.10]), (4000, 8200, 8192, [308.83, 322.53, 359.11, 429.71, 513.44]),
]


@pytest.mark.parametrize("M,N,K,us", TIMES)
def test_rule_takes_a_fast_tiling(rules, M, N, K, us):
    assert us[rules.tiling(M, N, K)] <= 1.12 * min(us)


# (M, N, K, us on the small-M kernel, us on the ring), measured as above.
FEW = [(1, 2560, 2048, 5.36, 7.36), (1, 16384, 16384, 53.0, 58.3), (8, 8192, 1024, 5.34, 6.28), (16, 2048, 8192, 10.6, 16.9),
       (16, 5000, 8192, 14.5, 17.4), (16, 32768, 4096, 33.5, 34.9), (17, 8200, 4096, 13.5, 11.1), (17, 32768, 2048, 19.1, 17.3),
       (17, 2048, 16384, 19.8, 29.3), (32, 2560, 2048, 6.41, 7.61), (32, 4096, 4096, 9.2, 10.7), (32, 2048, 16384, 24.6, 29.3), (40, 4096, 4096, 10.88, 10.81),
       (48, 2048, 8192, 18.8, 16.9), (64, 32768, 2048, 31.8, 19.2), (20, 8192, 1536, 7.69, 7.13)]


@pytest.mark.parametrize("M,N,K,small,ring", FEW)
def test_few_row_rule_takes_the_faster_kernel(rules, M, N, K, small, ring):
    assert rules.few(M, N) == (small < ring)


def test_split_takes_whole_rounds(rules):
    col = C.c_bool()
    assert rules.split(4000, 8200, 8192, C.byref(col)) == 8192 and col.value
    assert rules.split(8200, 4000, 8192, C.byref(col)) == 8192 and not col.value
    for shape in ((16384, 8192, 8192), (4096, 4096, 4096), (816, 32768, 2048), (816, 2560, 2048), (9000, 5000, 1024)):
        assert rules.split(*shape, C.byref(col)) == 0
    # The parts of a split: whole 256-wide tiles, then the rest, which is not split again for ever.
    for M, N in ((4100, 4096), (4096, 4104), (5000, 9000), (20000, 4100)):
        for K in (512, 4096, 16384):
            at = rules.split(M, N, K, C.byref(col))
            assert at % 256 == 0 and 0 <= at < (N if col.value else M)


def test_gpu_shapes_cover_every_kernel(rules):
    """Each kernel, each tiling and both ways to split have a shape among the GPU tests'."""
    col = C.c_bool()
    seen = set()
    for M, N, K in gpu.CASES:
        if rules.few(M, N):
            seen.add(("small", K % 128 == 64, M > 16))
        elif rules.split(M, N, K, C.byref(col)):
            seen.add(("split", bool(col.value)))
        else:
            seen.add(rules.tiling(M, N, K))
    assert seen >= {0, 1, 2, 3, 4, ("split", True), ("split", False), ("small", True, False), ("small", False, False), ("small", False, True),
                    ("small", True, True)}, seen
