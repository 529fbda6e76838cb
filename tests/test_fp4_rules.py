"""The rule that chooses the kernel and tile of a linear with 4-bit weights (csrc/lvx_fp4_rules.h, plain C++), evaluated on the CPU: the GPU tests' shapes
take every tile, with whole and ragged rows, columns and channels."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

import test_gpu_fp4_linear as gpu_tests

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_04677_amd", "csrc")
SOURCE = r"""
#include "lvx_fp4_rules.h"
extern "C" void plan(int mode, int M, int N, int K, int *out) {
    const lvx_fp4_plan_t p = lvx_fp4_plan(mode, M, N, K);
    out[0] = p.blocks, out[1] = p.groups;
}
extern "C" int resident(int bytes, int M, int N, int K) { return lvx_fp4_resident(bytes, M, N, K); }
extern "C" long long resident_bytes(int bytes, int M, int K, int nb) { return lvx_fp4_resident_bytes(bytes, M, K, nb); }
"""
BF16, WIDEN, NATIVE = 0, 1, 2


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    d = tmp_path_factory.mktemp("fp4_rules")
    (d / "rules.cpp").write_text(SOURCE)
    lib = str(d / "librules.so")
    r = subprocess.run([cxx, "-O1", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(d / "rules.cpp"), "-o", lib],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    so = C.CDLL(lib)

    def f(mode, M, N, K):
        out = (C.c_int * 2)()
        so.plan(mode, M, N, K, out)
        return tuple(out)
    so.resident_bytes.restype = C.c_longlong
    f.so = so
    return f


def test_every_tile_is_tested(plan):
    every = {BF16: {(2, 2), (1, 2), (1, 4)}, WIDEN: {(3, 2), (2, 2), (1, 2), (2, 4), (1, 4)}, NATIVE: {(3, 2), (2, 2), (1, 2), (2, 4), (1, 4)}}
    shapes = {s[:3] for s in gpu_tests.SHAPES + gpu_tests.TILES + gpu_tests.LONG + gpu_tests.FORMS}
    for mode, forms in every.items():
        seen = {plan(mode, *s) for s in shapes} - {(0, 0)}
        assert seen == forms, (mode, forms - seen)
        # every tile with a last step of fewer than 128 channels, and with more steps than the scales of one panel
        assert {plan(mode, *s) for s in gpu_tests.FORMS if s[2] % 128} >= forms
        assert {plan(mode, *s) for s in gpu_tests.FORMS if s[2] > 48 * 128} >= forms


def test_few_rows_and_small_products_take_no_tile(plan):
    for mode in (BF16, WIDEN, NATIVE):
        assert plan(mode, 1, 1 << 24, 128) == (0, 0) and plan(mode, 16, 15360, 5120) == (0, 0) and plan(mode, 100, 8, 32) == (0, 0)
        assert plan(mode, 1 << 20, 1 << 24, (1 << 31) - 32)[0] > 0


def test_rows_in_lds(plan):
    so = plan.so
    for (M, N, K), nb in gpu_tests.IN_LDS.items():
        assert (so.resident(2, M, N, K), so.resident(1, M, N, K)) == nb, (M, N, K)
    assert {n for pair in gpu_tests.IN_LDS.values() for n in pair} == {0, 1, 2, 4}
    for bytes_ in (1, 2):
        for M in range(1, 18):
            for K in list(range(4000 // 32 * 32, 200000, 1184)) + [(1 << 31) - 32]:
                for N in (8, 1280, 2568, 5120, 8200, 13824, 27648, 1 << 24):
                    nb = so.resident(bytes_, M, N, K)
                    # never more than a compute unit's LDS
                    assert nb == 0 or (M <= 16 and so.resident_bytes(bytes_, M, K, nb) <= 160 * 1024)


def test_rows_far_apart_take_no_tile(plan, tmp_path):
    (tmp_path / "call.cpp").write_text('#include "lvx_fp4_rules.h"\nextern "C" int blocks(int mode, int M, int N, int K, long long lda, long long ldw) '
                                       "{ return lvx_fp4_call_plan(mode, M, N, K, lda, ldw).blocks; }\n")
    lib = str(tmp_path / "libcall.so")
    subprocess.check_call([shutil.which("g++"), "-O1", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(tmp_path / "call.cpp"), "-o", lib])
    blocks = C.CDLL(lib).blocks
    blocks.argtypes = [C.c_int] * 4 + [C.c_longlong] * 2
    far, near = 1 << 24, (1 << 24) - 16
    for mode in (BF16, WIDEN, NATIVE):
        for M, N, K, *_ in gpu_tests.FAR_APART:
            assert blocks(mode, M, N, K, near, near) > 0 and blocks(mode, M, N, K, far, near) == 0 and blocks(mode, M, N, K, near, far) == 0
    # the largest offset of a tile: its last row or column, and the bytes of that
    assert 96 * near < 1 << 32 and 128 * near < 1 << 32
    # more than three blocks of rows beside few and many columns
    assert {(-(-M // 16) > 3, N >= 4096) for M, N, *_ in gpu_tests.FAR_APART} >= {(True, False), (True, True)}
