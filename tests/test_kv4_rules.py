"""The rule that chooses the form of the attention over the 4-bit cache (csrc/lvx_kv4_rules.h, plain C++), evaluated on the CPU: the GPU tests' shapes
take the forms that those tests say they take, and no plan leaves its workspace."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_kv4 as gpu_tests

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_04677_amd", "csrc")
SOURCE = r"""
#include "lvx_kv4_rules.h"
extern "C" {
void plan(int n_seqs, int kv_heads, int max_keys, int n_heads, int max_tokens, int *out) {
    const lvx_kv4_plan_t p = lvx_kv4_plan(n_seqs, kv_heads, max_keys, n_heads, max_tokens);
    out[0] = p.rows, out[1] = p.row_tiles, out[2] = p.splits;
}
unsigned long long partial_rows(int n_seqs, int max_keys, int n_heads, int max_tokens) { return lvx_kv4_partial_rows(n_seqs, max_keys, n_heads, max_tokens); }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    d = tmp_path_factory.mktemp("kv4_rules")
    (d / "rules.cpp").write_text(SOURCE)
    lib = str(d / "librules.so")
    r = subprocess.run([cxx, "-O1", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(d / "rules.cpp"), "-o", lib],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    so = C.CDLL(lib)
    so.partial_rows.restype = C.c_ulonglong

    def plan(seqs, kv, keys, heads, tokens):
        out = (C.c_int * 3)()
        so.plan(seqs, kv, keys, heads, tokens, out)
        return tuple(out)
    return plan, so.partial_rows


def test_forms_of_the_gpu_tests(rules):
    forms = set()
    for S, KV, group, n, L, form, splits in gpu_tests.FORMS:
        rows, row_tiles, got = rules[0](S, KV, L, KV * group, n)
        assert (rows, got > 1) == (form, splits), (S, KV, group, n, L, rows, got)
        assert row_tiles == -(-n * group // rows)
        forms.add((form, splits))
    assert len(forms) >= 6 and {f for f, _ in forms} == {16, 32, 64, 128}


def test_plans_stay_inside_the_workspace(rules):
    rng = random.Random(3)
    for _ in range(20000):
        S, KV, group = (rng.choice((1, 1, 2, 3, 8, 40, 500, 65535)), rng.choice((1, 1, 2, 4, 8, 40, 1024)), rng.choice((1, 2, 5, 8, 16, 64)))
        n = int(2 ** rng.uniform(0, 20)) if rng.random() < 0.9 else rng.choice((1, 2 ** 29 // (KV * group)))
        L = int(2 ** rng.uniform(0, 26))
        rows, row_tiles, splits = rules[0](S, KV, L, KV * group, n)
        assert rows in (16, 32, 64, 128) and rows * row_tiles >= n * group > rows * (row_tiles - 1)
        assert 1 <= splits <= min(64, -(-L // 64)) and (splits == 1 or splits * row_tiles * KV * S <= 512)
        if splits > 1:
            assert splits * n * S * KV * group <= rules[1](S, L, KV * group, n) and n * KV * group < 1 << 24


def test_forms_of_the_in_place_tests(rules):
    for S, KV, group, n, L, form in gpu_tests.IN_PLACE:
        assert rules[0](S, KV, L, KV * group, n)[0] == form and 0 < n * group % min(form, 32) < group
    assert {f for *_, f in gpu_tests.IN_PLACE} == {16, 32, 64, 128}
